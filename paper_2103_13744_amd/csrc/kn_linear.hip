// Products grouped by network with ragged sizes, and their gradients: kn_grouped_linear, kn_grouped_linear_dx,
// kn_grouped_linear_dw.
#include "kn_experts.h"

namespace {

constexpr int ANY_TILE = 64, ANY_STEP = 32;

// Any sizes, strides and alignment: values are fetched one by one, checked one by one, and laid out in the LDS with the
// contraction contiguous, so that a fragment is 8 neighbours of a row.  A workgroup of four wavefronts makes 64 x 64 results,
// each wavefront 32 x 32 of them as 2 x 2 products of 16 x 16.  REDUCE: the weight gradient, whose contraction is the group.
template <typename T, bool REDUCE>
__global__ void __launch_bounds__(256) k_product_any(KnProduct p)
{
    constexpr int W = sizeof(T) == 4 ? 4 : 8;       // values of a fragment
    constexpr int LD = ANY_STEP + 16 / sizeof(T);   // (a row more by 16 bytes: fragments of 16 rows spread over the banks)
    typedef T Frag __attribute__((ext_vector_type(W)));
    __shared__ __align__(16) T as[ANY_TILE * LD];
    __shared__ __align__(16) T bs[ANY_TILE * LD];
    const int tid = kn_thread(), lane = tid & 63, wave = tid >> 6;
    const int ntiles = (p.J + ANY_TILE - 1) / ANY_TILE;
    const int number = kn_block() / ntiles, j0 = (kn_block() % ntiles) * ANY_TILE;
    int32_t group, i0, iend, c0, cend;
    if constexpr (REDUCE) {
        const int itiles = (p.I + ANY_TILE - 1) / ANY_TILE;
        group = number / itiles;
        i0 = (number % itiles) * ANY_TILE;
        iend = p.I;
        c0 = kn_offset(p.offsets, group, p.M);
        cend = max(c0, kn_offset(p.offsets, group + 1, p.M));
    } else {
        const KnPiece piece = kn_find_piece(p.offsets, p.E, p.M, ANY_TILE, number);
        group = piece.group;
        i0 = piece.begin;
        iend = piece.end;
        c0 = 0;
        cend = group < p.E ? p.C : 0; // (rows without a network: zeros)
        if (i0 >= iend) return;
    }
    const T *a = (const T *)p.a, *b = (const T *)p.b;
    if constexpr (!REDUCE) b += (int64_t)group * p.b_group; // (group E: b is not read)
    const int wi = (wave >> 1) * 32, wj = (wave & 1) * 32;
    kn_f32x4 acc[2][2] = {};
    float colsum = 0.0f; // REDUCE with out_bias: thread j < 64 of a workgroup with i0 = 0 sums its column
    for (; c0 < cend; c0 += ANY_STEP) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < ANY_TILE * ANY_STEP / 256; ++t) {
            const int q = tid + 256 * t;
            // neighbouring threads take neighbouring values in memory
            int i, c;
            if constexpr (REDUCE) { i = q % ANY_TILE; c = q / ANY_TILE; } else { c = q % ANY_STEP; i = q / ANY_STEP; }
            T v = (T)0.0f;
            if (i0 + i < iend && c0 + c < cend) {
                const int32_t r = REDUCE ? c0 + c : i0 + i;
                const int32_t src = p.rows ? p.rows[r] : r;
                if ((uint32_t)src < (uint32_t)p.a_rows) v = a[(int64_t)src * p.lda + (REDUCE ? i0 + i : c0 + c)];
            }
            as[i * LD + c] = v;
            int j, d;
            if (REDUCE || p.b_j == 1) { j = q % ANY_TILE; d = q / ANY_TILE; } else { d = q % ANY_STEP; j = q / ANY_STEP; }
            T w = (T)0.0f;
            if (j0 + j < p.J && c0 + d < cend)
                w = REDUCE ? b[(int64_t)(c0 + d) * p.ldb + j0 + j] : b[(int64_t)(c0 + d) * p.b_c + (int64_t)(j0 + j) * p.b_j];
            bs[j * LD + d] = w;
        }
        __syncthreads();
        if constexpr (REDUCE)
            if (p.out_bias && i0 == 0 && tid < ANY_TILE)
                for (int c = 0; c < ANY_STEP; ++c) colsum += (float)bs[tid * LD + c];
#pragma unroll
        for (int c = 0; c < ANY_STEP; c += 4 * W) {
            Frag fa[2], fb[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                fa[u] = *(const Frag *)(as + (wi + 16 * u + (lane & 15)) * LD + c + (lane >> 4) * W);
                fb[u] = *(const Frag *)(bs + (wj + 16 * u + (lane & 15)) * LD + c + (lane >> 4) * W);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int v = 0; v < 2; ++v) acc[u][v] = kn_mfma(fa[u], fb[v], acc[u][v]);
        }
    }
    T *out = (T *)p.out;
    const T *bias = (const T *)p.bias, *mask = (const T *)p.mask;
    if constexpr (REDUCE) {
        out += (int64_t)group * p.o_group;
        if (p.out_bias && i0 == 0 && tid < ANY_TILE && j0 + tid < p.J) ((T *)p.out_bias)[(int64_t)group * p.J + j0 + tid] = (T)colsum;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int32_t i = i0 + wi + 16 * u + (lane >> 4) * 4 + r, j = j0 + wj + 16 * v + (lane & 15);
                if (i >= iend || j >= p.J) continue;
                float y = acc[u][v][r];
                if constexpr (!REDUCE) {
                    if (group < p.E) {
                        if (bias) y += (float)bias[(int64_t)group * p.J + j];
                        if (p.relu) y = y > 0.0f || y != y ? y : 0.0f; // (a NaN stays one)
                        if (mask) {
                            const int32_t src = p.mask_rows ? p.mask_rows[i] : i;
                            if ((uint32_t)src >= (uint32_t)p.m_rows || !((float)mask[(int64_t)src * p.ldm + j] > 0.0f)) y = 0.0f;
                        }
                    }
                }
                out[(int64_t)i * p.o_i + (int64_t)j * p.o_j] = (T)y;
            }
}

template <typename T, bool REDUCE> int launch_any(hipStream_t st, const KnProduct &p)
{
    const int64_t groups = REDUCE ? (int64_t)p.E * kn_div_up(p.I, ANY_TILE) : kn_pieces(p.M, p.E, ANY_TILE);
    const int64_t blocks = groups * kn_div_up(p.J, ANY_TILE);
    if (blocks > 0x7fffffffLL) return KN_E_UNSUPPORTED;
    hipLaunchKernelGGL((k_product_any<T, REDUCE>), dim3((unsigned)blocks), dim3(256), 0, st, p);
    KN_CHECK_LAUNCH();
    return KN_OK;
}

// What the three calls check alike
int check(const kn_linear_desc *d)
{
    if (!d || d->rows < 0 || d->x_rows < 0 || d->experts < 1 || d->n_in < 1 || d->n_out < 1 || !kn_dtype_ok(d->dtype) ||
        (d->w_layout != KN_W_IN_OUT && d->w_layout != KN_W_OUT_IN) || d->ldx < d->n_in)
        return KN_E_INVALID_ARG;
    if (d->rows > KN_MAX_ROWS || d->x_rows > KN_MAX_ROWS || d->experts > KN_MAX_EXPERTS || d->n_in > KN_MAX_WIDTH || d->n_out > KN_MAX_WIDTH)
        return KN_E_UNSUPPORTED;
    return KN_OK;
}

} // namespace

extern "C" int kn_grouped_linear(void *stream, const kn_linear_desc *d, const void *x, const void *w, const void *bias,
                                 const int32_t *offsets, const int32_t *rows, int32_t relu, void *y)
{
    KN_TRY(check(d));
    if (d->rows == 0) return KN_OK;
    if (!w || !offsets || !y || (d->x_rows > 0 && !x) || (!rows && d->x_rows < d->rows)) return KN_E_INVALID_ARG;
    KnProduct p = {};
    const bool io = d->w_layout == KN_W_IN_OUT;
    p.a = x; p.b = w; p.bias = bias; p.out = y; p.offsets = offsets; p.rows = rows;
    p.lda = d->ldx;
    p.b_group = (int64_t)d->n_in * d->n_out; p.b_c = io ? d->n_out : 1; p.b_j = io ? 1 : d->n_in;
    p.o_i = d->n_out; p.o_j = 1;
    p.M = (int32_t)d->rows; p.E = d->experts; p.J = d->n_out; p.C = d->n_in;
    p.a_rows = (int32_t)d->x_rows; p.relu = relu != 0;
    return kn_with_type(d->dtype, [&](auto v) { return launch_any<decltype(v), false>((hipStream_t)stream, p); });
}

extern "C" int kn_grouped_linear_dx(void *stream, const kn_linear_desc *d, const void *dy, const void *w, const void *x_relu,
                                    const int32_t *offsets, const int32_t *rows, void *dx)
{
    KN_TRY(check(d));
    if (d->rows == 0) return KN_OK;
    if (!dy || !w || !offsets || !dx || (x_relu && !rows && d->x_rows < d->rows)) return KN_E_INVALID_ARG;
    KnProduct p = {};
    const bool io = d->w_layout == KN_W_IN_OUT;
    p.a = dy; p.b = w; p.mask = x_relu; p.out = dx; p.offsets = offsets; p.rows = nullptr;
    p.lda = d->n_out; p.ldm = d->ldx;
    p.b_group = (int64_t)d->n_in * d->n_out; p.b_c = io ? 1 : d->n_in; p.b_j = io ? d->n_out : 1;
    p.o_i = d->n_in; p.o_j = 1;
    p.M = (int32_t)d->rows; p.E = d->experts; p.J = d->n_in; p.C = d->n_out;
    p.a_rows = p.M; p.m_rows = (int32_t)d->x_rows;
    p.mask_rows = x_relu ? rows : nullptr;
    return kn_with_type(d->dtype, [&](auto v) { return launch_any<decltype(v), false>((hipStream_t)stream, p); });
}

extern "C" int kn_grouped_linear_dw(void *stream, const kn_linear_desc *d, const void *x, const void *dy, const int32_t *offsets,
                                    const int32_t *rows, void *dw, void *db)
{
    KN_TRY(check(d));
    if (!offsets || !dw || (d->rows > 0 && (!dy || (d->x_rows > 0 && !x))) || (d->rows > 0 && !rows && d->x_rows < d->rows)) return KN_E_INVALID_ARG;
    KnProduct p = {};
    const bool io = d->w_layout == KN_W_IN_OUT;
    p.a = x; p.b = dy; p.out = dw; p.out_bias = db; p.offsets = offsets; p.rows = rows;
    p.lda = d->ldx; p.ldb = d->n_out;
    p.o_group = (int64_t)d->n_in * d->n_out; p.o_i = io ? d->n_out : 1; p.o_j = io ? 1 : d->n_in;
    p.M = (int32_t)d->rows; p.E = d->experts; p.I = d->n_in; p.J = d->n_out;
    p.a_rows = (int32_t)d->x_rows;
    return kn_with_type(d->dtype, [&](auto v) { return launch_any<decltype(v), true>((hipStream_t)stream, p); });
}
