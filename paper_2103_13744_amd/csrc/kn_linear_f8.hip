// Products grouped by network in 8-bit floating point (e4m3) with fp32 scales: kn_quantize_f8 (a scale per row and 128 inputs),
// kn_quantize_f8_weights (a scale per 128 x 128), kn_grouped_linear_f8.
#include "kn_experts.h"

namespace {

constexpr int F8_BLOCK = 128;
constexpr float F8_LARGEST = 448.0f, F8_TINY = 0x1p-100f;

// Scale of a block whose largest magnitude is `amax`, and a value's 8 bits: x / s is at most 448 but for the last bit of the
// quotient, which rounds to 448.  Both are divisions, not products with a reciprocal: the nearest e4m3 of the exact quotient's
// fp32 form.  A block of zeros keeps a finite scale.
__device__ __forceinline__ float f8_scale(float amax) { return fmaxf(amax, F8_TINY) / F8_LARGEST; }
__device__ __forceinline__ uint32_t f8_pack(float a, float b, float c, float d, float s)
{
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a / s, b / s, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c / s, d / s, v, true);
}
__device__ __forceinline__ float f8_row_max(float v)
{
    constexpr int ROW_ROR = 0x120; // dpp_ctrl encoding: rotation inside 16 lanes
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 8, 0xf, 0xf, false)));
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 4, 0xf, 0xf, false)));
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 2, 0xf, 0xf, false)));
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 1, 0xf, 0xf, false)));
}

// 16 lanes per row and block of 128 inputs, 8 values a lane.  Inputs beyond K are zeros.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) k_quantize_rows(const T *__restrict__ x, int64_t R, int32_t K, int64_t ld, int32_t kb,
                                                       uint8_t *__restrict__ q, float *__restrict__ scales)
{
    const int64_t g = ((int64_t)kn_block() * 256 + kn_thread()) >> 4;
    if (g >= R * kb) return;
    const int at = kn_thread() & 15;
    const int64_t row = g / kb;
    const int32_t blk = (int32_t)(g % kb), k0 = blk * F8_BLOCK + at * 8;
    float v[8];
    const T *src = x + row * ld + k0;
    if (WIDE && k0 + 8 <= K) {
        typedef T Piece __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
        for (int i = 0; i < 8; i += 16 / (int)sizeof(T)) {
            const Piece p = *(const Piece *)(src + i);
#pragma unroll
            for (int j = 0; j < 16 / (int)sizeof(T); ++j) v[i + j] = (float)p[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = k0 + i < K ? (float)src[i] : 0.0f;
    }
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(v[i]));
    const float s = f8_scale(f8_row_max(amax));
    uint2 out;
    out.x = f8_pack(v[0], v[1], v[2], v[3], s);
    out.y = f8_pack(v[4], v[5], v[6], v[7], s);
    *(uint2 *)(q + row * kb * F8_BLOCK + k0) = out;
    if (at == 0) scales[g] = s;
}

// One workgroup per 128 x 128 block of a network's weights, through the LDS (the two layouts differ in which index is next to
// which).  Outputs beyond N are not stored, inputs beyond K are zeros.
template <typename T>
__global__ void __launch_bounds__(256) k_quantize_weights(const T *__restrict__ w, int32_t N, int32_t K, int64_t s_n, int64_t s_k, int32_t nb,
                                                          int32_t kb, uint8_t *__restrict__ q, float *__restrict__ scales)
{
    constexpr int LD = F8_BLOCK + 1;
    __shared__ float t[F8_BLOCK / 2 * LD]; // half a block at a time
    __shared__ float part[4];
    const int64_t blk = kn_block();
    const int32_t bk = (int32_t)(blk % kb), bn = (int32_t)(blk / kb % nb);
    const int64_t e = blk / kb / nb;
    const T *src = w + e * N * K;
    float amax = 0.0f;
    for (int i = kn_thread(); i < F8_BLOCK * F8_BLOCK; i += 256) {
        const int32_t n = bn * F8_BLOCK + (s_n == 1 ? i % F8_BLOCK : i / F8_BLOCK), k = bk * F8_BLOCK + (s_n == 1 ? i / F8_BLOCK : i % F8_BLOCK);
        if (n < N && k < K) amax = fmaxf(amax, fabsf((float)src[n * s_n + k * s_k]));
    }
    amax = f8_row_max(amax);
    amax = fmaxf(amax, __shfl_xor(amax, 16));
    amax = fmaxf(amax, __shfl_xor(amax, 32));
    if ((kn_thread() & 63) == 0) part[kn_thread() >> 6] = amax;
    __syncthreads();
    const float s = f8_scale(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
    if (kn_thread() == 0) scales[blk] = s;
    for (int half = 0; half < 2; ++half) { // 64 outputs each
        __syncthreads();
        for (int i = kn_thread(); i < F8_BLOCK / 2 * F8_BLOCK; i += 256) {
            const int ln = s_n == 1 ? i % 64 : i / F8_BLOCK, lk = s_n == 1 ? i / 64 : i % F8_BLOCK;
            const int32_t n = bn * F8_BLOCK + half * 64 + ln, k = bk * F8_BLOCK + lk;
            t[ln * LD + lk] = n < N && k < K ? (float)src[n * s_n + k * s_k] : 0.0f;
        }
        __syncthreads();
        for (int i = kn_thread(); i < 64 * F8_BLOCK / 4; i += 256) {
            const int ln = i / 32, lk = i % 32 * 4;
            const int32_t n = bn * F8_BLOCK + half * 64 + ln;
            const float *v = t + ln * LD + lk;
            if (n < N) *(uint32_t *)(q + (e * N + n) * kb * F8_BLOCK + bk * F8_BLOCK + lk) = f8_pack(v[0], v[1], v[2], v[3], s);
        }
    }
}

struct F8Args {
    const uint8_t *x, *w;
    const float *xs, *ws;
    const void *bias;
    void *y;
    const int32_t *offsets, *rows;
    int32_t M, E, N, kb, x_rows, relu;
};

// 128 x 128 results per workgroup of four wavefronts, 64 x 64 each; a step is a block of 128 inputs, which is one instruction's
// contraction, so that every product starts from zero and is scaled, in fp32, as it is added.
template <typename T>
__global__ void __launch_bounds__(256) k_linear_f8(F8Args p)
{
    constexpr int TILE = 128;
    __shared__ kn_u32x4 as[TILE * 8], bs[TILE * 8]; // rows of 128 bytes; 16-byte piece c of row r lies at c ^ (r & 7)
    __shared__ float sa[TILE];
    const int tid = kn_thread(), lane = tid & 63, wave = tid >> 6;
    const int ntiles = (p.N + TILE - 1) / TILE;
    const KnPiece piece = kn_find_piece(p.offsets, p.E, p.M, TILE, kn_block() / ntiles);
    const int j0 = (kn_block() % ntiles) * TILE;
    if (piece.begin >= piece.end) return;
    const int64_t kp = (int64_t)p.kb * F8_BLOCK;
    const bool some = piece.group < p.E;
    const int64_t group = some ? piece.group : 0;
    const uint8_t *arow[4], *brow[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) { // thread's pieces: row t * 32 + tid / 8, 16 bytes tid % 8
        const int r = t * 32 + tid / 8;
        const int32_t i = piece.begin + r;
        int32_t src = -1;
        if (i < piece.end) src = p.rows ? p.rows[i] : i;
        arow[t] = (uint32_t)src < (uint32_t)p.x_rows ? p.x + src * kp + tid % 8 * 16 : nullptr;
        brow[t] = j0 + r < p.N ? p.w + (group * p.N + j0 + r) * kp + tid % 8 * 16 : nullptr;
    }
    int32_t srow = -1; // threads 0 .. 127: the row whose scale they fetch
    if (tid < TILE && piece.begin + tid < piece.end) {
        srow = p.rows ? p.rows[piece.begin + tid] : piece.begin + tid;
        if ((uint32_t)srow >= (uint32_t)p.x_rows) srow = -1;
    }
    const float *ws = p.ws + (group * ntiles + j0 / TILE) * p.kb;
    const int wi = (wave >> 1) * 64, wj = (wave & 1) * 64;
    kn_f32x4 acc[4][4] = {};
    for (int b = 0; b < (some ? p.kb : 0); ++b) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int r = t * 32 + tid / 8, at = r * 8 + ((tid & 7) ^ (r & 7));
            as[at] = arow[t] ? *(const kn_u32x4 *)(arow[t] + b * F8_BLOCK) : kn_u32x4{0, 0, 0, 0};
            bs[at] = brow[t] ? *(const kn_u32x4 *)(brow[t] + b * F8_BLOCK) : kn_u32x4{0, 0, 0, 0};
        }
        if (tid < TILE) sa[tid] = srow >= 0 ? p.xs[(int64_t)srow * p.kb + b] * ws[b] : 0.0f;
        __syncthreads();
        union Frag { kn_u32x4 h[2]; kn_i32x8 v; } fa[4], fb[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int ra = wi + 16 * u + (lane & 15), rb = wj + 16 * u + (lane & 15), c = lane >> 4;
            fa[u].h[0] = as[ra * 8 + (c ^ (ra & 7))];
            fa[u].h[1] = as[ra * 8 + ((c + 4) ^ (ra & 7))];
            fb[u].h[0] = bs[rb * 8 + (c ^ (rb & 7))];
            fb[u].h[1] = bs[rb * 8 + ((c + 4) ^ (rb & 7))];
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const kn_f32x4 s = *(const kn_f32x4 *)(sa + wi + 16 * u + (lane >> 4) * 4);
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const kn_f32x4 r = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fa[u].v, fb[v].v, kn_f32x4{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[u][v][i] = fmaf(r[i], s[i], acc[u][v][i]);
            }
        }
    }
    T *y = (T *)p.y;
    const T *bias = (const T *)p.bias;
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int32_t i = piece.begin + wi + 16 * u + (lane >> 4) * 4 + r, j = j0 + wj + 16 * v + (lane & 15);
                if (i >= piece.end || j >= p.N) continue;
                float o = acc[u][v][r];
                if (some) {
                    if (bias) o += (float)bias[group * p.N + j];
                    if (p.relu) o = o > 0.0f || o != o ? o : 0.0f;
                }
                y[(int64_t)i * p.N + j] = (T)o;
            }
}

} // namespace

extern "C" int kn_quantize_f8(void *stream, const void *x, int32_t dtype, int64_t R, int32_t K, int64_t ld, void *q, float *scales)
{
    if (R < 0 || K < 1 || ld < K || !kn_dtype_ok(dtype) || (R > 0 && (!x || !q || !scales)) || ((uintptr_t)q & 15)) return KN_E_INVALID_ARG;
    if (R > KN_MAX_ROWS || K > KN_MAX_WIDTH) return KN_E_UNSUPPORTED;
    if (R == 0) return KN_OK;
    const int32_t kb = (int32_t)kn_div_up(K, F8_BLOCK);
    const int64_t blocks = kn_div_up(R * kb, 16);
    if (blocks > 0x7fffffffLL) return KN_E_UNSUPPORTED;
    const bool wide = ((uintptr_t)x & 15) == 0 && ld * kn_item(dtype) % 16 == 0;
    return kn_with_type(dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        auto kernel = wide ? k_quantize_rows<E_, true> : k_quantize_rows<E_, false>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, (const E_ *)x, R, K, ld, kb, (uint8_t *)q, scales);
        KN_CHECK_LAUNCH();
        return KN_OK;
    });
}

extern "C" int kn_quantize_f8_weights(void *stream, const void *w, int32_t dtype, int32_t w_layout, int32_t experts, int32_t n_in, int32_t n_out, void *q,
                                      float *scales)
{
    if (!w || !q || !scales || experts < 1 || n_in < 1 || n_out < 1 || !kn_dtype_ok(dtype) || (w_layout != KN_W_IN_OUT && w_layout != KN_W_OUT_IN) ||
        ((uintptr_t)q & 15))
        return KN_E_INVALID_ARG;
    if (experts > KN_MAX_EXPERTS || n_in > KN_MAX_WIDTH || n_out > KN_MAX_WIDTH) return KN_E_UNSUPPORTED;
    const int32_t nb = (int32_t)kn_div_up(n_out, F8_BLOCK), kb = (int32_t)kn_div_up(n_in, F8_BLOCK);
    const int64_t blocks = (int64_t)experts * nb * kb;
    if (blocks > 0x7fffffffLL) return KN_E_UNSUPPORTED;
    const bool io = w_layout == KN_W_IN_OUT;
    return kn_with_type(dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        hipLaunchKernelGGL((k_quantize_weights<E_>), dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, (const E_ *)w, n_out, n_in,
                           (int64_t)(io ? 1 : n_in), (int64_t)(io ? n_out : 1), nb, kb, (uint8_t *)q, scales);
        KN_CHECK_LAUNCH();
        return KN_OK;
    });
}

extern "C" int kn_grouped_linear_f8(void *stream, const kn_linear_desc *d, const void *xq, const float *xs, const void *wq, const float *ws,
                                    const void *bias, const int32_t *offsets, const int32_t *rows, int32_t relu, void *y)
{
    if (!d || d->rows < 0 || d->x_rows < 0 || d->experts < 1 || d->n_in < 1 || d->n_out < 1 || !kn_dtype_ok(d->dtype)) return KN_E_INVALID_ARG;
    if (d->rows > KN_MAX_ROWS || d->x_rows > KN_MAX_ROWS || d->experts > KN_MAX_EXPERTS || d->n_in > KN_MAX_WIDTH || d->n_out > KN_MAX_WIDTH)
        return KN_E_UNSUPPORTED;
    if (d->rows == 0) return KN_OK;
    if (!wq || !ws || !offsets || !y || (d->x_rows > 0 && (!xq || !xs)) || (!rows && d->x_rows < d->rows) || (((uintptr_t)xq | (uintptr_t)wq) & 15))
        return KN_E_INVALID_ARG;
    F8Args p = {(const uint8_t *)xq, (const uint8_t *)wq, xs, ws, bias, y, offsets, rows, (int32_t)d->rows, d->experts, d->n_out,
                (int32_t)kn_div_up(d->n_in, F8_BLOCK), (int32_t)d->x_rows, relu != 0};
    const int64_t blocks = kn_pieces(d->rows, d->experts, 128) * kn_div_up(d->n_out, 128);
    if (blocks > 0x7fffffffLL) return KN_E_UNSUPPORTED;
    return kn_with_type(d->dtype, [&](auto v) -> int {
        hipLaunchKernelGGL((k_linear_f8<decltype(v)>), dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, p);
        KN_CHECK_LAUNCH();
        return KN_OK;
    });
}
