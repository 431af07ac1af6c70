// Products grouped by network in 8-bit floating point (e4m3) with fp32 scales: kn_quantize_f8 (a scale per row and 128 inputs),
// kn_quantize_f8_weights (a scale per 128 x 128), kn_grouped_linear_f8; and rows kept in 8 bits for a backward pass: kn_save_f8, kn_restore_f8.
#include "kn_tile.h"

namespace {

constexpr int F8_BLOCK = 128;
constexpr float F8_INVERSE = 1.0f / 448.0f, F8_TINY = 0x1p-100f; // 448: the type's largest value

// Scale of a block whose largest magnitude is `amax`: amax times the fp32 next to 1 / 448, rounded once.  A value's 8 bits are the
// nearest e4m3 (ties to even) of the fp32 quotient x / s; the quotient of amax may pass 448 by its last bit and rounds to 448.  Both
// roundings matter to the bit: inputs of 16 bits lie on ties of the 8-bit type now and then, which an s one bit off breaks the
// other way.  A block of zeros keeps a finite scale.
__device__ __forceinline__ float f8_scale(float amax) { return fmaxf(amax, F8_TINY) * F8_INVERSE; }
__device__ __forceinline__ uint32_t f8_pack(float a, float b, float c, float d, float s)
{
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(a / s, b / s, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c / s, d / s, v, true);
}
// 16 lanes per row and block of 128 inputs, 8 values a lane.  Inputs beyond K are zeros.  Bound by its bytes: 16,411 x 2048 in bf16, 25 us,
// 4.1 TB/s.
template <typename T>
__global__ void __launch_bounds__(256) k_quantize_rows(const T *__restrict__ x, int64_t R, int32_t K, int64_t ld, int32_t kb,
                                                       uint8_t *__restrict__ q, float *__restrict__ scales, int32_t first)
{
    const int64_t g = (((int64_t)first + kn_block()) * 256 + kn_thread()) >> 4;
    if (g >= R * kb) return;
    const int at = kn_thread() & 15;
    const int64_t row = g / kb;
    const int32_t blk = (int32_t)(g % kb), k0 = blk * F8_BLOCK + at * 8;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; i += 16 / (int)sizeof(T)) {
        const typename KnFrag<T>::Type p = kn_any_piece(x + row * ld, k0 + i, K);
#pragma unroll
        for (int j = 0; j < 16 / (int)sizeof(T); ++j) v[i + j] = (float)p[j];
    }
    float amax = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = fmaxf(amax, fabsf(v[i]));
    const float s = f8_scale(kn_row_max(amax));
    uint2 out;
    out.x = f8_pack(v[0], v[1], v[2], v[3], s);
    out.y = f8_pack(v[4], v[5], v[6], v[7], s);
    *(uint2 *)(q + row * kb * F8_BLOCK + k0) = out;
    if (at == 0) scales[g] = s;
}

// The power of two of a block of saved values: the least n >= -100 with amax <= 448 2^n (448 = 1.75 2^8), so that a value's quotient is exact and its 8 bits
// are rounded once; the value that they stand for is exact in the 16-bit types.
constexpr int SAVED_LEAST = -100;
// Of the largest values of a type some would round to a power of two that it does not have (65504 to 2^16): they are kept as 240 2^n instead.
template <typename T> constexpr int saved_most() { return std::is_same<T, _Float16>::value ? 8 : 120; }
__device__ __forceinline__ int saved_exponent(float amax)
{
    const int b = __float_as_int(amax);
    return max((b >> 23) - 127 - 8 + ((b & 0x7fffff) > 0x600000 ? 1 : 0), SAVED_LEAST);
}
// LANES per row and block of 128 values (16, or as many as a shorter row fills), 8 values a lane.  A value above zero keeps its sign: what would round to zero becomes the smallest
// value, 2^-9.  What is not finite has no part in the scale: +infinity becomes the NaN without, NaN and -infinity the one with the sign bit.
// Bound by its bytes: 16,411 x 2048 in bf16: 23 us, 4.4 TB/s; 524,291 x 64 in fp16: 25, 4.1 TB/s (16 lanes a row: 41).
template <typename T, int LANES>
__global__ void __launch_bounds__(256) k_save_rows(const T *__restrict__ x, int64_t R, int32_t K, int64_t ld, int32_t kb, uint8_t *__restrict__ q,
                                                   uint8_t *__restrict__ exponents, int32_t first)
{
    const int64_t g = (((int64_t)first + kn_block()) * 256 + kn_thread()) / LANES;
    if (g >= R * kb) return;
    const int at = kn_thread() & (LANES - 1);
    const int64_t row = g / kb;
    const int32_t blk = (int32_t)(g % kb), k0 = blk * KN_SAVED_BLOCK + at * 8, bytes = (K + 15) & ~15;
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; i += 16 / (int)sizeof(T)) {
        const typename KnFrag<T>::Type p = kn_any_piece(x + row * ld, k0 + i, K);
#pragma unroll
        for (int j = 0; j < 16 / (int)sizeof(T); ++j) v[i + j] = (float)p[j];
    }
    float amax = 0.0f;
    bool finite = true;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float m = fabsf(v[i]);
        const bool good = m < INFINITY;
        finite &= good;
        amax = good ? fmaxf(amax, m) : amax;
    }
    if constexpr (LANES == 16) amax = kn_row_max(amax);
    else
#pragma unroll
        for (int d = LANES / 2; d > 0; d >>= 1) amax = fmaxf(amax, __shfl_xor(amax, d));
    const int n = saved_exponent(amax);
    const float inverse = __int_as_float((127 - n) << 23);
    const float cap = n == saved_most<T>() ? 240.0f : 448.0f;
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        t[i] = fminf(fmaxf(v[i] * inverse, -cap), cap); // (what is not finite is looked at below)
        t[i] = v[i] > 0.0f ? fmaxf(t[i], 0x1p-9f) : t[i];
    }
    uint32_t out[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(t[4 * h], t[4 * h + 1], 0, false);
        out[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(t[4 * h + 2], t[4 * h + 3], w, true);
    }
    if (!finite) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (!(fabsf(v[i]) < INFINITY)) {
                const int shift = 8 * (i & 3);
                out[i / 4] = (out[i / 4] & ~(0xffu << shift)) | (v[i] > 0.0f ? 0x7fu : 0xffu) << shift;
            }
    }
    if (k0 < bytes) *(uint2 *)(q + row * bytes + k0) = make_uint2(out[0], out[1]);
    if (at == 0) exponents[g] = (uint8_t)(n + 127);
}

// The values that saved rows stand for: a thread per 8 of them.  16,411 x 2048 in bf16: 16.5 us, 6.1 TB/s (some of it from the caches).
template <typename T>
__global__ void __launch_bounds__(256) k_restore_rows(const uint8_t *__restrict__ q, const uint8_t *__restrict__ exponents, int64_t R, int32_t K, int32_t kb,
                                                      T *__restrict__ x, int32_t first)
{
    const int32_t eights = (K + 7) / 8, bytes = (K + 15) & ~15;
    const int64_t at = ((int64_t)first + kn_block()) * 256 + kn_thread();
    if (at >= R * eights) return;
    const int64_t row = at / eights;
    const int32_t k = (int32_t)(at % eights) * 8;
    const uint2 v = *(const uint2 *)(q + row * bytes + k);
    const float power = kn_power(exponents[row * kb + k / KN_SAVED_BLOCK]);
    T wide[8];
    kn_widen_saved<T>(v.x, power, wide);
    kn_widen_saved<T>(v.y, power, wide + 4);
    typename KnEight<T>::Piece o;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] = wide[i];
    KnEight<T>::store(x + row * K, k, K, o);
}

// One workgroup per 128 x 128 block of a network's weights, through the LDS (the two layouts differ in which index is next to
// which).  Outputs beyond N are not stored, inputs beyond K are zeros.  Done once per weights, and not tuned.
template <typename T>
__global__ void __launch_bounds__(256) k_quantize_weights(const T *__restrict__ w, int32_t N, int32_t K, int64_t s_n, int64_t s_k, int32_t nb,
                                                          int32_t kb, uint8_t *__restrict__ q, float *__restrict__ scales, int32_t first)
{
    constexpr int LD = F8_BLOCK + 1;
    __shared__ float t[F8_BLOCK / 2 * LD]; // half a block at a time
    __shared__ float part[4];
    const int64_t blk = first + kn_block();
    const int32_t bk = (int32_t)(blk % kb), bn = (int32_t)(blk / kb % nb);
    const int64_t e = blk / kb / nb;
    const T *src = w + e * N * K;
    float amax = 0.0f;
    for (int i = kn_thread(); i < F8_BLOCK * F8_BLOCK; i += 256) {
        const int32_t n = bn * F8_BLOCK + (s_n == 1 ? i % F8_BLOCK : i / F8_BLOCK), k = bk * F8_BLOCK + (s_n == 1 ? i / F8_BLOCK : i % F8_BLOCK);
        if (n < N && k < K) amax = fmaxf(amax, fabsf((float)src[n * s_n + k * s_k]));
    }
    amax = kn_row_max(amax);
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
    int32_t first; // number of the launch's first workgroup
};

// 32 values of 8 bits as 4 fragments of 8 in fp16, which holds every e4m3 value (448 down to 2^-9, NaN) exactly
struct F8Wide {
    kn_f16x8 part[4];
};
__device__ __forceinline__ F8Wide f8_widen(kn_u32x4 lo, kn_u32x4 hi)
{
    typedef _Float16 Pair __attribute__((ext_vector_type(2)));
    F8Wide w;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const uint32_t v = q < 4 ? lo[q] : hi[q - 4];
        const Pair a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, 1.0f, true);
        w.part[q / 2][q % 2 * 4] = a[0];
        w.part[q / 2][q % 2 * 4 + 1] = a[1];
        w.part[q / 2][q % 2 * 4 + 2] = b[0];
        w.part[q / 2][q % 2 * 4 + 3] = b[1];
    }
    return w;
}

// Tiles of BM x BN results, WR x WC wavefronts, NB stages in the LDS, fetched ahead.  A stage is a block of 128 inputs, whose sum
// starts from zero and is scaled, in fp32, as it is added.  The 8-bit matrix instructions do not hold it in 32 bits: each 8 neighbouring
// products are brought to the largest one's exponent and cut off 13 bits below it, so that of 8 products, one of them 2^14 times the others,
// one is left.  Values are widened to fp16 on their way from the LDS instead (their products are exact in fp32), and the
// 16-bit instruction's sums are fp32's.  Fragments of the
// weights are the first operand: a lane's four results are neighbours in a row, and one factor, the product of the row's
// scale and the weights', serves all of them.  The four lanes of a row hold the factors of four blocks and hand them to each other:
// in the LDS they took the place of a workgroup.
// Measured: 32,822 rows through an index, 16 networks 2048 x 2048: 290 us, 950 TFLOP/s (the 8-bit instructions: 205).  32 rows in about 20
// of 32 networks 2560 x 2048: 27 us, 4.0 TB/s.
template <typename T, int BM, int BN, int WR, int WC, int NB>
__global__ void __launch_bounds__(WR * WC * 64) k_linear_f8(F8Args p, int32_t blocks)
{
    constexpr int NW = WR * WC, STAGE = (BM + BN) * 128, U = BM / WR / 16, V = BN / WC / 16;
    static_assert(F8_BLOCK % BN == 0, "a tile's columns share a scale");
    typedef KnRowLoader<uint8_t, BM, NW, true> LoadA;
    typedef KnRowLoader<uint8_t, BN, NW, true> LoadB;
    constexpr int WN = BN / WC, LD = WN + 4, LR = WN / 8;
    constexpr int BYTES = NB * STAGE > NW * 16 * LD * 4 ? NB * STAGE : NW * 16 * LD * 4;
    __shared__ __align__(16) char lds_[BYTES];
    KN_LDS char *lds = (KN_LDS char *)lds_;
    const int tid = kn_thread(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ntiles = (p.N + BN - 1) / BN;
    // (where a network has a piece or none, its columns go to all XCDs: only some networks have rows, XCDs should be alike)
    const int32_t number = p.M < (int64_t)BM * p.E ? p.first + kn_block() : kn_xcd_order(p.first + kn_block(), blocks);
    const KnPiece piece = kn_find_piece(p.offsets, p.E, p.M, BM, number / ntiles);
    const int j0 = number % ntiles * BN;
    if (piece.begin >= piece.end) return;
    const int64_t kp = (int64_t)p.kb * F8_BLOCK;
    const bool some = piece.group < p.E;
    const int64_t group = some ? piece.group : 0;
    LoadA la;
    LoadB lb;
    la.start(wave, lane, [&](int r) {
        const int32_t i = min(piece.begin + r, piece.end - 1), src = p.rows ? p.rows[i] : i;
        return p.x + ((uint32_t)src < (uint32_t)p.x_rows ? src : 0) * kp;
    });
    lb.start(wave, lane, [&](int r) { return p.w + (group * p.N + min(j0 + r, p.N - 1)) * kp; });
    const int32_t steps = some && p.x_rows > 0 ? p.kb : 0; // (an x without rows is not looked at)
    constexpr int LOADS = LoadA::N + LoadB::N;
    auto fetch = [&](int s, int at) {
        la.fetch(lds + at * STAGE, wave, lane, F8_BLOCK);
        lb.fetch(lds + at * STAGE + BM * 128, wave, lane, F8_BLOCK);
    };
    const float *ws = p.ws + (group * ((p.N + F8_BLOCK - 1) / F8_BLOCK) + j0 / F8_BLOCK) * p.kb;
    const int wi = (wave / WC) * (BM / WR), wj = (wave % WC) * WN;
    const float *xs[U]; // this lane's row's scales, from its own of four on
    bool there[U];      // (a row that x does not have goes through with row 0's values, and is zeros in the end: a product with zero would keep a NaN)
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t i = min(piece.begin + wi + 16 * u + (lane & 15), piece.end - 1), src = p.rows ? p.rows[i] : i;
        there[u] = (uint32_t)src < (uint32_t)p.x_rows;
        xs[u] = p.xs + (int64_t)(there[u] ? src : 0) * p.kb;
    }
    float asked[U], asked_w, factor[U];
    auto ask = [&](int s) { // (behind the last block: the last one's, unused)
        const int b = min(s + (lane >> 4), steps - 1);
#pragma unroll
        for (int u = 0; u < U; ++u) asked[u] = xs[u][b];
        asked_w = ws[b];
    };
    kn_f32x4 acc[U][V] = {};
    if (steps > 0) {
        ask(0);
        for (int s = 0; s < NB - 1 && s < steps; ++s) fetch(s, s);
        for (int s = 0, at = 0; s < steps; ++s) {
            if (s + NB - 1 <= steps) kn_stage_barrier<(NB - 2) * LOADS>();
            else kn_stage_barrier();
            if (s + NB - 1 < steps) fetch(s + NB - 1, at == 0 ? NB - 1 : at - 1);
            if (s % 4 == 0) {
#pragma unroll
                for (int u = 0; u < U; ++u) factor[u] = asked[u] * asked_w;
                if (s + 4 < steps) ask(s + 4);
            }
            const KN_LDS char *ta = lds + at * STAGE, *tb = ta + BM * 128;
            auto frag = [&](const KN_LDS char *tile, int r0) { // (which 8 inputs of the 128 a lane has in which part is the same in a and b)
                const int r = r0 + (lane & 15);
                return f8_widen(*(const KN_LDS kn_u32x4 *)(tile + kn_row_byte(r, lane >> 4)), *(const KN_LDS kn_u32x4 *)(tile + kn_row_byte(r, 4 + (lane >> 4))));
            };
            F8Wide fb[V];
#pragma unroll
            for (int v = 0; v < V; ++v) fb[v] = frag(tb, wj + 16 * v);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const F8Wide fa = frag(ta, wi + 16 * u);
                const float f = __shfl(factor[u], (lane & 15) + 16 * (s & 3));
                kn_f32x4 r[V] = {};
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int v = 0; v < V; ++v) r[v] = kn_mfma(fb[v].part[q], fa.part[q], r[v]);
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[u][v][i] = fmaf(r[v][i], f, acc[u][v][i]);
            }
            at = at + 1 == NB ? 0 : at + 1;
        }
    }
    kn_stage_barrier(); // (the tiles' LDS is used again)
    KN_LDS float *mine = (KN_LDS float *)(lds + wave * (16 * LD * 4));
    T *y = (T *)p.y;
    const T *bias = (const T *)p.bias;
    const int cj = lane % LR * 8;
    const int32_t j = j0 + wj + cj;
    float add[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) add[q] = bias && some && j < p.N ? (float)bias[group * p.N + min(j + q, p.N - 1)] : 0.0f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int v = 0; v < V; ++v) *(KN_LDS kn_f32x4 *)(mine + (lane & 15) * LD + 16 * v + (lane >> 4) * 4) = there[u] ? acc[u][v] : kn_f32x4{0, 0, 0, 0};
        kn_lanes_meet();
#pragma unroll
        for (int h = 0; h < (16 * LR + 63) / 64; ++h) {
            const int r = h * (64 / LR) + lane / LR;
            const int32_t i = piece.begin + wi + 16 * u + r;
            if (r >= 16 || i >= piece.end || j >= p.N) continue;
            const kn_f32x4 lo = *(const KN_LDS kn_f32x4 *)(mine + r * LD + cj), hi = *(const KN_LDS kn_f32x4 *)(mine + r * LD + cj + 4);
            const float s[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            typename KnEight<T>::Piece o;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                float t = s[q] + add[q];
                if (p.relu) t = t > 0.0f || t != t ? t : 0.0f; // (a NaN stays one)
                o[q] = (T)t;
            }
            KnEight<T>::store(y + (int64_t)i * p.N, j, p.N, o);
        }
        kn_lanes_meet();
    }
}

template <typename T, int BM, int BN, int WR, int WC, int NB> int launch_f8(hipStream_t st, const F8Args &p)
{
    const int64_t blocks = kn_pieces(p.M, p.E, BM) * kn_div_up(p.N, BN);
    return kn_launch(blocks, WR * WC * 64, [&](dim3 grid, int32_t first) {
        F8Args q = p;
        q.first = first;
        hipLaunchKernelGGL((k_linear_f8<T, BM, BN, WR, WC, NB>), grid, dim3(WR * WC * 64), 0, st, q, (int32_t)blocks);
    });
}

} // namespace

extern "C" int kn_quantize_f8(void *stream, const void *x, int32_t dtype, int64_t R, int32_t K, int64_t ld, void *q, float *scales)
{
    if (R < 0 || K < 1 || ld < K || !kn_dtype_ok(dtype) || (R > 0 && (!x || !q || !scales)) || ((uintptr_t)q & 15)) return KN_E_INVALID_ARG;
    if (R > KN_MAX_ROWS || K > KN_MAX_WIDTH) return KN_E_UNSUPPORTED;
    if (R == 0) return KN_OK;
    const int32_t kb = (int32_t)kn_div_up(K, F8_BLOCK);
    const int64_t blocks = kn_div_up(R * kb, 16);
    return kn_with_type(dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        return kn_launch(blocks, 256, [&](dim3 grid, int32_t first) {
            hipLaunchKernelGGL((k_quantize_rows<E_>), grid, dim3(256), 0, (hipStream_t)stream, (const E_ *)x, R, K, ld, kb, (uint8_t *)q, scales, first);
        });
    });
}

extern "C" int kn_save_f8(void *stream, const void *x, int32_t dtype, int64_t R, int32_t K, int64_t ld, void *q, uint8_t *exponents)
{
    if (R < 0 || K < 1 || ld < K || !kn_dtype_ok(dtype) || (R > 0 && (!x || !q || !exponents)) || ((uintptr_t)q & 15)) return KN_E_INVALID_ARG;
    if (R > KN_MAX_ROWS || K > KN_MAX_WIDTH) return KN_E_UNSUPPORTED;
    if (R == 0) return KN_OK;
    const int32_t kb = (int32_t)kn_div_up(K, KN_SAVED_BLOCK);
    return kn_with_type(dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        const int lanes = K <= 32 ? 4 : K <= 64 ? 8 : 16;
        auto kernel = K <= 32 ? k_save_rows<E_, 4> : K <= 64 ? k_save_rows<E_, 8> : k_save_rows<E_, 16>;
        return kn_launch(kn_div_up(R * kb * lanes, 256), 256, [&](dim3 grid, int32_t first) {
            hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)stream, (const E_ *)x, R, K, ld, kb, (uint8_t *)q, exponents, first);
        });
    });
}

extern "C" int kn_restore_f8(void *stream, const void *q, const uint8_t *exponents, int64_t R, int32_t K, int32_t dtype, void *x)
{
    if (R < 0 || K < 1 || !kn_dtype_ok(dtype) || (R > 0 && (!x || !q || !exponents)) || ((uintptr_t)q & 15)) return KN_E_INVALID_ARG;
    if (R > KN_MAX_ROWS || K > KN_MAX_WIDTH) return KN_E_UNSUPPORTED;
    if (R == 0) return KN_OK;
    const int32_t kb = (int32_t)kn_div_up(K, KN_SAVED_BLOCK);
    return kn_with_type(dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        return kn_launch(kn_div_up(R * kn_div_up(K, 8), 256), 256, [&](dim3 grid, int32_t first) {
            hipLaunchKernelGGL((k_restore_rows<E_>), grid, dim3(256), 0, (hipStream_t)stream, (const uint8_t *)q, exponents, R, K, kb, (E_ *)x, first);
        });
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
    const bool io = w_layout == KN_W_IN_OUT;
    return kn_with_type(dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        return kn_launch(blocks, 256, [&](dim3 grid, int32_t first) {
            hipLaunchKernelGGL((k_quantize_weights<E_>), grid, dim3(256), 0, (hipStream_t)stream, (const E_ *)w, n_out, n_in,
                               (int64_t)(io ? 1 : n_in), (int64_t)(io ? n_out : 1), nb, kb, (uint8_t *)q, scales, first);
        });
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
    // Which tile (us; 32, 64 and 192 rows x 128): 7,791 rows, 7 networks 2048 x 64: 16, 22, 37; 2,048 rows, 32 networks 2560 x 2048: 61, 65, 89;
    // 12,000 rows, 64 networks 512 x 512: 19, 19, 21; 8,728 rows, 5 networks 576 x 2048: 43, 39, 41; 8,192 rows, 16 networks 2048 x 2048:
    // 110, 101, 98; 32,768 of them: 399, 343, 294.
    const int64_t each = p.M / p.E; // rows of a network, on average
    auto tiles = [&](int64_t bm) { return kn_div_up(p.M, bm) * kn_div_up(p.N, 128); };
    return kn_with_type(d->dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        hipStream_t st = (hipStream_t)stream;
        if (each >= 512 && tiles(192) >= 256) return launch_f8<E_, 192, 128, 2, 2, 2>(st, p);
        if (each >= 128 && tiles(64) >= 128) return launch_f8<E_, 64, 128, 1, 4, 2>(st, p);
        return launch_f8<E_, 32, 128, 1, 4, 2>(st, p);
    });
}
