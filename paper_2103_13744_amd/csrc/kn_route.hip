// The choice of networks per row by a learned router (kn_route: top-k of a softmax, and the rows' order by network), the weighted
// sum of the networks' results (kn_combine), and their gradients.
#include "kn_experts.h"

namespace {

constexpr int ROUTE_MAX_EXPERTS = 1024, ROUTE_MAX_K = 32;
constexpr int ROUTE_PAIRS = 2048; // pairs (row, choice) that a workgroup orders by itself
constexpr int ROUTE_THREADS = 512;

template <typename T> __device__ __forceinline__ float to_float(T v) { return (float)v; }

// Largest value among the 16 lanes of a row of the wavefront, in all of them: rotations inside the row.
__device__ __forceinline__ float row_max(float v)
{
    constexpr int ROW_ROR = 0x120; // dpp_ctrl encoding
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 8, 0xf, 0xf, false)));
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 4, 0xf, 0xf, false)));
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 2, 0xf, 0xf, false)));
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 1, 0xf, 0xf, false)));
}
__device__ __forceinline__ float row_sum(float v)
{
    constexpr int ROW_ROR = 0x120;
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 8, 0xf, 0xf, false));
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 4, 0xf, 0xf, false));
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 2, 0xf, 0xf, false));
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 1, 0xf, 0xf, false));
}
// G = 16: a row of the wavefront works on a row of logits; 64: the whole wavefront
template <int G> __device__ __forceinline__ float group_max(float v)
{
    v = row_max(v);
    if constexpr (G == 64) {
        v = fmaxf(v, __shfl_xor(v, 16));
        v = fmaxf(v, __shfl_xor(v, 32));
    }
    return v;
}
template <int G> __device__ __forceinline__ float group_sum(float v)
{
    v = row_sum(v);
    if constexpr (G == 64) {
        v += __shfl_xor(v, 16);
        v += __shfl_xor(v, 32);
    }
    return v;
}
template <int G> __device__ __forceinline__ uint64_t group_ballot(bool v, int lane)
{
    const uint64_t b = __ballot(v);
    return G == 64 ? b : (b >> (lane & 48)) & 0xffffull;
}

struct RouteArgs {
    const void *logits;
    int64_t ld;
    int32_t T, E, k, renorm;
    float *weights;
    int32_t *ids, *slots, *rows, *offsets, *hist; // hist: a histogram per workgroup, ROUTE_PAIRS / k rows of logits each
    int32_t tokens_per_block;
};

// Top-k of the rows [t0, t1) of logits: G lanes a row, each with V neighbouring logits in registers, so that the first lane of
// a ballot holds the lowest index among equal values.  k times the largest is taken out; the statistics of the softmax are
// held in 32 bits.  `count`: a histogram in the LDS.
template <typename T, int G, int V>
__device__ void choose(const RouteArgs &p, int32_t t0, int32_t t1, int32_t *count)
{
    const int lane = kn_thread() & 63, at = lane & (G - 1);
    const T *logits = (const T *)p.logits;
    const int per_round = (int)blockDim.x / G;
    for (int32_t base = t0; base < t1; base += per_round) {
        const int32_t t = base + kn_thread() / G;
        const bool there = t < t1; // (lanes without a row stay: the whole wavefront takes part in the ballots)
        float v[V];
        bool nan = false;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int32_t e = at * V + i;
            v[i] = there && e < p.E ? to_float(logits[(int64_t)t * p.ld + e]) : -INFINITY;
            nan |= v[i] != v[i];
        }
        const bool poisoned = group_ballot<G>(nan, lane) != 0;
        float top = -INFINITY, total = 0.0f, mine = 0.0f; // mine: the value of choice `at` (choices G * n + at: k <= 32, G >= 16)
        float all = 0.0f;
        int32_t chosen = -1, chosen2 = -1;
        float mine2 = 0.0f;
        for (int j = 0; j < p.k; ++j) {
            float best = v[0];
#pragma unroll
            for (int i = 1; i < V; ++i) best = fmaxf(best, v[i]); // (a NaN is never the larger)
            const float m = group_max<G>(best);
            if (j == 0) {
                top = m;
                if (!p.renorm) {
                    float s = 0.0f;
#pragma unroll
                    for (int i = 0; i < V; ++i) s += v[i] == -INFINITY ? 0.0f : expf(v[i] - top);
                    all = group_sum<G>(s);
                }
            }
            const bool some = m > -INFINITY; // (uniform in the group)
            const uint64_t holds = group_ballot<G>(some && best == m, lane);
            const int owner = (int)__ffsll((unsigned long long)holds) - 1;
            int32_t e = -1;
            if (at == owner) {
#pragma unroll
                for (int i = V - 1; i >= 0; --i)
                    if (v[i] == m) e = at * V + i;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (at * V + i == e) v[i] = -INFINITY;
            }
            e = __shfl(e, owner < 0 ? lane : (lane & ~(G - 1)) + owner);
            const float w = some ? expf(m - top) : 0.0f;
            total += w;
            if (at == (j & (G - 1))) {
                if (j < G) { mine = w; chosen = e; } else { mine2 = w; chosen2 = e; }
            }
        }
        if (!there) continue;
        const float scale = p.renorm ? total : all;
        for (int n = 0; n < 2; ++n) {
            const int j = at + n * G;
            if (j >= p.k) break;
            const int32_t e = n ? chosen2 : chosen;
            const int64_t pair = (int64_t)t * p.k + j;
            float w = e >= 0 ? (n ? mine2 : mine) / scale : 0.0f;
            if (poisoned) w = NAN;
            p.weights[pair] = w;
            p.ids[pair] = e;
            atomicAdd(&count[e >= 0 ? e : p.E], 1); // (a sum of whole numbers: any order gives the same)
        }
    }
}

template <typename T, int G, int V>
__global__ void __launch_bounds__(ROUTE_THREADS) k_route_choose(RouteArgs p)
{
    __shared__ int32_t count[ROUTE_MAX_EXPERTS + 1];
    for (int e = kn_thread(); e <= p.E; e += ROUTE_THREADS) count[e] = 0;
    __syncthreads();
    const int32_t t0 = kn_block() * p.tokens_per_block;
    choose<T, G, V>(p, t0, min(p.T, t0 + p.tokens_per_block), count);
    __syncthreads();
    for (int e = kn_thread(); e <= p.E; e += ROUTE_THREADS) p.hist[(int64_t)kn_block() * (p.E + 1) + e] = count[e];
}

// Places of the pairs of one workgroup: start[e] in the LDS is the place of its first pair of expert e.  Stable: wavefront w
// takes the w-th part of the pairs, 64 neighbours a step; a pair's rank among its step's comes from ballots over the
// bits of the expert's number.  `seen`: (wavefronts, E + 1) counts.
__device__ void place(const RouteArgs &p, int32_t p0, int32_t p1, int32_t *start, int32_t *seen)
{
    constexpr int WAVES = ROUTE_THREADS / 64, STEPS = ROUTE_PAIRS / ROUTE_THREADS;
    const int lane = kn_thread() & 63, wave = kn_thread() >> 6, bins = p.E + 1;
    for (int i = kn_thread(); i < WAVES * bins; i += ROUTE_THREADS) seen[i] = 0;
    __syncthreads();
    int32_t rank[STEPS], key[STEPS];
    int32_t *own = seen + wave * bins;
    const int bits = 32 - __clz(p.E);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int32_t q = p0 + (wave * STEPS + s) * 64 + lane;
        const bool there = q < p1;
        int32_t e = there ? p.ids[q] : -1;
        e = there && e < 0 ? p.E : e;
        key[s] = e;
        uint64_t same = __ballot(there);
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot((e >> b) & 1);
            same &= (e >> b) & 1 ? set : ~set;
        }
        rank[s] = 0;
        if (there) {
            const uint64_t below = same & ((1ull << lane) - 1);
            rank[s] = own[e] + __popcll(below); // (the wavefront's lanes read before the last of them writes: one wavefront, in order)
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if ((same >> lane) == 1ull) own[e] = rank[s] + 1;
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    for (int e = kn_thread(); e < bins; e += ROUTE_THREADS) {
        int32_t sum = start[e];
        for (int w = 0; w < WAVES; ++w) {
            const int32_t n = seen[w * bins + e];
            seen[w * bins + e] = sum;
            sum += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        if (key[s] < 0) continue;
        const int32_t q = p0 + (wave * STEPS + s) * 64 + lane;
        const int32_t at = own[key[s]] + rank[s];
        p.slots[q] = at;
        p.rows[at] = q / p.k;
    }
}

// Every workgroup sums the histograms of those before it, and all of them, by itself: they lie in the L2, and a launch
// between the two kernels costs more than reading them does.
__global__ void __launch_bounds__(ROUTE_THREADS) k_route_place(RouteArgs p, int32_t blocks)
{
    extern __shared__ int32_t lds[];
    const int bins = p.E + 1;
    int32_t *start = lds, *total = start + bins, *seen = total + bins, *scan = seen + (ROUTE_THREADS / 64) * bins;
    for (int e = kn_thread(); e < bins; e += ROUTE_THREADS) {
        int32_t before = 0, all = 0;
        for (int b = 0; b < blocks; ++b) {
            const int32_t n = p.hist[(int64_t)b * bins + e];
            before += b < kn_block() ? n : 0;
            all += n;
        }
        start[e] = before;
        total[e] = all;
    }
    __syncthreads();
    int32_t carry = 0;
    for (int e0 = 0; e0 < bins; e0 += ROUTE_THREADS) {
        const int e = e0 + kn_thread();
        int32_t sum;
        const int32_t ex = kn_block_exclusive_scan(e < bins ? total[e] : 0, scan, sum);
        if (e < bins) {
            start[e] += carry + ex;
            if (kn_block() == 0) p.offsets[e] = carry + ex; // (offsets[E]: where the pairs without an expert begin)
        }
        carry += sum;
    }
    const int32_t p0 = kn_block() * p.tokens_per_block * p.k;
    place(p, p0, (int32_t)min((int64_t)p.T * p.k, (int64_t)p0 + (int64_t)p.tokens_per_block * p.k), start, seen);
}

__global__ void k_route_none(int32_t *offsets, int32_t n)
{
    const int i = kn_block() * 256 + kn_thread();
    if (i < n) offsets[i] = 0;
}

// One wavefront per row of logits.  renormalised: dl_j = w_j (g_j - sum of w g), zeros elsewhere; else with the softmax over all
// p_e: dl_e = p_e ([e chosen] g_e - sum of w g).
template <typename T>
__global__ void __launch_bounds__(256) k_route_backward(RouteArgs p, const float *__restrict__ dweights, T *__restrict__ dlogits)
{
    const int lane = kn_thread() & 63;
    const int32_t t = kn_block() * 4 + (kn_thread() >> 6);
    if (t >= p.T) return;
    const T *l = (const T *)p.logits + (int64_t)t * p.ld;
    T *d = dlogits + (int64_t)t * p.E;
    const int64_t pair = (int64_t)t * p.k + lane;
    int32_t e = -1;
    float w = 0.0f, g = 0.0f;
    if (lane < p.k) {
        e = p.ids[pair];
        if ((uint32_t)e >= (uint32_t)p.E) e = -1;
        if (e >= 0) { w = p.weights[pair]; g = dweights[pair]; }
    }
    float mean = group_sum<64>(w * g);
    float top = -INFINITY, all = 0.0f;
    if (!p.renorm) {
        for (int i = lane; i < p.E; i += 64) top = fmaxf(top, to_float(l[i]));
        top = group_max<64>(top);
        for (int i = lane; i < p.E; i += 64) {
            const float v = to_float(l[i]);
            all += v == -INFINITY ? 0.0f : expf(v - top);
        }
        all = group_sum<64>(all);
    }
    for (int i0 = 0; i0 < p.E; i0 += 64) {
        const int i = i0 + lane;
        float gi = 0.0f, wi = 0.0f;
        bool hit = false;
        for (int j = 0; j < p.k; ++j) {
            const int32_t ej = __builtin_amdgcn_readlane(e, j);
            const float gj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(g), j));
            const float wj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), j));
            if (ej == i) { gi = gj; wi = wj; hit = true; }
        }
        if (i >= p.E) continue;
        float v = 0.0f;
        if (p.renorm) {
            if (hit) v = wi * (gi - mean);
        } else if (top > -INFINITY) {
            const float z = to_float(l[i]);
            const float pi = hit ? wi : z == -INFINITY ? 0.0f : expf(z - top) / all;
            v = pi * (gi - mean);
        }
        d[i] = (T)v;
    }
}

// 16 bytes of values
template <typename T> struct Vec {
    static constexpr int N = 16 / sizeof(T);
    typedef T Type __attribute__((ext_vector_type(16 / sizeof(T))));
};

// out[t] = sum over j of weights[t, j] y[slots[t, j]]: a thread per V neighbouring values of a row.  V: 16 bytes where the rows
// are made of whole such pieces, else 1.
template <typename T, int V>
__global__ void __launch_bounds__(256) k_combine(const T *__restrict__ y, const int32_t *__restrict__ slots, const float *__restrict__ weights,
                                                 int32_t M, int32_t D, int32_t Tn, int32_t k, T *__restrict__ out)
{
    typedef T Piece __attribute__((ext_vector_type(V)));
    const int32_t pieces = D / V;
    const int64_t q = (int64_t)kn_block() * 256 + kn_thread();
    if (q >= (int64_t)Tn * pieces) return;
    const int32_t t = (int32_t)(q / pieces), c = (int32_t)(q % pieces);
    float acc[V] = {};
    for (int j = 0; j < k; ++j) {
        const int32_t s = slots[(int64_t)t * k + j];
        if ((uint32_t)s >= (uint32_t)M) continue;
        const float w = weights ? weights[(int64_t)t * k + j] : 1.0f;
        const Piece v = *(const Piece *)(y + (int64_t)s * D + (int64_t)c * V);
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = fmaf(w, (float)v[i], acc[i]);
    }
    Piece r;
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = (T)acc[i];
    *(Piece *)(out + (int64_t)t * D + (int64_t)c * V) = r;
}

// dy[slots[t, j]] = weights[t, j] dout[t], dweights[t, j] = <dout[t], y[slots[t, j]]>: a wavefront per pair, so that a row of
// dout is read k times, but for the first from the caches.
template <typename T, int V>
__global__ void __launch_bounds__(256) k_combine_backward(const T *__restrict__ dout, const T *__restrict__ y, const int32_t *__restrict__ slots,
                                                          const float *__restrict__ weights, int32_t M, int32_t D, int64_t pairs, int32_t k,
                                                          T *__restrict__ dy, float *__restrict__ dweights)
{
    typedef T Piece __attribute__((ext_vector_type(V)));
    const int lane = kn_thread() & 63;
    const int64_t q = (int64_t)kn_block() * 4 + (kn_thread() >> 6);
    if (q >= pairs) return;
    const int32_t s = slots[q];
    const bool there = (uint32_t)s < (uint32_t)M;
    const T *g = dout + (q / k) * D;
    const float w = weights ? weights[q] : 1.0f;
    float dot = 0.0f;
    if (there)
        for (int32_t c = lane * V; c < D; c += 64 * V) {
            const Piece a = *(const Piece *)(g + c);
            Piece r;
            if (dweights) {
                const Piece b = *(const Piece *)(y + (int64_t)s * D + c);
#pragma unroll
                for (int i = 0; i < V; ++i) dot = fmaf((float)a[i], (float)b[i], dot);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) r[i] = (T)(w * (float)a[i]);
            *(Piece *)(dy + (int64_t)s * D + c) = r;
        }
    if (dweights) {
        dot = group_sum<64>(dot);
        if (lane == 0) dweights[q] = dot;
    }
}

bool route_supported(int64_t T, int32_t E, int32_t k) { return E <= ROUTE_MAX_EXPERTS && k <= ROUTE_MAX_K && T * k <= KN_MAX_ROWS; }
bool route_valid(int64_t T, int32_t E, int32_t k) { return T >= 0 && E >= 1 && k >= 1 && k <= E; }
int32_t route_tokens_per_block(int32_t k) { return ROUTE_PAIRS / k; }

template <typename T> int route_choose(hipStream_t st, const RouteArgs &p, int32_t blocks)
{
#define KN_CHOOSE(G, V) hipLaunchKernelGGL((k_route_choose<T, G, V>), dim3(blocks), dim3(ROUTE_THREADS), 0, st, p)
    if (p.E <= 16) KN_CHOOSE(16, 1);
    else if (p.E <= 64) KN_CHOOSE(16, 4);
    else if (p.E <= 128) KN_CHOOSE(16, 8);
    else if (p.E <= 256) KN_CHOOSE(16, 16);
    else KN_CHOOSE(64, 16);
#undef KN_CHOOSE
    KN_CHECK_LAUNCH();
    return KN_OK;
}

} // namespace

extern "C" int kn_route_workspace_bytes(int64_t T, int32_t E, int32_t k, int64_t *out_bytes)
{
    if (!out_bytes || !route_valid(T, E, k)) return KN_E_INVALID_ARG;
    if (!route_supported(T, E, k)) return KN_E_UNSUPPORTED;
    *out_bytes = kn_align_up(kn_div_up(T > 0 ? T : 1, route_tokens_per_block(k)) * (E + 1) * 4, 256);
    return KN_OK;
}

extern "C" int kn_route(void *stream, const void *logits, int32_t dtype, int64_t T, int32_t E, int64_t ld, int32_t k, int32_t renormalize,
                        float *weights, int32_t *ids, int32_t *slots, int32_t *rows, int32_t *offsets, void *workspace, int64_t workspace_bytes)
{
    if (!route_valid(T, E, k) || !kn_dtype_ok(dtype) || ld < E || !offsets || (T > 0 && (!logits || !weights || !ids || !slots || !rows)))
        return KN_E_INVALID_ARG;
    if (!route_supported(T, E, k)) return KN_E_UNSUPPORTED;
    hipStream_t st = (hipStream_t)stream;
    if (T == 0) {
        hipLaunchKernelGGL(k_route_none, dim3((unsigned)kn_div_up(E + 1, 256)), dim3(256), 0, st, offsets, E + 1);
        KN_CHECK_LAUNCH();
        return KN_OK;
    }
    int64_t need = 0;
    KN_TRY(kn_route_workspace_bytes(T, E, k, &need));
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need) return KN_E_WORKSPACE;
    RouteArgs p = {logits, ld, (int32_t)T, E, k, renormalize != 0, weights, ids, slots, rows, offsets, (int32_t *)workspace, route_tokens_per_block(k)};
    const int32_t blocks = (int32_t)kn_div_up(T, p.tokens_per_block);
    KN_TRY(kn_with_type(dtype, [&](auto v) -> int { return route_choose<decltype(v)>(st, p, blocks); }));
    const size_t lds = (size_t)((2 + ROUTE_THREADS / 64) * (E + 1) + 16) * 4;
    hipLaunchKernelGGL(k_route_place, dim3(blocks), dim3(ROUTE_THREADS), lds, st, p, blocks);
    KN_CHECK_LAUNCH();
    return KN_OK;
}

extern "C" int kn_route_backward(void *stream, const void *logits, int32_t dtype, int64_t T, int32_t E, int64_t ld, int32_t k, int32_t renormalize,
                                 const float *weights, const int32_t *ids, const float *dweights, void *dlogits)
{
    if (!route_valid(T, E, k) || !kn_dtype_ok(dtype) || ld < E || (T > 0 && (!logits || !weights || !ids || !dweights || !dlogits))) return KN_E_INVALID_ARG;
    if (!route_supported(T, E, k)) return KN_E_UNSUPPORTED;
    if (T == 0) return KN_OK;
    RouteArgs p = {logits, ld, (int32_t)T, E, k, renormalize != 0, const_cast<float *>(weights), const_cast<int32_t *>(ids), nullptr, nullptr, nullptr, nullptr, 0};
    return kn_with_type(dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        hipLaunchKernelGGL((k_route_backward<E_>), dim3((unsigned)kn_div_up(T, 4)), dim3(256), 0, (hipStream_t)stream, p, dweights, (E_ *)dlogits);
        KN_CHECK_LAUNCH();
        return KN_OK;
    });
}

static int combine_check(int32_t dtype, int64_t M, int64_t D, int64_t T, int32_t k)
{
    if (M < 0 || D < 1 || T < 0 || k < 1 || !kn_dtype_ok(dtype)) return KN_E_INVALID_ARG;
    if (M > KN_MAX_ROWS || D > KN_MAX_WIDTH || T * k > KN_MAX_ROWS) return KN_E_UNSUPPORTED;
    return KN_OK;
}
static bool whole_pieces(int64_t D, int32_t dtype, const void *a, const void *b, const void *c)
{
    return D * kn_item(dtype) % 16 == 0 && (((uintptr_t)a | (uintptr_t)b | (uintptr_t)c) & 15) == 0;
}

extern "C" int kn_combine(void *stream, const void *y, int32_t dtype, int64_t M, int32_t D, const int32_t *slots, const float *weights, int64_t T,
                          int32_t k, void *out)
{
    KN_TRY(combine_check(dtype, M, D, T, k));
    if (T == 0) return KN_OK;
    if ((M > 0 && !y) || !slots || !out) return KN_E_INVALID_ARG;
    return kn_with_type(dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        constexpr int V = 16 / sizeof(E_);
        const bool wide = whole_pieces(D, dtype, y, out, nullptr);
        const int64_t blocks = kn_div_up(T * (wide ? D / V : D), 256);
        if (blocks > 0x7fffffffLL) return KN_E_UNSUPPORTED;
        auto kernel = wide ? k_combine<E_, V> : k_combine<E_, 1>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, (const E_ *)y, slots, weights, (int32_t)M, D, (int32_t)T,
                           k, (E_ *)out);
        KN_CHECK_LAUNCH();
        return KN_OK;
    });
}

extern "C" int kn_combine_backward(void *stream, const void *dout, const void *y, int32_t dtype, int64_t M, int32_t D, const int32_t *slots,
                                   const float *weights, int64_t T, int32_t k, void *dy, float *dweights)
{
    KN_TRY(combine_check(dtype, M, D, T, k));
    if (T == 0) return KN_OK;
    if (!dout || !slots || (M > 0 && (!dy || (dweights && !y)))) return KN_E_INVALID_ARG;
    return kn_with_type(dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        constexpr int V = 16 / sizeof(E_);
        auto kernel = whole_pieces(D, dtype, dout, dweights ? y : nullptr, dy) ? k_combine_backward<E_, V> : k_combine_backward<E_, 1>;
        hipLaunchKernelGGL(kernel, dim3((unsigned)kn_div_up(T * k, 4)), dim3(256), 0, (hipStream_t)stream, (const E_ *)dout, (const E_ *)y, slots,
                           weights, (int32_t)M, D, T * k, k, (E_ *)dy, dweights);
        KN_CHECK_LAUNCH();
        return KN_OK;
    });
}
