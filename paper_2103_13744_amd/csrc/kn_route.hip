// The choice of networks per row by a learned router (kn_route: top-k of a softmax, and the rows' order by network), the weighted
// sum of the networks' results (kn_combine), and their gradients.
#include "kn_experts.h"

namespace {

constexpr int ROUTE_MAX_EXPERTS = 1024, ROUTE_MAX_K = 32;
constexpr int ROUTE_THREADS = 512;
constexpr int ROUTE_TOKENS = 64;                          // rows of logits of a workgroup
constexpr int ROUTE_PAIRS = ROUTE_TOKENS * ROUTE_MAX_K;   // pairs (row, choice) that it orders at most

template <typename T> __device__ __forceinline__ float to_float(T v) { return (float)v; }

// Sum over the 16 lanes of a row of the wavefront, in all of them: rotations inside the row
__device__ __forceinline__ float row_sum(float v)
{
    constexpr int ROW_ROR = 0x120; // dpp_ctrl encoding
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 8, 0xf, 0xf, true));
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 4, 0xf, 0xf, true));
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 2, 0xf, 0xf, true));
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 1, 0xf, 0xf, true));
}
// G = 16: a row of the wavefront works on a row of logits; 64: the whole wavefront
template <int G> __device__ __forceinline__ float group_max(float v)
{
    v = kn_row_max(v);
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

// The same for whole numbers of 16 lanes
__device__ __forceinline__ int32_t row_max_i32(int32_t v)
{
    constexpr int ROW_ROR = 0x120;
    v = max(v, __builtin_amdgcn_update_dpp(0, v, ROW_ROR + 8, 0xf, 0xf, true));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, ROW_ROR + 4, 0xf, 0xf, true));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, ROW_ROR + 2, 0xf, 0xf, true));
    return max(v, __builtin_amdgcn_update_dpp(0, v, ROW_ROR + 1, 0xf, 0xf, true));
}
template <int G> __device__ __forceinline__ int32_t group_max_i32(int32_t v)
{
    v = row_max_i32(v);
    if constexpr (G == 64) {
        v = max(v, __shfl_xor(v, 16));
        v = max(v, __shfl_xor(v, 32));
    }
    return v;
}

struct RouteArgs {
    const void *logits;
    int64_t ld;
    int32_t T, E, k, renorm;
    float *weights;
    int32_t *ids, *slots, *rows, *offsets;
    int32_t *hist;   // (E + 1, workgroups): pairs of each expert in each workgroup, then those before it
    int32_t *totals; // E + 1
    int32_t wide;    // a lane's logits are one aligned piece
    int32_t blocks, first; // workgroups in all, number of the launch's first one
};

// The V logits of row t that lane `at` holds: neighbours, -infinity behind the end
template <typename T, int V> __device__ __forceinline__ void load_logits(const RouteArgs &p, int32_t t, bool there, int at, float v[V])
{
    typedef T Piece __attribute__((ext_vector_type(V)));
    const T *l = (const T *)p.logits + (int64_t)t * p.ld + at * V;
    if (p.wide) {
        const bool in = there && at * V < p.E;
        Piece x = {};
        if (in) x = *(const Piece *)l;
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = in ? to_float((T)x[i]) : -INFINITY;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = there && at * V + i < p.E ? to_float(l[i]) : -INFINITY;
    }
}

// Logits as whole numbers of the same order (both zeros alike, a NaN below everything): comparing and taking the largest is one
// instruction each, also across lanes.
constexpr int32_t KEY_NONE = INT32_MIN, KEY_LOWEST = (int32_t)0x807fffff; // nothing; -infinity
__device__ __forceinline__ int32_t key_of(float v)
{
    const int32_t b = __float_as_int(v + 0.0f);
    return v != v ? KEY_NONE : b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float value_of(int32_t key) { return __int_as_float(key ^ ((key >> 31) & 0x7fffffff)); }

// Top-k of the rows [t0, t1) of logits: G lanes a row, each with V neighbouring logits in registers, so that the first lane of
// those that hold the largest holds the lowest index.  k times the largest is taken out; the statistics of the softmax are held in
// 32 bits.  In the LDS: `count`, a histogram; `chosen`, the experts of the rows that are being worked on.
// Measured: 32,768 rows of 128 logits in fp32, k = 8: 12.5 us, bound by vector instructions (some 80 per choice of 4 rows); their
// order takes 4 + 6 us more, in launches of latency.  16 rows of 64, k = 4, order included: 3.8 us, one launch.
template <typename T, int G, int V>
__device__ void choose(const RouteArgs &p, int32_t t0, int32_t t1, int32_t *count, int32_t *chosen)
{
    const int lane = kn_thread() & 63, at = lane & (G - 1);
    constexpr int PER_ROUND = ROUTE_THREADS / G;
    const uint64_t before = ((1ull << lane) - 1) & ~((1ull << (lane & ~(G - 1))) - 1); // the row's lanes before this one
    int32_t *mine = chosen + kn_thread() / G * ROUTE_MAX_K; // (of one wavefront alone)
    for (int32_t base = t0; base < t1; base += PER_ROUND) {
        const int32_t t = base + kn_thread() / G;
        const bool there = t < t1; // (lanes without a row stay: the whole wavefront takes part in the ballots)
        float v[V];
        int32_t key[V];
        load_logits<T, V>(p, t, there, at, v);
        bool nan = false;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            nan |= v[i] != v[i];
            key[i] = key_of(v[i]);
        }
        const bool poisoned = group_ballot<G>(nan, lane) != 0;
        float all = 0.0f;
        int32_t first = KEY_NONE, value[2] = {KEY_NONE, KEY_NONE}; // value: the keys of choices at and at + G
        for (int j = 0; j < p.k; ++j) {
            int32_t best = key[0];
#pragma unroll
            for (int i = 1; i < V; ++i) best = max(best, key[i]);
            const int32_t m = group_max_i32<G>(best);
            if (j == 0) {
                first = m;
                if (!p.renorm) {
                    const float top = value_of(m);
                    float s = 0.0f;
#pragma unroll
                    for (int i = 0; i < V; ++i) s += key[i] <= KEY_LOWEST ? 0.0f : expf(v[i] - top);
                    all = group_sum<G>(s);
                }
            }
            const uint64_t holds = __ballot(best == m);
            if (best == m && m > KEY_LOWEST && (holds & before) == 0) {
                int i0 = 0;
#pragma unroll
                for (int i = V - 1; i >= 0; --i) i0 = key[i] == m ? i : i0;
#pragma unroll
                for (int i = 0; i < V; ++i) key[i] = i == i0 ? KEY_NONE : key[i];
                mine[j] = at * V + i0;
            }
            if (at == (j & (G - 1))) value[j / G] = m;
        }
        const float top = value_of(first);
        const float z[2] = {value[0] > KEY_LOWEST ? expf(value_of(value[0]) - top) : 0.0f, value[1] > KEY_LOWEST ? expf(value_of(value[1]) - top) : 0.0f};
        const float scale = p.renorm ? group_sum<G>(z[0] + z[1]) : all;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (there)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                const int j = at + n * G;
                if (j >= p.k) break;
                const int32_t e = value[n] > KEY_LOWEST ? mine[j] : -1;
                const int64_t pair = (int64_t)t * p.k + j;
                p.weights[pair] = poisoned ? NAN : e >= 0 ? z[n] / scale : 0.0f;
                p.ids[pair] = e;
                atomicAdd(&count[e >= 0 ? e : p.E], 1); // (a sum of whole numbers: any order gives the same)
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// Places of the pairs [p0, p1) of one workgroup: start[e] in the LDS is the place of its first pair of expert e.  Stable: wavefront w
// takes the w-th part of the pairs, 64 neighbours a step; a pair's rank among its step's comes from ballots over the
// bits of the expert's number.  `seen`: (wavefronts, E + 1) counts.
__device__ void place(const RouteArgs &p, int32_t p0, int32_t p1, const int32_t *start, int32_t *seen)
{
    constexpr int WAVES = ROUTE_THREADS / 64, STEPS = ROUTE_PAIRS / ROUTE_THREADS;
    const int lane = kn_thread() & 63, wave = kn_thread() >> 6, bins = p.E + 1;
    const int steps = (p1 - p0 + ROUTE_THREADS - 1) / ROUTE_THREADS; // (of a wavefront)
    for (int i = kn_thread(); i < WAVES * bins; i += ROUTE_THREADS) seen[i] = 0;
    __syncthreads();
    int32_t rank[STEPS], key[STEPS];
    int32_t *own = seen + wave * bins;
    const int bits = 32 - __clz(p.E);
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        key[s] = -1;
        rank[s] = 0;
        if (s >= steps) continue;
        const int32_t q = p0 + (wave * steps + s) * 64 + lane;
        const bool there = q < p1;
        int32_t e = there ? p.ids[q] : -1;
        e = there && e < 0 ? p.E : e;
        key[s] = e;
        uint64_t same = __ballot(there);
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot((e >> b) & 1);
            same &= (e >> b) & 1 ? set : ~set;
        }
        if (there) {
            rank[s] = own[e] + __popcll(same & ((1ull << lane) - 1)); // (every lane has read before one of them writes: one wavefront)
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
        const int32_t q = p0 + (wave * steps + s) * 64 + lane;
        const int32_t at = own[key[s]] + rank[s];
        p.slots[q] = at;
        p.rows[at] = q / p.k;
    }
}

// start[e] += the sum of counts before e, offsets where asked for
__device__ void scan_counts(const RouteArgs &p, const int32_t *counts, int32_t *start, int32_t *scratch, bool store)
{
    int32_t carry = 0;
    for (int e0 = 0; e0 <= p.E; e0 += ROUTE_THREADS) {
        const int e = e0 + kn_thread();
        int32_t sum;
        const int32_t before = kn_block_exclusive_scan(e <= p.E ? counts[e] : 0, scratch, sum);
        if (e <= p.E) {
            start[e] += carry + before;
            if (store) p.offsets[e] = carry + before; // (offsets[E]: where the pairs without an expert begin)
        }
        carry += sum;
    }
}

// ONE: all rows are one workgroup's, which places them too; else its histogram is left for k_route_scan and k_route_place
template <typename T, int G, int V, bool ONE>
__global__ void __launch_bounds__(ROUTE_THREADS) k_route_choose(RouteArgs p)
{
    extern __shared__ int32_t lds[];
    __shared__ int32_t chosen[ROUTE_THREADS / G * ROUTE_MAX_K], scratch[16];
    const int bins = p.E + 1;
    int32_t *count = lds, *start = count + bins, *seen = start + bins; // (start, seen: ONE only)
    for (int e = kn_thread(); e < bins; e += ROUTE_THREADS) count[e] = 0;
    __syncthreads();
    const int32_t block = p.first + kn_block(), t0 = block * ROUTE_TOKENS, t1 = min(p.T, t0 + ROUTE_TOKENS);
    choose<T, G, V>(p, t0, t1, count, chosen);
    __syncthreads();
    if constexpr (ONE) {
        for (int e = kn_thread(); e < bins; e += ROUTE_THREADS) start[e] = 0;
        __threadfence_block(); // (this workgroup's ids are read again below)
        __syncthreads();
        scan_counts(p, count, start, scratch, true);
        __syncthreads();
        place(p, 0, p.T * p.k, start, seen);
    } else {
        for (int e = kn_thread(); e < bins; e += ROUTE_THREADS) p.hist[(int64_t)e * p.blocks + block] = count[e];
    }
}

// One workgroup per expert: its pairs before each workgroup, and in all
__global__ void __launch_bounds__(256) k_route_scan(RouteArgs p)
{
    __shared__ int32_t scratch[16];
    const int32_t blocks = p.blocks;
    int32_t *h = p.hist + (int64_t)kn_block() * blocks;
    int32_t carry = 0;
    for (int32_t b0 = 0; b0 < blocks; b0 += 256) {
        const int32_t b = b0 + kn_thread();
        int32_t sum;
        const int32_t before = kn_block_exclusive_scan(b < blocks ? h[b] : 0, scratch, sum);
        if (b < blocks) h[b] = carry + before;
        carry += sum;
    }
    if (kn_thread() == 0) p.totals[kn_block()] = carry;
}

// SCANNED: k_route_scan has been there.  Else every workgroup sums the few histograms by itself, which takes less than a launch.
constexpr int ROUTE_FEW_BLOCKS = 64;
template <bool SCANNED> __global__ void __launch_bounds__(ROUTE_THREADS) k_route_place(RouteArgs p)
{
    extern __shared__ int32_t lds[];
    __shared__ int32_t scratch[16];
    const int32_t bins = p.E + 1, blocks = p.blocks, block = p.first + kn_block();
    int32_t *start = lds, *seen = start + bins, *total = seen; // (the totals are read before `seen` is written)
    for (int e = kn_thread(); e < bins; e += ROUTE_THREADS) {
        const int32_t *h = p.hist + (int64_t)e * blocks;
        if constexpr (SCANNED) {
            start[e] = h[block];
        } else {
            int32_t before = 0, all = 0;
            for (int b = 0; b < blocks; ++b) {
                before += b < block ? h[b] : 0;
                all += h[b];
            }
            start[e] = before;
            total[e] = all;
        }
    }
    __syncthreads();
    scan_counts(p, SCANNED ? p.totals : total, start, scratch, block == 0);
    __syncthreads();
    const int32_t p0 = block * ROUTE_TOKENS * p.k;
    place(p, p0, (int32_t)min((int64_t)p.T * p.k, (int64_t)p0 + ROUTE_TOKENS * p.k), start, seen);
}

__global__ void k_route_none(int32_t *offsets, int32_t n)
{
    const int i = kn_block() * 256 + kn_thread();
    if (i < n) offsets[i] = 0;
}

// Rows of logits as in `choose`.  The chosen experts' gradients are brought to their places through a row in the LDS.  renormalised:
// dl_j = w_j (g_j - sum of w g), zeros elsewhere; else, with the softmax p over all: dl_e = p_e ([e chosen] g_e - sum of w g).
// Measured: the same 32,768 rows, 7 us, 2.8 TB/s of mostly zeros.
template <typename T, int G, int V>
__global__ void __launch_bounds__(256) k_route_backward(RouteArgs p, const float *__restrict__ dweights, T *__restrict__ dlogits)
{
    __shared__ float lds[256 * V];
    const int lane = kn_thread() & 63, at = lane & (G - 1);
    float *row = lds + (kn_thread() & ~(G - 1)) * V; // (of one wavefront alone)
    const int32_t t = (p.first + kn_block()) * (256 / G) + kn_thread() / G;
    const bool there = t < p.T;
    const float other = __int_as_float(0x7fc00001); // marks an expert that was not chosen (no product here has these bits)
#pragma unroll
    for (int i = 0; i < V; ++i) row[at * V + i] = p.renorm ? 0.0f : other;
    int32_t e[2] = {-1, -1};
    float w[2] = {0.0f, 0.0f}, g[2] = {0.0f, 0.0f}, part = 0.0f;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        const int j = at + n * G;
        if (there && j < p.k) {
            const int64_t pair = (int64_t)t * p.k + j;
            e[n] = p.ids[pair];
            if ((uint32_t)e[n] >= (uint32_t)p.E) e[n] = -1;
            if (e[n] >= 0) { w[n] = p.weights[pair]; g[n] = dweights[pair]; }
            part += w[n] * g[n];
        }
    }
    const float mean = group_sum<G>(part);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int n = 0; n < 2; ++n)
        if (e[n] >= 0) row[e[n]] = w[n] * (g[n] - mean);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    float d[V];
#pragma unroll
    for (int i = 0; i < V; ++i) d[i] = row[at * V + i];
    if (!p.renorm) {
        float v[V], best = -INFINITY, s = 0.0f;
        load_logits<T, V>(p, t, there, at, v);
#pragma unroll
        for (int i = 0; i < V; ++i) best = fmaxf(best, v[i]);
        const float top = group_max<G>(best);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[i] = v[i] == -INFINITY ? 0.0f : expf(v[i] - top);
            s += v[i];
        }
        const float all = group_sum<G>(s);
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (__float_as_int(d[i]) == __float_as_int(other)) d[i] = top > -INFINITY ? v[i] / all * -mean : 0.0f;
    }
    if (!there) return;
    typedef T Piece __attribute__((ext_vector_type(V)));
    T *out = dlogits + (int64_t)t * p.E + at * V;
    if (p.wide) {
        Piece x;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (T)d[i];
        if (at * V < p.E) *(Piece *)out = x;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (at * V + i < p.E) out[i] = (T)d[i];
    }
}

// V neighbouring values of a row.  WHOLE: rows are made of such pieces, each on a multiple of its size; else they lie anywhere, and a row's
// last piece is its last V values, some of which the piece before has too (narrower rows: V = 1).  Rows of 2,468 values, 25,295 of 2 in bf16: pieces
// anywhere 213 us for the sums and their gradients, single values 582.
template <typename T, int V, bool WHOLE> struct RowPiece {
    typedef T Type __attribute__((ext_vector_type(V), aligned((WHOLE ? V : 1) * sizeof(T))));
};

// out[t] = sum over j of weights[t, j] y[slots[t, j]]: a thread per piece of a row, 16 bytes or one value.  Bound by its bytes.  STREAM: what
// is read and written once goes past the caches, where y does not stay in them anyway (us; kept in them, past them; rows of 4 x 2048 in
// bf16 but where said; y of the call before or another one): 32 MiB: 8 and 9; 64: 14 and 17; 128: 26 or 33, 30 or 32; 128 (2 each): 31 or 36, 36 or
// 37; 188 (fp32): 35 or 45, 42 or 44; 256: 68, 61 (5.5 TB/s); 256 (fp32): 66, 58; 256 (8 x 512): 65, 55; 1,024 (8 each): 242, 217.
constexpr int64_t COMBINE_STREAM = 3 << 26; // bytes of y
template <typename T, int V, bool WHOLE, bool STREAM>
__global__ void __launch_bounds__(256) k_combine(const T *__restrict__ y, const int32_t *__restrict__ slots, const float *__restrict__ weights,
                                                 int32_t M, int32_t D, int32_t Tn, int32_t k, T *__restrict__ out, int32_t first)
{
    typedef typename RowPiece<T, V, WHOLE>::Type Piece;
    const int32_t pieces = (D + V - 1) / V;
    const int64_t q = ((int64_t)first + kn_block()) * 256 + kn_thread();
    if (q >= (int64_t)Tn * pieces) return;
    const int32_t t = (int32_t)(q / pieces), c = WHOLE ? (int32_t)(q % pieces) * V : min((int32_t)(q % pieces) * V, D - V);
    float acc[V] = {};
    for (int j = 0; j < k; ++j) {
        const int32_t s = slots[(int64_t)t * k + j];
        if ((uint32_t)s >= (uint32_t)M) continue;
        const float w = weights ? weights[(int64_t)t * k + j] : 1.0f;
        const Piece *at = (const Piece *)(y + (int64_t)s * D + c);
        const Piece v = STREAM ? __builtin_nontemporal_load(at) : *at;
#pragma unroll
        for (int i = 0; i < V; ++i) acc[i] = fmaf(w, (float)v[i], acc[i]);
    }
    Piece r;
#pragma unroll
    for (int i = 0; i < V; ++i) r[i] = (T)acc[i];
    Piece *to = (Piece *)(out + (int64_t)t * D + c);
    if (STREAM) __builtin_nontemporal_store(r, to);
    else *to = r;
}

// dy[slots[t, j]] = weights[t, j] dout[t], dweights[t, j] = <dout[t], y[slots[t, j]]>: a wavefront per pair; a row of
// dout is read k times, but for the first from the caches.  Bound by its bytes (the same sizes, 604 MB: 118 us, 5.1 TB/s; a
// wavefront per row of dout, four pairs at a time: 143).
template <typename T, int V, bool WHOLE>
__global__ void __launch_bounds__(256) k_combine_backward(const T *__restrict__ dout, const T *__restrict__ y, const int32_t *__restrict__ slots,
                                                          const float *__restrict__ weights, int32_t M, int32_t D, int64_t pairs, int32_t k,
                                                          T *__restrict__ dy, float *__restrict__ dweights, int32_t first)
{
    typedef typename RowPiece<T, V, WHOLE>::Type Piece;
    const int lane = kn_thread() & 63;
    const int64_t q = ((int64_t)first + kn_block()) * 4 + (kn_thread() >> 6);
    if (q >= pairs) return;
    const int32_t s = slots[q];
    const bool there = (uint32_t)s < (uint32_t)M;
    const T *g = dout + (q / k) * D;
    const float w = weights ? weights[q] : 1.0f;
    float dot = 0.0f;
    if (there)
        for (int32_t own = lane * V; own < D; own += 64 * V) {
            const int32_t c = WHOLE ? own : min(own, D - V);
            const Piece a = *(const Piece *)(g + c);
            Piece r;
            if (dweights) {
                const Piece b = *(const Piece *)(y + (int64_t)s * D + c);
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (WHOLE || c + i >= own) dot = fmaf((float)a[i], (float)b[i], dot); // (each value once)
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

bool route_supported(int64_t T, int32_t E, int32_t k) { return E <= ROUTE_MAX_EXPERTS && k <= ROUTE_MAX_K && T <= KN_MAX_ROWS && T * k <= KN_MAX_ROWS; }
bool route_valid(int64_t T, int32_t E, int32_t k) { return T >= 0 && E >= 1 && k >= 1 && k <= E; }

// Calls f with the lanes that take a row of E logits and the logits that each of them holds.
template <int N> struct Int { static constexpr int n = N; };
template <typename F> int route_shape(int32_t E, F &&f)
{
    if (E <= 16) return f(Int<16>(), Int<1>());
    if (E <= 64) return f(Int<16>(), Int<4>());
    if (E <= 128) return f(Int<16>(), Int<8>());
    if (E <= 256) return f(Int<16>(), Int<16>());
    return f(Int<64>(), Int<16>());
}
// Whether every lane's V values are one aligned piece, in each of the rows
bool route_wide(const void *at, int64_t ld, int32_t E, int V, int item)
{
    const int bytes = V * item, align = bytes < 16 ? bytes : 16;
    return E % V == 0 && ((uintptr_t)at & (align - 1)) == 0 && ld * item % align == 0;
}

} // namespace

extern "C" int kn_route_workspace_bytes(int64_t T, int32_t E, int32_t k, int64_t *out_bytes)
{
    if (!out_bytes || !route_valid(T, E, k)) return KN_E_INVALID_ARG;
    if (!route_supported(T, E, k)) return KN_E_UNSUPPORTED;
    *out_bytes = T <= ROUTE_TOKENS ? 0 : kn_align_up((kn_div_up(T, ROUTE_TOKENS) + 1) * (E + 1) * 4, 256);
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
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)) return KN_E_WORKSPACE;
    const int32_t blocks = (int32_t)kn_div_up(T, ROUTE_TOKENS);
    RouteArgs p = {logits, ld, (int32_t)T, E, k, renormalize != 0, weights, ids, slots, rows, offsets, (int32_t *)workspace, (int32_t *)workspace + (int64_t)blocks * (E + 1), 0, blocks, 0};
    const size_t seen = (size_t)(ROUTE_THREADS / 64) * (E + 1) * 4, bins = (size_t)(E + 1) * 4;
    KN_TRY(kn_with_type(dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        return route_shape(E, [&](auto g, auto n) -> int {
            constexpr int G = decltype(g)::n, V = decltype(n)::n;
            p.wide = route_wide(logits, ld, E, V, sizeof(E_));
            return kn_launch(blocks, ROUTE_THREADS, [&](dim3 grid, int32_t first) {
                p.first = first;
                if (blocks == 1) hipLaunchKernelGGL((k_route_choose<E_, G, V, true>), grid, dim3(ROUTE_THREADS), 2 * bins + seen, st, p);
                else hipLaunchKernelGGL((k_route_choose<E_, G, V, false>), grid, dim3(ROUTE_THREADS), bins, st, p);
            });
        });
    }));
    if (blocks == 1) return KN_OK;
    if (blocks > ROUTE_FEW_BLOCKS) {
        hipLaunchKernelGGL(k_route_scan, dim3(E + 1), dim3(256), 0, st, p);
        KN_CHECK_LAUNCH();
    }
    return kn_launch(blocks, ROUTE_THREADS, [&](dim3 grid, int32_t first) {
        p.first = first;
        hipLaunchKernelGGL(blocks > ROUTE_FEW_BLOCKS ? k_route_place<true> : k_route_place<false>, grid, dim3(ROUTE_THREADS), bins + seen, st, p);
    });
}

extern "C" int kn_route_backward(void *stream, const void *logits, int32_t dtype, int64_t T, int32_t E, int64_t ld, int32_t k, int32_t renormalize,
                                 const float *weights, const int32_t *ids, const float *dweights, void *dlogits)
{
    if (!route_valid(T, E, k) || !kn_dtype_ok(dtype) || ld < E || (T > 0 && (!logits || !weights || !ids || !dweights || !dlogits))) return KN_E_INVALID_ARG;
    if (!route_supported(T, E, k)) return KN_E_UNSUPPORTED;
    if (T == 0) return KN_OK;
    RouteArgs p = {logits, ld, (int32_t)T, E, k, renormalize != 0, const_cast<float *>(weights), const_cast<int32_t *>(ids), nullptr, nullptr, nullptr, nullptr, nullptr, 0, 0, 0};
    return kn_with_type(dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        return route_shape(E, [&](auto g, auto n) -> int {
            constexpr int G = decltype(g)::n, V = decltype(n)::n;
            p.wide = route_wide(logits, ld, E, V, sizeof(E_)) && route_wide(dlogits, E, E, V, sizeof(E_));
            return kn_launch(kn_div_up(T, 256 / G), 256, [&](dim3 grid, int32_t first) {
                p.first = first;
                hipLaunchKernelGGL((k_route_backward<E_, G, V>), grid, dim3(256), 0, (hipStream_t)stream, p, dweights, (E_ *)dlogits);
            });
        });
    });
}

static int combine_check(int32_t dtype, int64_t M, int64_t D, int64_t T, int32_t k)
{
    if (M < 0 || D < 1 || T < 0 || k < 1 || !kn_dtype_ok(dtype)) return KN_E_INVALID_ARG;
    if (M > KN_MAX_ROWS || D > KN_MAX_WIDTH || T > KN_MAX_ROWS || T * k > KN_MAX_ROWS) return KN_E_UNSUPPORTED;
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
        const int64_t blocks = kn_div_up(T * (D < V ? D : kn_div_up(D, V)), 256);
        auto kernel = D < V ? k_combine<E_, 1, true, false> : !wide ? k_combine<E_, V, false, false>
                    : M * D * (int64_t)sizeof(E_) < COMBINE_STREAM ? k_combine<E_, V, true, false> : k_combine<E_, V, true, true>;
        return kn_launch(blocks, 256, [&](dim3 grid, int32_t first) {
            hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)stream, (const E_ *)y, slots, weights, (int32_t)M, D, (int32_t)T, k, (E_ *)out, first);
        });
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
        auto kernel = D < V ? k_combine_backward<E_, 1, true>
                    : whole_pieces(D, dtype, dout, dweights ? y : nullptr, dy) ? k_combine_backward<E_, V, true> : k_combine_backward<E_, V, false>;
        return kn_launch(kn_div_up(T * k, 4), 256, [&](dim3 grid, int32_t first) {
            hipLaunchKernelGGL(kernel, grid, dim3(256), 0, (hipStream_t)stream, (const E_ *)dout, (const E_ *)y, slots, weights, (int32_t)M, D, T * k, k,
                               (E_ *)dy, dweights, first);
        });
    });
}
