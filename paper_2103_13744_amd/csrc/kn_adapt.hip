// A layer that all networks share, with a low-rank product of each network's own beside it (kn_adapted_linear), and its gradients.
//
// y_i = x_i W + h_i B_e, h_i = s_e x_i A_e.  The second part is the first's contraction, made longer: a tile of rows meets n networks, and their B one
// under the other are a matrix of n times the rank rows, before which a row's h stands in the columns of its own network, between zeros.  So
// rows of all networks share tiles of W, whatever their order costs is the contraction of a few more steps, and y is written once.
#include "kn_tile.h"

#include <type_traits>

namespace {

// h(i, j) = scale_e sum over c of a(i, c) b_e(c, j), rows of `rp` values with zeros behind the rank; net(i): the row's network, or -1
struct Down {
    const void *a, *b;
    const float *scales;
    void *h;
    int32_t *net;
    const int32_t *offsets, *rows;
    int64_t lda, b_group, b_c, b_j;
    int32_t M, E, C, rank, rp, a_rows;
    int32_t first; // number of the launch's first workgroup
    // what the networks' second products are made with, `values` of each: whether a network's are not all finite is left in apart[network] (k_adapt_down)
    const void *next;
    int64_t values;
    int32_t *apart;
    float *wide; // nullable: h before it is rounded, in rows of rp (few rows)
};
// What the shared product takes beside its own operands
struct Beside {
    const void *h, *b;
    const int32_t *net, *apart; // apart: a network's b has infinities or NaN
    const float *wide;          // Down's
    int64_t b_group, b_c, b_j;
    int32_t E, rank, rp;
};

// Values k .. k + W - 1 of a contraction of C in steps of `step`
template <typename T> __device__ __forceinline__ typename KnFrag<T>::Type strided_piece(const T *at, int64_t step, int32_t k, int32_t C)
{
    typename KnFrag<T>::Type f;
#pragma unroll
    for (int q = 0; q < 16 / (int)sizeof(T); ++q) {
        const T v = at[min(k + q, C - 1) * step];
        f[q] = k + q < C ? v : (T)0.0f;
    }
    return f;
}

// 16 U rows of one network by 16 V columns: a workgroup's WAVES wavefronts take turns of AHEAD steps of the contraction, straight into registers, one asked
// for while another is multiplied, and are summed in the order of their numbers.  Where b's columns are contiguous (not its contraction) and in whole 16-byte
// pieces, 16-bit values are turned by the transposing read of an LDS that each wavefront has for itself; else they are fetched one by one, eight for a fragment.
// Bound by the rows' bytes: 16,384 rows of 12 networks, 2048 values, rank 32 in bf16: 24 us, 2.8 TB/s; 32,768 rows of 1024, rank 16: 18, 3.7 TB/s.  Two
// fragments of rows and four wavefronts; one to four, two to eight, two or four steps under way: 23 to 33.
enum { B_ROWS, B_COLS, B_PIECES };
template <typename T, int B, int U, int V, int WAVES, int AHEAD> struct Sums {
    static constexpr int W = 16 / sizeof(T), KS = 4 * W, LD = 16 * V + 4, WORDS = WAVES * 16 * U * LD;
    static constexpr bool COLS = B == B_COLS, TURN_B = B == B_PIECES;
    static_assert(!TURN_B || 16 * U * LD * 4 >= V * 1024, "");
    // Leaves each wavefront's sums over its turns among the steps [first, last) in `red`: row r and column j of wavefront w at (w 16 U + r) LD + j.  arow: the lane's rows
    // (column l % 16 of each 16), b: the first value of column j0, whose columns are b_j apart and whose contraction b_c.
    static __device__ __forceinline__ void run(const T *const arow[U], const T *b, int64_t b_c, int64_t b_j, int32_t columns, int32_t C, int32_t first, int32_t last, float *red)
    {
        typedef typename KnFrag<T>::Type Frag;
        const int tid = kn_thread(), lane = tid & 63, col = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        KN_LDS char *turn = (KN_LDS char *)red + wave * (16 * U * LD * 4);
        const T *brow[V];
#pragma unroll
        for (int v = 0; v < V; ++v) // (TURN_B: of the lane's v-th piece)
            brow[v] = b + (TURN_B ? min((lane + 64 * v) % (2 * V) * W, columns - W) : min(16 * v + col, columns - 1)) * b_j;
        kn_f32x4 acc[U][V] = {};
        struct Steps { Frag a[AHEAD][U], b[AHEAD][V]; };
        uint32_t none; // (rows are fetched as they lie)
        auto load = [&](Steps &x, int32_t s) { // (behind the last step: the row's end, unused)
#pragma unroll
            for (int n = 0; n < AHEAD; ++n) {
                const int32_t k = (s + n) * KS + W * g;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if constexpr (TURN_B) x.b[n][v] = *(const Frag *)(brow[v] + min((s + n) * KS + (lane + 64 * v) / (2 * V), C - 1) * b_c);
                    else if constexpr (COLS)
#pragma unroll
                        for (int q = 0; q < W; ++q) x.b[n][v][q] = brow[v][min(k + q, C - 1) * b_c];
                    else x.b[n][v] = kn_row_ask<T>(brow[v], k, C, false, none);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) x.a[n][u] = kn_row_ask<T>(arow[u], k, C, false, none);
            }
        };
        auto multiply = [&](Steps &x, int32_t s) {
#pragma unroll
            for (int n = 0; n < AHEAD; ++n) {
                const int32_t at = s + n, k = at * KS + W * g;
                if (at >= last) return;
                if ((at + 1) * KS > C) {
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        if constexpr (TURN_B) {
                            if (at * KS + (lane + 64 * v) / (2 * V) >= C) x.b[n][v] = Frag{};
                        } else if constexpr (COLS)
#pragma unroll
                            for (int q = 0; q < W; ++q) x.b[n][v][q] = k + q < C ? x.b[n][v][q] : (T)0.0f;
                        else kn_row_place<T>(x.b[n][v], brow[v], k, C, false, 0);
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) kn_row_place<T>(x.a[n][u], arow[u], k, C, false, 0);
                }
                if constexpr (TURN_B) {
#pragma unroll
                    for (int v = 0; v < V; ++v) *(KN_LDS Frag *)(turn + kn_turned_byte<V>((lane + 64 * v) / (2 * V), (lane + 64 * v) % (2 * V))) = x.b[n][v];
                    kn_lanes_meet();
#pragma unroll
                    for (int v = 0; v < V; ++v) x.b[n][v] = __builtin_bit_cast(Frag, kn_turned_frag<V>(turn, v, lane));
                    kn_lanes_meet();
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int v = 0; v < V; ++v) acc[u][v] = kn_mfma(x.b[n][v], x.a[n][u], acc[u][v]);
            }
        };
        if (!TURN_B && C < W) { // (rows of less than a piece: one step)
            if (first + wave < last) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const Frag fb = COLS ? strided_piece<T>(brow[v], b_c, W * g, C) : kn_any_piece<T>(brow[v], W * g, C);
#pragma unroll
                    for (int u = 0; u < U; ++u) acc[u][v] = kn_mfma(fb, kn_any_piece<T>(arow[u], W * g, C), acc[u][v]);
                }
            }
        } else if (first + wave * AHEAD < last) {
            constexpr int TURN = AHEAD * WAVES;
            Steps even, odd;
            load(even, first + wave * AHEAD);
            for (int32_t s = first + wave * AHEAD; s < last; s += 2 * TURN) {
                load(odd, s + TURN);
                multiply(even, s);
                load(even, s + 2 * TURN);
                multiply(odd, s + TURN);
            }
        }
        // (a lane's four results are neighbours in a row; a wavefront's part of `red` is what it turned b in)
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int v = 0; v < V; ++v) *(kn_f32x4 *)(red + ((wave * U + u) * 16 + col) * LD + 16 * v + 4 * g) = acc[u][v];
        __syncthreads();
    }
    static __device__ __forceinline__ kn_f32x4 of(const float *red, int r, int j)
    {
        kn_f32x4 y = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) y += *(const kn_f32x4 *)(red + (w * 16 * U + r) * LD + j);
        return y;
    }
};

// Whether a value is an infinity or a NaN
__device__ __forceinline__ bool not_finite(float v) { return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ bool not_finite(_Float16 v) { return (__builtin_bit_cast(uint16_t, v) & 0x7c00u) == 0x7c00u; }
__device__ __forceinline__ bool not_finite(__bf16 v) { return (__builtin_bit_cast(uint16_t, v) & 0x7f80u) == 0x7f80u; }

// The h of 16 U rows of one network, 16 V values.  WIDE: in 32 bits, too, where asked for
template <typename T, int B, int U, int V, int WAVES, int AHEAD, bool WIDE> __device__ __forceinline__ void down_piece(const Down &p, int32_t number, float *red)
{
    typedef Sums<T, B, U, V, WAVES, AHEAD> Core;
    const int tid = kn_thread(), col = tid & 15;
    const int ntiles = (p.rp + 16 * V - 1) / (16 * V);
    const KnPiece piece = kn_find_piece(p.offsets, p.E, p.M, 16 * U, number / ntiles);
    const int j0 = number % ntiles * 16 * V;
    if (piece.begin >= piece.end) return;
    const bool some = piece.group < p.E;
    const int64_t group = some ? piece.group : 0;
    const T *arow[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t i = min(piece.begin + 16 * u + col, piece.end - 1), src = p.rows ? p.rows[i] : i;
        arow[u] = (const T *)p.a + (int64_t)((uint32_t)src < (uint32_t)p.a_rows ? src : 0) * p.lda;
    }
    Core::run(arow, (const T *)p.b + group * p.b_group + j0 * p.b_j, p.b_c, p.b_j, p.rank - j0, p.C, 0,
              some && p.a_rows > 0 ? (p.C + Core::KS - 1) / Core::KS : 0, red);
    const float scale = p.scales && some ? p.scales[group] : 1.0f;
    for (int q = tid; q < 16 * U * 4 * V; q += WAVES * 64) {
        const int r = q / (4 * V), cj = q % (4 * V) * 4, j = j0 + cj;
        const int32_t i = piece.begin + r;
        if (i >= piece.end) continue;
        if (j == 0) p.net[i] = some ? piece.group : -1;
        if (j >= p.rp) continue;
        kn_f32x4 y = {0, 0, 0, 0};
        if (!p.rows || (uint32_t)p.rows[i] < (uint32_t)p.a_rows) y = Core::of(red, r, cj);
        typedef T Four __attribute__((ext_vector_type(4)));
        Four o;
#pragma unroll
        for (int n = 0; n < 4; ++n) o[n] = j + n < p.rank ? (T)(scale * y[n]) : (T)0.0f; // (16 bits: what the matrix cores take; fp16: what its range holds)
        *(Four *)((T *)p.h + (int64_t)i * p.rp + j) = o;
        if constexpr (WIDE && sizeof(T) == 2) {
            kn_f32x4 whole;
#pragma unroll
            for (int n = 0; n < 4; ++n) whole[n] = j + n < p.rank ? scale * y[n] : 0.0f;
            if (p.wide) *(kn_f32x4 *)(p.wide + (int64_t)i * p.rp + j) = whole;
        }
    }
}
// Whether the values that network `group` makes its second product with are all finite, if it has rows: a workgroup of its own, so that they are looked at while the
// first product is made
template <typename T, int WAVES> __device__ __forceinline__ void look_at(const Down &p, int32_t group, float *red)
{
    constexpr int W = 16 / sizeof(T), AHEAD = 8, STEP = WAVES * 64 * W;
    if (kn_offset(p.offsets, group, p.M) >= kn_offset(p.offsets, group + 1, p.M)) return;
    const int tid = kn_thread();
    const T *values = (const T *)p.next + group * p.values;
    bool any = false;
    if (p.values < W) {
        any = not_finite(values[min((int64_t)tid, p.values - 1)]);
    } else {
        for (int64_t at = (int64_t)tid * W; at < p.values; at += AHEAD * STEP) {
            typename KnAny<T>::Piece v[AHEAD];
#pragma unroll
            for (int n = 0; n < AHEAD; ++n) { // (behind the end: the last ones again)
                const int64_t from = at + n * STEP, last = p.values - W;
                v[n] = *(const typename KnAny<T>::Piece *)(values + (from < last ? from : last));
            }
#pragma unroll
            for (int n = 0; n < AHEAD; ++n)
#pragma unroll
                for (int q = 0; q < W; ++q) any |= not_finite((T)v[n][q]);
        }
    }
    int32_t *found = (int32_t *)red;
    const bool of_wave = __ballot(any) != 0;
    if ((tid & 63) == 0) found[tid >> 6] = of_wave;
    __syncthreads();
    if (tid == 0) {
        int32_t all = 0;
        for (int w = 0; w < WAVES; ++w) all |= found[w];
        p.apart[group] = all;
    }
}
template <typename T, int B, int U, int V, int WAVES, int AHEAD> __global__ void __launch_bounds__(WAVES * 64) k_adapt_down(Down p)
{
    __shared__ __align__(16) float red[Sums<T, B, U, V, WAVES, AHEAD>::WORDS];
    const int32_t block = p.first + kn_block();
    if (block < p.E) look_at<T, WAVES>(p, block, red);
    else down_piece<T, B, U, V, WAVES, AHEAD, false>(p, block - p.E, red);
}

// Few rows (16 U at most): one launch leaves h and the shared product's sums, cut into parts of the contraction so that all of w is on its way at once; the
// second adds the parts up and what h has to add.  One row 2048 x 2048: 5.2 and 3.4 us; 48 rows of 32 networks 2048 x 2560, rank 16: 9.2 and 4.3 (as tiles, with
// k_adapt_down before them, 17 and 20).
struct Few {
    float *sums;       // (parts, M, J)
    int32_t parts, each; // of so many steps
    int32_t products;  // workgroups of the shared product
};
constexpr int FEW_ROWS = 64;
template <typename T, int B, int U, int V, int DOWN_V> __global__ void __launch_bounds__(512) k_adapt_few(KnProduct p, Down down, Few few)
{
    typedef Sums<T, B, U, V, 8, 1> Core;
    typedef Sums<T, B, 1, DOWN_V, 8, 2> Low;
    __shared__ __align__(16) float red[Core::WORDS > Low::WORDS ? Core::WORDS : Low::WORDS];
    const int32_t block = kn_block();
    if (block >= few.products) {
        down_piece<T, B, 1, DOWN_V, 8, 2, true>(down, block - few.products, red);
        return;
    }
    const int tid = kn_thread(), col = tid & 15;
    const int ntiles = (p.J + 16 * V - 1) / (16 * V), number = kn_xcd_order(block, few.products);
    const int part = number / ntiles, j0 = number % ntiles * 16 * V;
    const T *arow[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int32_t i = min(16 * u + col, p.M - 1), src = p.rows ? p.rows[i] : i;
        arow[u] = (const T *)p.a + (int64_t)((uint32_t)src < (uint32_t)p.a_rows ? src : 0) * p.lda;
    }
    const int32_t steps = p.a_rows > 0 ? (p.C + Core::KS - 1) / Core::KS : 0;
    Core::run(arow, (const T *)p.b + j0 * p.b_j, p.b_c, p.b_j, p.J - j0, p.C, min(part * few.each, steps), min((part + 1) * few.each, steps), red);
    for (int q = tid; q < 16 * U * 4 * V; q += 512) {
        const int i = q / (4 * V), cj = q % (4 * V) * 4, j = j0 + cj;
        if (i >= p.M || j >= p.J) continue;
        const kn_f32x4 y = Core::of(red, i, cj);
        float *to = few.sums + ((int64_t)part * p.M + i) * p.J + j;
        if (p.J % 4 == 0) *(kn_f32x4 *)to = y;
        else
#pragma unroll
            for (int n = 0; n < 4; ++n)
                if (j + n < p.J) to[n] = y[n];
    }
}
// Four results of a row per thread.  H: what h is read in, T where it is what the caller gets (the result is made of that h, whose gradient the backward call takes, and is
// the same whether h is asked for or not); else, for the backward call's g, 32 bits, which is summed in fp32 here and needs no rounding.
template <typename T, typename H> __global__ void __launch_bounds__(128) k_adapt_few_join(KnProduct p, Beside beside, Few few)
{
    typedef T Four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
    typedef float Sum __attribute__((ext_vector_type(4), aligned(4)));
    const int32_t fours = (p.J + 3) / 4, q = kn_block() * 128 + kn_thread();
    const int32_t i = q / fours, j = q % fours * 4;
    if (i >= p.M) return;
    const bool whole = j + 4 <= p.J;
    const int32_t net = beside.net[i];
    float y[4] = {};
    for (int part = 0; part < few.parts; ++part) {
        const float *from = few.sums + ((int64_t)part * p.M + i) * p.J + j;
        Sum v = {};
        if (whole) v = *(const Sum *)from;
        else
#pragma unroll
            for (int n = 0; n < 4; ++n) v[n] = from[min(n, p.J - 1 - j)];
#pragma unroll
        for (int n = 0; n < 4; ++n) y[n] += v[n];
    }
    if ((uint32_t)net < (uint32_t)beside.E && p.a_rows > 0) {
        const H *h = (const H *)(sizeof(H) == sizeof(T) ? beside.h : beside.wide) + (int64_t)i * beside.rp;
        const T *b = (const T *)beside.b + net * beside.b_group + j * beside.b_j;
        float low[4] = {};
        if (beside.b_j == 1 && beside.b_c != 1) {
#pragma unroll 8
            for (int32_t c = 0; c < beside.rank; ++c) {
                Four v;
                if (whole) v = *(const Four *)(b + c * beside.b_c);
                else
#pragma unroll
                    for (int n = 0; n < 4; ++n) v[n] = b[c * beside.b_c + min(n, p.J - 1 - j)];
                const float a = (float)h[c];
#pragma unroll
                for (int n = 0; n < 4; ++n) low[n] = fmaf(a, (float)v[n], low[n]);
            }
        } else {
            constexpr int W = 16 / sizeof(T);
            for (int32_t c = 0; c < beside.rank; c += W) { // (h has zeros behind the rank)
                typedef H Piece __attribute__((ext_vector_type(W)));
                const Piece a = *(const Piece *)(h + c);
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const typename KnFrag<T>::Type v = kn_any_piece<T>(b + min(n, p.J - 1 - j) * beside.b_j, c, beside.rank);
#pragma unroll
                    for (int w = 0; w < W; ++w) low[n] = fmaf((float)a[w], (float)v[w], low[n]);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < 4; ++n) y[n] += low[n];
    }
    const bool out_of_x = p.rows && (uint32_t)p.rows[i] >= (uint32_t)p.a_rows;
    const int32_t src = p.mask_rows ? p.mask_rows[i] : i;
    const T *mask = p.mask && (uint32_t)src < (uint32_t)p.m_rows ? (const T *)p.mask + (int64_t)src * p.ldm + j : nullptr;
    Four o;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const int at = min(n, p.J - 1 - j);
        float v = out_of_x ? 0.0f : y[n];
        if (p.bias) v += (float)((const T *)p.bias)[j + at];
        if (p.relu) v = v > 0.0f || v != v ? v : 0.0f; // (a NaN stays one)
        if (p.mask && !(mask && (float)mask[at] > 0.0f)) v = 0.0f;
        o[n] = (T)v;
    }
    T *out = (T *)p.out + (int64_t)i * p.o_i + j;
    if (whole) *(Four *)out = o;
    else
#pragma unroll
        for (int n = 0; n < 4; ++n)
            if (j + n < p.J) out[n] = o[n];
}

// A stage of the rows' h, row-wise: row r's stand at columns slot_r * rp of the longer contraction
template <typename T, int R, int NW, bool DIRECT> struct LoadH {
    static constexpr int N = R / 8 / NW, CS = 128 / sizeof(T), W = 16 / sizeof(T);
    const T *at[N];
    int32_t first[N]; // column of the row's first value (negative: none)
    typename KnFrag<T>::Type held[DIRECT ? 1 : N];
    int32_t piece, rp;
    __device__ __forceinline__ void start(int wave, int lane, const T *h, int32_t width, int32_t begin, int32_t end, const KN_LDS int32_t *slots)
    {
        piece = (lane & 7) ^ (lane >> 3);
        rp = width;
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int r = (wave * N + t) * 8 + (lane >> 3);
            const int32_t slot = slots[r];
            first[t] = slot < 0 ? -1 : slot * rp;
            at[t] = h + (int64_t)min(begin + r, end - 1) * rp;
        }
    }
    __device__ __forceinline__ const T *from(int t, int s) const // (nullptr: zeros)
    {
        const int32_t q = s * CS + piece * W - first[t];
        return first[t] >= 0 && q >= 0 && q < rp ? at[t] + q : nullptr;
    }
    __device__ __forceinline__ void ask(int s)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const T *v = from(t, s);
            held[t] = typename KnFrag<T>::Type{};
            if (v) held[t] = *(const typename KnFrag<T>::Type *)v;
        }
    }
    __device__ __forceinline__ void fetch(KN_LDS char *tile, int wave, int lane, int s)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            if constexpr (DIRECT) {
                const T *v = from(t, s);
                kn_fetch(v ? (const void *)v : (const void *)&kn_zeros, tile + (wave * N + t) * 1024);
            } else {
                *(KN_LDS typename KnFrag<T>::Type *)(tile + (wave * N + t) * 1024 + lane * 16) = held[t];
            }
        }
    }
};
// A stage of the networks' B one under the other, column-wise (COLS) or row-wise, R columns of it
template <typename T, int R, int NW, int LIST, bool COLS, bool DIRECT> struct LoadB {
    static constexpr int CS = 128 / sizeof(T), W = 16 / sizeof(T), PR = R / W, RP = 64 / PR, N = COLS ? CS / RP / NW : R / 8 / NW;
    typename KnFrag<T>::Type held[DIRECT ? 1 : N];
    const T *b;
    int32_t nets[LIST]; // lane l's: of networks l, 64 + l, ..
    int64_t group, along, across;
    int32_t j0, J, count, rp, rank;
    __device__ __forceinline__ void start(const Beside &p, int32_t first, int32_t columns, const KN_LDS int32_t *of, int32_t n, int lane)
    {
        b = (const T *)p.b;
#pragma unroll
        for (int c = 0; c < LIST; ++c) nets[c] = of[64 * c + lane];
        group = p.b_group; along = p.b_c; across = p.b_j;
        j0 = first; J = columns; count = n; rp = p.rp; rank = p.rank;
    }
    // where the lane's piece t of stage s begins (nullptr: zeros), and how many of its values are there
    __device__ __forceinline__ const T *from(int wave, int lane, int t, int s, int32_t &left) const
    {
        int32_t c, k;
        if constexpr (COLS) {
            const int r = (wave * N + t) * RP + lane / PR;
            c = s * CS + r;
            k = ((lane % PR) ^ kn_col_swizzle<T, COLS ? R : 64>(r)) * W;
            if (DIRECT) k = min(k, J - j0 - W);
            left = J - j0 - k;
        } else {
            k = min((wave * N + t) * 8 + (lane >> 3), J - 1 - j0);
            c = s * CS + ((lane & 7) ^ (lane >> 3)) * W;
        }
        const int32_t slot = (uint32_t)c / (uint32_t)rp, q = c - slot * rp;
        if constexpr (!COLS) left = rank - q;
        int32_t net = __shfl(nets[0], slot & 63);
#pragma unroll
        for (int c = 1; c < LIST; ++c) {
            const int32_t more = __shfl(nets[c], slot & 63);
            net = slot >> 6 == c ? more : net;
        }
        if (slot >= count || net < 0 || q >= rank || left <= 0) return nullptr;
        return b + net * group + q * along + (j0 + k) * across;
    }
    __device__ __forceinline__ void ask(int wave, int lane, int s)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            int32_t left;
            const T *v = from(wave, lane, t, s, left);
            held[t] = typename KnFrag<T>::Type{};
            if (v) held[t] = kn_any_piece<T>(v, 0, left);
        }
    }
    __device__ __forceinline__ void fetch(KN_LDS char *tile, int wave, int lane, int s)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            if constexpr (DIRECT) {
                int32_t left;
                const T *v = from(wave, lane, t, s, left);
                kn_fetch(v ? (const void *)v : (const void *)&kn_zeros, tile + (wave * N + t) * 1024);
            } else {
                *(KN_LDS typename KnFrag<T>::Type *)(tile + (wave * N + t) * 1024 + lane * 16) = held[t];
            }
        }
    }
};

// Tiles of BM x BN results, WR x WC wavefronts, NB stages in the LDS, of which one is multiplied while the others are fetched, as in the grouped products; behind the
// stages of the shared contraction come those of the tile's networks.  There a row meets other networks' values with zeros, and a zero times what is not finite is a
// NaN: networks with such values are left out, and their rows get their part at the end, value by value.  COLS: the columns of w and b are contiguous (else the contraction is).  DIRECT: rows
// of whole 16-byte pieces throughout.
// Measured: 16,384 rows of 12 networks 2048 x 2048, rank 32 in bf16: 165 us, 845 TFLOP/s (150 to 167 from day to day), where one product of the library of 8192 x 8192 x 8192
// reaches 1,221.  The networks that a tile meets add their number times the rank to the contraction: two and a rank of 32 one stage of 64, but 32 of rank 64 as much as W's 2048.  A
// network that is left out costs its rows: one of 129 rows 175 -> 254 us, one of 14,813 816, for the whole call.  Tiles of
// 192 x 128 (too few registers for two workgroups at a time): 222.
// (128 x 128: registers for two workgroups at a time)
template <typename T, bool COLS, bool DIRECT, int BM, int BN, int WR, int WC, int NB>
__global__ void __launch_bounds__(WR * WC * 64, DIRECT && BM == 128 ? 4 : 1) k_adapt_up(KnProduct p, Beside beside, int32_t blocks)
{
    constexpr int NW = WR * WC, STAGE = (BM + BN) * 128, U = BM / WR / 16, V = BN / WC / 16, CS = 128 / sizeof(T), LIST = (BM + 63) / 64;
    typedef typename KnFrag<T>::Type Frag;
    static_assert(DIRECT || NB == 2, "");
    static_assert(BM <= NW * 64, "a thread looks at a row");
    typedef KnRowLoader<T, BM, NW, DIRECT> LoadA;
    constexpr int BYTES = NB * STAGE > NW * 16 * (BN / WC + 4) * 4 ? NB * STAGE : NW * 16 * (BN / WC + 4) * 4;
    __shared__ __align__(16) char lds_[BYTES];
    KN_LDS char *lds = (KN_LDS char *)lds_;
    const int tid = kn_thread(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ntiles = (p.J + BN - 1) / BN;
    const int32_t number = kn_xcd_order(p.first + kn_block(), blocks);
    const int32_t begin = number / ntiles * BM, end = min(p.M, begin + BM);
    const int j0 = number % ntiles * BN;
    LoadH<T, BM, NW, DIRECT> lh;
    LoadB<T, BN, NW, LIST, COLS, DIRECT> lo;
    int32_t count = 0;
    bool apart = false; // networks that are left out
    { // (in the stages' LDS, before they are there: with more of it there would be one workgroup at a time)
        KN_LDS int32_t *slots = (KN_LDS int32_t *)lds, *nets = slots + BM, *met = nets + 64 * LIST; // a row's place among the tile's networks (-1: none), the
        const int32_t i = begin + tid;                                                         // networks, how many begin in a wavefront's rows
        const bool in = tid < BM && i < end;
        const int32_t net = in ? beside.net[i] : -1, before = in && tid > 0 ? beside.net[i - 1] : -1;
        const bool known = (uint32_t)net < (uint32_t)beside.E, left_out = known && beside.apart[net] != 0, begins = known && net != before;
        const uint64_t all = __ballot(begins), out = __ballot(left_out);
        if (lane == 0) {
            met[wave] = __popcll(all);
            met[NW + wave] = out != 0;
        }
        __syncthreads();
        int32_t rank = __popcll(all & ((2ull << lane) - 1)) - 1;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (w < wave) rank += met[w];
            count += met[w];
            apart |= met[NW + w] != 0;
        }
        if (tid < BM) slots[tid] = known && !left_out ? rank : -1;
        if (begins) nets[rank] = left_out ? -1 : net; // (it keeps its place: the others' sums are as they were)
        count = __builtin_amdgcn_readfirstlane(count); // (alike for all lanes)
        apart = __builtin_amdgcn_readfirstlane(apart);
        __syncthreads();
        lh.start(wave, lane, (const T *)beside.h, beside.rp, begin, end, slots);
        lo.start(beside, j0, p.J, nets, count, lane);
        __syncthreads();
    }
    const T *a = (const T *)p.a, *b = (const T *)p.b;
    LoadA la;
    la.start(wave, lane, [&](int r) {
        const int32_t i = min(begin + r, end - 1);
        const int32_t src = p.rows ? p.rows[i] : i;
        return a + (int64_t)((uint32_t)src < (uint32_t)p.a_rows ? src : 0) * p.lda;
    });
    KnRowLoader<T, BN, NW, DIRECT> lbr;
    KnColLoader<T, BN, NW, DIRECT> lbc;
    if constexpr (COLS) lbc.start(wave, lane, b + j0, p.b_c, p.J - j0);
    else lbr.start(wave, lane, [&](int r) { return b + (int64_t)min(j0 + r, p.J - 1) * p.b_j; });
    const int32_t C = p.a_rows > 0 ? p.C : 0, shared = (C + CS - 1) / CS, steps = C > 0 ? shared + (count * beside.rp + CS - 1) / CS : 0;
    constexpr int LOADS = LoadA::N + (COLS ? lbc.N : lbr.N); // a wavefront's, per stage
    static_assert(LOADS == lh.N + lo.N, "");
    constexpr int LATER = DIRECT ? (NB - 2) * LOADS : 63; // (loads into registers are waited for where they are put down)
    auto fetch = [&](int s, int at) {
        KN_LDS char *tile = lds + at * STAGE;
        if (s < shared) {
            la.fetch(tile, wave, lane, C - s * CS);
            if constexpr (COLS) lbc.fetch(tile + BM * 128, wave, lane, C - s * CS);
            else lbr.fetch(tile + BM * 128, wave, lane, C - s * CS);
        } else {
            lh.fetch(tile, wave, lane, s - shared);
            lo.fetch(tile + BM * 128, wave, lane, s - shared);
        }
        if (!DIRECT && s + 1 >= shared && s + 1 < steps) {
            lh.ask(s + 1 - shared);
            lo.ask(wave, lane, s + 1 - shared);
        }
    };
    const int wi = (wave / WC) * (BM / WR), wj = (wave % WC) * (BN / WC);
    kn_f32x4 acc[U][V] = {};
    Frag fa[2][U], fb[2][V];
    auto read = [&](int at, int kk) {
        const KN_LDS char *ta = lds + at * STAGE, *tb = ta + BM * 128;
#pragma unroll
        for (int u = 0; u < U; ++u) fa[kk][u] = kn_row_frag<T>(ta, wi + 16 * u, kk, lane);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if constexpr (COLS) fb[kk][v] = kn_col_frag<T, BN>(tb, wj + 16 * v, kk, lane);
            else fb[kk][v] = kn_row_frag<T>(tb, wj + 16 * v, kk, lane);
        }
    };
    auto march = [&](auto rows_there) {
        constexpr bool ROWS = decltype(rows_there)::value;
        auto multiply = [&](int kk) {
            if constexpr (ROWS) {
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int v = 0; v < V; ++v) acc[u][v] = kn_mfma(fb[kk][v], fa[kk][u], acc[u][v]);
                kn_interleave<U, V, T, COLS>();
            }
        };
        if constexpr (ROWS) read(0, 0);
        for (int s = 0, at = 0; s < steps; ++s) {
            const int next = at + 1 == NB ? 0 : at + 1;
            if constexpr (ROWS) read(at, 1);
            multiply(0);
            if (s + NB <= steps) kn_stage_barrier<LATER>();
            else kn_stage_barrier<0>();
            if (s + NB < steps) fetch(s + NB, at);
            if constexpr (ROWS) read(next, 0); // (behind the last stage: what happens to lie there, unused)
            multiply(1);
            at = next;
        }
    };
    if (steps > 0) {
        la.ask_first(C);
        if constexpr (COLS) lbc.ask_first(wave, lane, C);
        else lbr.ask_first(C);
        for (int s = 0; s < NB && s < steps; ++s) fetch(s, s);
        if (DIRECT && steps >= NB) kn_stage_barrier<(NB - 1) * LOADS>();
        else kn_stage_barrier<0>();
        if (WR == 1 || begin + wi < end) march(std::true_type());
        else march(std::false_type());
    }
    kn_stage_barrier(); // (the tiles' LDS is used again)
    // 16 rows of the wavefront's results at a time, in LDS of its own
    constexpr int WN = BN / WC, LD = WN + 4, LR = WN / 8; // LR lanes take a row
    KN_LDS float *mine = (KN_LDS float *)(lds + wave * (16 * LD * 4));
    static_assert(64 % LR == 0, "");
    const int cj = lane % LR * 8;
    const int32_t j = j0 + wj + cj;
    float add[8];
    kn_bias_of<T>(p, true, 0, j, add);
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int v = 0; v < V; ++v) *(KN_LDS kn_f32x4 *)(mine + (lane & 15) * LD + 16 * v + (lane >> 4) * 4) = acc[u][v];
        kn_lanes_meet();
#pragma unroll
        for (int h = 0; h < (16 * LR + 63) / 64; ++h) {
            const int r = h * (64 / LR) + lane / LR;
            const int32_t i = begin + wi + 16 * u + r;
            if (r >= 16 || i >= end || j >= p.J) continue;
            const kn_f32x4 lo4 = *(const KN_LDS kn_f32x4 *)(mine + r * LD + cj), hi4 = *(const KN_LDS kn_f32x4 *)(mine + r * LD + cj + 4);
            float y[8] = {lo4[0], lo4[1], lo4[2], lo4[3], hi4[0], hi4[1], hi4[2], hi4[3]};
            if (apart && C > 0) {
                const int32_t net = beside.net[i];
                if ((uint32_t)net < (uint32_t)beside.E && beside.apart[net]) {
                    const T *h = (const T *)beside.h + (int64_t)i * beside.rp, *v = (const T *)beside.b + net * beside.b_group;
#pragma unroll 1
                    for (int q = 0; q < 8; ++q) {
                        const T *column = v + min(j + q, p.J - 1) * beside.b_j;
                        float low = 0.0f;
#pragma unroll 1
                        for (int32_t c = 0; c < beside.rank; ++c) low = fmaf((float)h[c], (float)column[c * beside.b_c], low);
#pragma unroll
                        for (int n = 0; n < 8; ++n) y[n] += n == q ? low : 0.0f;
                    }
                }
            }
            kn_finish<T>(p, true, i, j, add, y);
        }
        kn_lanes_meet();
    }
}

// Rows of `rank` values in rows of whole 16-byte pieces, zeros behind them, of the networks that have rows: a thread per piece.  Else one factor's short rows would send the
// whole shared product through registers (16,384 rows of 12 networks 2048 x 2048 of rank 4, contraction contiguous, in bf16: 249 us, 172 with this).
template <typename T> __global__ void __launch_bounds__(256) k_adapt_pad(const T *__restrict__ b, T *__restrict__ to, const int32_t *__restrict__ offsets, int32_t M, int32_t rows,
                                                                        int32_t rank, int32_t rp, int32_t blocks, int32_t first)
{
    constexpr int W = 16 / sizeof(T);
    const int32_t block = first + kn_block(), net = block / blocks, pieces = rp / W;
    if (kn_offset(offsets, net, M) >= kn_offset(offsets, net + 1, M)) return;
    const int64_t q = (int64_t)(block % blocks) * 256 + kn_thread();
    if (q >= (int64_t)rows * pieces) return;
    const int64_t row = (int64_t)net * rows + q / pieces;
    const int32_t k = (int32_t)(q % pieces) * W;
    *(typename KnFrag<T>::Type *)(to + row * rp + k) = kn_any_piece<T>(b + row * rank, k, rank);
}

// strided_piece of a small matrix (less than 4 GiB) at an address that all lanes share: offsets of 32 bits, one addition for a value.  `at`: of the lane's first
// value; `step`: bytes from one to the next
template <typename T> __device__ __forceinline__ typename KnFrag<T>::Type strided_near(const T *base, uint32_t at, uint32_t step, int32_t k, int32_t C, bool tail)
{
    typename KnFrag<T>::Type f;
    uint32_t off = at + (uint32_t)k * step;
    const uint32_t last = at + (uint32_t)(C - 1) * step;
#pragma unroll
    for (int q = 0; q < 16 / (int)sizeof(T); ++q, off += step) f[q] = *(const T *)((const char *)base + min(off, last));
    if (tail)
#pragma unroll
        for (int q = 0; q < 16 / (int)sizeof(T); ++q) f[q] = k + q < C ? f[q] : (T)0.0f;
    return f;
}

// Layers of the small networks' kind (contraction up to KF fragments, columns up to V of 16, or a few such tiles; a rank of up to 16), of any sizes, strides and
// alignment: a wavefront takes SMALL_ROWS rows of one network by itself, the shared weights in the LDS, as fragments, and the network's own in its registers, and
// makes h and y at once: rows are read once, and nothing goes through memory between the two products.  Lanes hand each other h where they hold four of a row's values
// as results and take eight as an operand (16 bits; in fp32 both are the same four).  262,145 rows of 4,096 networks 63 x 32, rank 4: 45 us in fp32 (2.4 TB/s; the
// matrix cores are busy a third of the time), 25 in bf16; with the shared weights in registers and by 64-bit addresses 49 and 29.
constexpr int SMALL_ROWS = 32, SMALL_WAVES = 4, SMALL_MOST = 128; // (the last: the widest)
template <typename T, bool COLS, int KF, int V, bool ODD>
__global__ void __launch_bounds__(SMALL_WAVES * 64) k_adapt_small(KnProduct p, Down down, Beside beside, int32_t pieces)
{
    constexpr int W = KnSmallFrag<T>::W, KS = KnSmallFrag<T>::KS, SUBS = SMALL_ROWS / 16, PAIR = W / 4, RUNS = V / PAIR;
    typedef typename KnFrag<T>::Type Frag;
    typedef T Run __attribute__((ext_vector_type(W), aligned(sizeof(T)))); // wherever they lie
    typedef T Four __attribute__((ext_vector_type(4)));
    __shared__ __align__(16) T rows_of[SMALL_WAVES][16 * 16 * V + W]; // 16 rows of results of a wavefront, as they follow one another
    const int lane = kn_thread() & 63, col = lane & 15, g = lane >> 4;
    __shared__ __align__(16) Frag shared[KF][V][64];
    const int wave = __builtin_amdgcn_readfirstlane(kn_thread() >> 6);
    T *line = rows_of[wave];
    const int ntiles = (p.J + 16 * V - 1) / (16 * V), block = p.first + kn_block();
    const int32_t number = block / ntiles * SMALL_WAVES + wave, j0 = block % ntiles * 16 * V, C = p.C;
    const bool any = p.a_rows > 0;
    // A lane's four results of W / 4 products are neighbours, W of them: the products' columns are dealt out in fours
    auto column = [&](int v) { return min(j0 + v / PAIR * (16 * PAIR) + (col >> 2) * W + v % PAIR * 4 + (col & 3), p.J - 1); };
#pragma unroll
    for (int f = 0; f < KF * V / SMALL_WAVES; ++f) {
        const int n = f * SMALL_WAVES + wave, k = n / V, v = n % V;
        const int32_t c = k * KS + g * W, j = column(v);
        Frag w;
        if constexpr (COLS) {
            w = strided_near<T>((const T *)p.b, j * sizeof(T), (uint32_t)p.b_c * sizeof(T), c, C, (k + 1) * KS > C);
        } else {
            uint32_t fifth = 0;
            const bool odd = ODD && (((uintptr_t)p.b / sizeof(T) | p.b_j) & 1);
            w = kn_row_ask<T>((const T *)p.b + j * p.b_j, c, C, odd, fifth);
            if (C >= W) kn_row_place<T>(w, (const T *)p.b + j * p.b_j, c, C, odd, fifth);
        }
        shared[k][v][lane] = w;
    }
    const KnPiece piece = number < pieces ? kn_find_piece(down.offsets, down.E, p.M, SMALL_ROWS, number) : KnPiece{0, 0, 0};
    __syncthreads();
    if (piece.begin >= piece.end) return;
    const bool some = piece.group < down.E;
    const int64_t group = some ? piece.group : 0;
    Frag fa[SUBS][KF], la[KF], lb[V];
    bool there[SUBS];
    if (any) {
        const T *arow[SUBS], *lrow = (const T *)down.b + group * down.b_group + min(col, down.rank - 1) * down.b_j;
        uint32_t fifth_a[SUBS][KF], fifth_l[KF];
        const bool odd_a = ODD && (((uintptr_t)p.a / sizeof(T) | p.lda) & 1), odd_l = ODD && (((uintptr_t)down.b / sizeof(T) | down.b_j) & 1);
#pragma unroll
        for (int s = 0; s < SUBS; ++s) {
            const int32_t i = min(piece.begin + 16 * s + col, piece.end - 1), src = p.rows ? p.rows[i] : i;
            there[s] = (uint32_t)src < (uint32_t)p.a_rows;
            arow[s] = (const T *)p.a + (int64_t)(there[s] ? src : 0) * p.lda;
        }
#pragma unroll
        for (int k = 0; k < KF; ++k) {
            const int32_t c = k * KS + g * W;
            if constexpr (COLS) la[k] = strided_near<T>((const T *)down.b + group * down.b_group, min(col, down.rank - 1) * sizeof(T), (uint32_t)down.b_c * sizeof(T), c, C, (k + 1) * KS > C);
            else la[k] = kn_row_ask<T>(lrow, c, C, odd_l, fifth_l[k]);
        }
#pragma unroll
        for (int s = 0; s < SUBS; ++s)
#pragma unroll
            for (int k = 0; k < KF; ++k) fa[s][k] = kn_row_ask<T>(arow[s], k * KS + g * W, C, odd_a, fifth_a[s][k]);
        const T *b = (const T *)beside.b + group * beside.b_group;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int32_t j = column(v);
            if constexpr (COLS) lb[v] = strided_near<T>(b, j * sizeof(T), (uint32_t)beside.b_c * sizeof(T), g * W, beside.rank, true);
            else lb[v] = kn_any_piece<T>(b + j * beside.b_j, g * W, beside.rank);
        }
        if (C >= W && (ODD || C % W)) {
#pragma unroll
            for (int k = 0; k < KF; ++k) {
                if (!ODD && (k + 1) * KS <= C) continue;
                const int32_t c = k * KS + g * W;
#pragma unroll
                for (int s = 0; s < SUBS; ++s) kn_row_place<T>(fa[s][k], arow[s], c, C, odd_a, fifth_a[s][k]);
                if constexpr (!COLS) kn_row_place<T>(la[k], lrow, c, C, odd_l, fifth_l[k]);
            }
        }
    }
    const float scale = some && down.scales ? down.scales[group] : 1.0f;
    const bool together = p.J % W != 0 && ntiles == 1; // rows that follow one another without whole pieces of their own: stored as one line
    // W neighbours j .. of a row of J (behind its end: the last one, unused)
    auto run = [&](const T *row, int32_t j) {
        Run f;
        if (j + W <= p.J) f = *(const Run *)(row + j);
        else
#pragma unroll
            for (int r = 0; r < W; ++r) f[r] = row[min(j + r, p.J - 1)];
        return f;
    };
    const T *bias = (const T *)p.bias, *mask = (const T *)p.mask;
    Run add[RUNS], m[SUBS][RUNS]; // (a lane's columns are j0 + 4 W n + W g .. + W - 1)
#pragma unroll
    for (int n = 0; n < RUNS; ++n) add[n] = bias ? run(bias, min(j0 + 4 * W * n + W * g, p.J - 1)) : Run{};
    if (mask) { // (asked for before the first result is stored, not one after the other's)
#pragma unroll
        for (int s = 0; s < SUBS; ++s) {
            const int32_t i = min(piece.begin + 16 * s + col, piece.end - 1), src = p.mask_rows ? p.mask_rows[i] : i;
            const bool in = (uint32_t)src < (uint32_t)p.m_rows;
#pragma unroll
            for (int n = 0; n < RUNS; ++n) {
                m[s][n] = Run{};
                if (in) m[s][n] = run(mask + (int64_t)src * p.ldm, min(j0 + 4 * W * n + W * g, p.J - 1));
            }
        }
    }
    kn_f32x4 sums[SUBS][V] = {}, lows[SUBS] = {};
    if (any) {
#pragma unroll
        for (int k = 0; k < KF; ++k) {
#pragma unroll
            for (int s = 0; s < SUBS; ++s) lows[s] = kn_mfma(la[k], fa[s][k], lows[s]);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const Frag w = shared[k][v][lane];
#pragma unroll
                for (int s = 0; s < SUBS; ++s) sums[s][v] = kn_mfma(w, fa[s][k], sums[s][v]);
            }
        }
    }
#pragma unroll
    for (int s = 0; s < SUBS; ++s) {
        const int32_t i = piece.begin + 16 * s + col;
        if (piece.begin + 16 * s >= piece.end) break;
        kn_f32x4 *acc = sums[s];
        const kn_f32x4 low = lows[s];
        Four h; // of row `col`: values 4 g .. + 3
#pragma unroll
        for (int r = 0; r < 4; ++r) h[r] = some && any && there[s] && 4 * g + r < down.rank ? (T)(scale * low[r]) : (T)0.0f;
        if (j0 == 0 && i < piece.end && 4 * g < down.rp) *(Four *)((T *)down.h + (int64_t)i * down.rp + 4 * g) = h;
        if (any) {
            Frag hf;
            if constexpr (sizeof(T) == 4) {
                hf = h;
            } else { // values 8 g .. + 7: those of lanes 2 g and 2 g + 1 of the row's four (behind the 16th: zeros, as B's are)
                union { Four v; uint32_t u[2]; } mine;
                union { Frag v; uint32_t u[4]; } all;
                mine.v = h;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const uint32_t v = __shfl(mine.u[q & 1], (2 * (g & 1) + (q >> 1)) * 16 + col);
                    all.u[q] = g < 2 ? v : 0;
                }
                hf = all.v;
            }
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] = kn_mfma(lb[v], hf, acc[v]);
            if (!there[s])
#pragma unroll
                for (int v = 0; v < V; ++v) acc[v] = kn_f32x4{0, 0, 0, 0};
        }
        T *out = (T *)p.out + (int64_t)i * p.o_i, *first = (T *)p.out + (int64_t)(i - col) * p.o_i;
        const int shift = (int)((uintptr_t)first / sizeof(T) % W); // (of the first result in its 16 bytes)
#pragma unroll
        for (int n = 0; n < RUNS; ++n) {
            const int32_t j = j0 + 4 * W * n + W * g;
            if (j >= p.J || i >= piece.end) continue;
            Run o;
#pragma unroll
            for (int r = 0; r < W; ++r) {
                float y = acc[n * PAIR + r / 4][r % 4];
                if (bias) y += (float)add[n][r];
                if (p.relu) y = y > 0.0f || y != y ? y : 0.0f; // (a NaN stays one)
                if (mask && !((float)m[s][n][r] > 0.0f)) y = 0.0f;
                o[r] = (T)y;
            }
            if (together) {
#pragma unroll
                for (int r = 0; r < W; ++r)
                    if (j + r < p.J) line[shift + col * p.J + j + r] = o[r];
            } else if (j + W <= p.J) {
                *(Run *)(out + j) = o;
            } else {
#pragma unroll
                for (int r = 0; r < W; ++r)
                    if (j + r < p.J) out[j + r] = o[r];
            }
        }
        if (together) {
            kn_lanes_meet();
            const int end = shift + min(16, piece.end - (i - col)) * p.J;
            for (int q = lane * W; q < end; q += 64 * W) {
                if (q >= shift && q + W <= end) *(Frag *)(first + q - shift) = *(const Frag *)(line + q);
                else
                    for (int r = max(q, shift); r < min(q + W, end); ++r) first[r - shift] = line[r];
            }
            kn_lanes_meet();
        }
    }
}

template <typename T, bool COLS, int KF, int V, bool ODD> int launch_small_of(hipStream_t st, const Down &down, const KnProduct &p, const Beside &beside)
{
    const int64_t pieces = kn_pieces(p.M, down.E, SMALL_ROWS);
    return kn_launch(kn_div_up(pieces, SMALL_WAVES) * kn_div_up(p.J, 16 * V), SMALL_WAVES * 64, [&](dim3 grid, int32_t first) {
        KnProduct q = p;
        q.first = first;
        hipLaunchKernelGGL((k_adapt_small<T, COLS, KF, V, ODD>), grid, dim3(SMALL_WAVES * 64), 0, st, q, down, beside, (int32_t)pieces);
    });
}
template <typename T, bool COLS, int KF, int V> int launch_small_v(hipStream_t st, const Down &down, const KnProduct &p, const Beside &beside)
{
    if constexpr (sizeof(T) == 2) { // rows that begin between two words
        if (((uintptr_t)p.a / 2 | p.lda | (COLS ? 0 : (uintptr_t)p.b / 2 | p.b_j | (uintptr_t)down.b / 2 | down.b_j)) & 1) return launch_small_of<T, COLS, KF, V, true>(st, down, p, beside);
    }
    return launch_small_of<T, COLS, KF, V, false>(st, down, p, beside);
}
template <typename T, bool COLS> int launch_small(hipStream_t st, const Down &down, const KnProduct &p, const Beside &beside)
{
    const int kf = (p.C + KnSmallFrag<T>::KS - 1) / KnSmallFrag<T>::KS;
    if constexpr (sizeof(T) == 4) {
        if (kf > 4) return launch_small_v<T, COLS, 8, 2>(st, down, p, beside);
        return p.J <= 32 ? launch_small_v<T, COLS, 4, 2>(st, down, p, beside) : launch_small_v<T, COLS, 4, 4>(st, down, p, beside);
    } else {
        if (kf > 2) return launch_small_v<T, COLS, 4, 4>(st, down, p, beside);
        return p.J <= 32 ? launch_small_v<T, COLS, 2, 2>(st, down, p, beside) : launch_small_v<T, COLS, 2, 4>(st, down, p, beside);
    }
}

template <typename T, int B, int U, int V, int WAVES, int AHEAD> int launch_down_of(hipStream_t st, const Down &p)
{
    return kn_launch(p.E + kn_pieces(p.M, p.E, 16 * U) * kn_div_up(p.rp, 16 * V), WAVES * 64, [&](dim3 grid, int32_t first) {
        Down q = p;
        q.first = first;
        hipLaunchKernelGGL((k_adapt_down<T, B, U, V, WAVES, AHEAD>), grid, dim3(WAVES * 64), 0, st, q);
    });
}
// One wavefront where the contraction is short, and where one looks at a network's second factor in a single go (8 KiB); else its fetches are waited for one after
// the other.  Measured (us, whole call, one / four / eight wavefronts): 65,536 rows of 4,096 networks 64 x 136, rank 4 in bf16, factors of 1 KiB, 33 / 76 / 76; 20,000 of 1,000
// 128 x 256, rank 8, 4 KiB, 19 / 26 / 26, in fp32, 8 KiB, 38 / 44 / 44; 4,096 of 128 128 x 512, rank 16 in bf16, 16 KiB, 22 / 15 / 15; 16,384 of 64 128 x 1024, 32 KiB, 26 / 24 / 26; 4,096
// of one 256 x 2048, rank 64, 256 KiB, 44 / 23 / 23.
template <typename T, int B, int V> int launch_down_columns(hipStream_t st, const Down &p)
{
    if (p.C * (int64_t)sizeof(T) <= 512 && p.values * (int64_t)sizeof(T) <= 8192) return launch_down_of<T, B, 2, V, 1, 2>(st, p);
    if (p.M / p.E >= 32) return launch_down_of<T, B, 2, V, 4, 2>(st, p);
    return launch_down_of<T, B, 1, V, 8, 2>(st, p);
}
template <typename T, int B> int launch_down_of_b(hipStream_t st, const Down &p)
{
    if (p.rp <= 16) return launch_down_columns<T, B, 1>(st, p);
    return p.rp <= 32 ? launch_down_columns<T, B, 2>(st, p) : launch_down_columns<T, B, 4>(st, p);
}
template <typename T> int launch_down(hipStream_t st, const Down &p, bool cols)
{
    if (!cols) return launch_down_of_b<T, B_ROWS>(st, p);
    if constexpr (sizeof(T) == 2) {
        if (p.rank % 8 == 0 && p.C >= 8 && ((uintptr_t)p.b & 15) == 0) return launch_down_of_b<T, B_PIECES>(st, p);
    }
    return launch_down_of_b<T, B_COLS>(st, p);
}

template <typename T, bool COLS, bool DIRECT, int BM, int BN, int WR, int WC, int NB> int launch_tiles(hipStream_t st, const KnProduct &p, const Beside &beside)
{
    const int64_t blocks = kn_div_up(p.M, BM) * kn_div_up(p.J, BN);
    return kn_launch(blocks, WR * WC * 64, [&](dim3 grid, int32_t first) {
        KnProduct q = p;
        q.first = first;
        hipLaunchKernelGGL((k_adapt_up<T, COLS, DIRECT, BM, BN, WR, WC, NB>), grid, dim3(WR * WC * 64), 0, st, q, beside, (int32_t)blocks);
    });
}

// Whether the rows of all operands are made of whole 16-byte pieces
template <typename T, bool COLS> bool rows_of_pieces(const KnProduct &p, const Beside &beside)
{
    constexpr int64_t W = 16 / sizeof(T);
    return (((uintptr_t)p.a | (uintptr_t)p.b | (uintptr_t)beside.b) & 15) == 0 && p.C % W == 0 && p.lda % W == 0 && (COLS ? p.J % W == 0 : beside.rank % W == 0);
}
// Layers of up to 128 x 128 and a rank of up to 16: by a wavefront per 32 rows (small), or the two kernels (us, small / tiles; rank 8, columns contiguous):
//   rows, networks         262,144, 4,096   262,144, 64   20,000, 4,096   2,000, 500
//   fp32   64 x 64               84/96          64/83          31/21          9/11
//          128 x 64             133/130        101/122         49/27         13/13
//          64 x 128             157/116        117/108         52/34         12/11
//          128 x 128            238/167        187/153         86/43         18/13
//   fp16   64 x 64               30/50          25/47          13/14          6/9
//          128 x 64              47/62          35/56          18/16          7/9
//          64 x 128              53/48          40/44          19/17          6/9
//          128 x 128             93/65          63/56          29/18          7/9
// and 262,145 rows of 1,600 networks 91 x 64 in bf16, which are not whole pieces, 41/78.
template <typename T> bool small_layer(const KnProduct &p, const Down &down, bool pieces)
{
    if (p.C > SMALL_MOST || p.J > SMALL_MOST || down.rp > 16) return false;
    if (!pieces) return true;
    if (p.M <= 8192) return sizeof(T) == 2 || p.J <= 64;
    return p.J <= 64 && p.M / down.E >= 16 && (sizeof(T) == 2 || p.C <= 64);
}

// Which tiles: the largest of which there are enough for the chip.  Measured (us, both kernels; 16 networks, rank 16, 2048 x 2048, columns contiguous, bf16):
//   rows                          100    256    512    1,024   2,048   4,096
//   32 x 64, four stages         19.7   20.5   26.0    41.1    71.9     144
//   64 x 64, four stages         21.6   22.1   24.4    28.6    48.0      86
//   64 x 128, three stages       25.7   25.9   27.2    28.1    35.0      57
//   128 x 128, two               33.6   33.6   35.0    34.8    36.3      48
// rows that are not whole pieces (1023 x 1025, 256, 1,024 and 4,096 rows): 32 x 64 29, 38, 67; 128 x 128 39, 38, 59.  fp32 (1024 x 1024): 32 x 64 28, 38, 107; 64 x 64 38,
// 40, 98; 64 x 128 61, 60, 92; 128 x 128 98, 93, 97.
template <typename T, bool COLS> int launch_up(hipStream_t st, const KnProduct &p, const Beside &beside)
{
    auto tiles = [&](int64_t bm) { return (p.M + bm - 1) / bm * ((p.J + 127) / 128); };
    const bool direct = rows_of_pieces<T, COLS>(p, beside);
    const bool narrow = p.J <= 64 || tiles(64) < 256;
    if constexpr (sizeof(T) == 4) {
        if (!direct) return narrow ? launch_tiles<T, COLS, false, 32, 64, 1, 4, 2>(st, p, beside) : launch_tiles<T, COLS, false, 64, 128, 1, 4, 2>(st, p, beside);
        return narrow ? launch_tiles<T, COLS, true, 32, 64, 1, 4, 4>(st, p, beside) : launch_tiles<T, COLS, true, 64, 128, 1, 4, 2>(st, p, beside);
    } else {
        if (!direct) return narrow ? launch_tiles<T, COLS, false, 32, 64, 1, 4, 2>(st, p, beside) : launch_tiles<T, COLS, false, 128, 128, 2, 4, 2>(st, p, beside);
        if (p.J > 64 && tiles(128) >= 384) return launch_tiles<T, COLS, true, 128, 128, 2, 4, 2>(st, p, beside);
        if (p.J > 64 && tiles(64) >= 256) return launch_tiles<T, COLS, true, 64, 128, 1, 4, 3>(st, p, beside);
        if (kn_div_up(p.M, 64) * kn_div_up(p.J, 64) >= 256) return launch_tiles<T, COLS, true, 64, 64, 2, 2, 4>(st, p, beside);
        return launch_tiles<T, COLS, true, 32, 64, 1, 4, 4>(st, p, beside);
    }
}

// How few rows' product is cut: up to 16 rows by 16 columns, more by 32, and the contraction until there are 128 workgroups, in no part of less than a step per
// wavefront.  Measured (us; one row 2048 x 2048, 48 rows 2048 x 2560 with 32 networks, bf16, both launches): 16 columns, 128 workgroups 9.1, 16.2; 32
// columns, 128 10.0, 14.2; 32, 256 12.4, 15.9; 32, 512 15.1, 20.5; 64, 128 11.2, 14.8.
int few_columns(int64_t M) { return M <= 16 ? 16 : 32; }
Few few_of(int64_t M, int32_t J, int32_t C, int item)
{
    Few f = {};
    const int64_t tiles = kn_div_up(J, few_columns(M)), steps = kn_div_up(C, 64 / item);
    int64_t parts = kn_div_up(128, tiles);
    if (parts > kn_div_up(steps, 8)) parts = kn_div_up(steps, 8);
    f.each = (int32_t)kn_div_up(steps, parts);
    f.parts = (int32_t)kn_div_up(steps, f.each);
    f.products = (int32_t)(tiles * f.parts);
    return f;
}
int64_t few_bytes(int64_t M, int32_t J, int32_t C, int item) { return M > FEW_ROWS ? 0 : kn_align_up(few_of(M, J, C, item).parts * M * J * 4, 256); }

template <typename T, int B, int U, int DOWN_V> int launch_few_of(hipStream_t st, const Down &down, const KnProduct &p, const Few &few)
{
    const int64_t blocks = few.products + kn_pieces(down.M, down.E, 16) * kn_div_up(down.rp, 16 * DOWN_V);
    hipLaunchKernelGGL((k_adapt_few<T, B, U, U == 1 ? 1 : 2, DOWN_V>), dim3((unsigned)blocks), dim3(512), 0, st, p, down, few);
    KN_CHECK_LAUNCH();
    return KN_OK;
}
template <typename T, int B, int U> int launch_few_rank(hipStream_t st, const Down &down, const KnProduct &p, const Few &few)
{
    return down.rp <= 16 ? launch_few_of<T, B, U, 1>(st, down, p, few) : launch_few_of<T, B, U, 2>(st, down, p, few);
}
template <typename T, int B> int launch_few_rows(hipStream_t st, const Down &down, const KnProduct &p, const Few &few)
{
    if (p.M <= 16) return launch_few_rank<T, B, 1>(st, down, p, few);
    return p.M <= 32 ? launch_few_rank<T, B, 2>(st, down, p, few) : launch_few_rank<T, B, 4>(st, down, p, few);
}
template <typename T> int launch_few_b(hipStream_t st, const Down &down, const KnProduct &p, const Few &few, bool cols)
{
    if (!cols) return launch_few_rows<T, B_ROWS>(st, down, p, few);
    if constexpr (sizeof(T) == 2) {
        if (p.J % 8 == 0 && down.rank % 8 == 0 && p.C >= 8 && (((uintptr_t)p.b | (uintptr_t)down.b) & 15) == 0) return launch_few_rows<T, B_PIECES>(st, down, p, few);
    }
    return launch_few_rows<T, B_COLS>(st, down, p, few);
}
template <typename T> int launch_few(hipStream_t st, const Down &down, const KnProduct &p, const Beside &beside, bool cols, float *sums)
{
    Few few = few_of(p.M, p.J, p.C, sizeof(T));
    few.sums = sums;
    KN_TRY(launch_few_b<T>(st, down, p, few, cols));
    const dim3 grid((unsigned)kn_div_up((int64_t)p.M * kn_div_up(p.J, 4), 128));
    if (sizeof(T) == 2 && beside.wide) hipLaunchKernelGGL((k_adapt_few_join<T, float>), grid, dim3(128), 0, st, p, beside, few);
    else hipLaunchKernelGGL((k_adapt_few_join<T, T>), grid, dim3(128), 0, st, p, beside, few);
    KN_CHECK_LAUNCH();
    return KN_OK;
}

// Both products of a call on `a` (rows through `rows`): h = scale a b_e, out = a w + h c_e.  cols: the columns of b and w are contiguous, and c's; else their contractions
// are.  sums: room for few rows' parts.
// padded: room for the factor c in rows of whole pieces (padded_bytes), or nullptr
int run(hipStream_t st, int32_t dtype, bool cols, const Down &down, const KnProduct &up, const Beside &beside, float *sums, void *padded)
{
    return kn_with_type(dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        // (very many networks of a very large rank: the other way's launches are cut)
        if (up.M <= FEW_ROWS && down.E * (int64_t)down.rp <= 1 << 24) return launch_few<E_>(st, down, up, beside, cols, sums);
        if (small_layer<E_>(up, down, cols ? rows_of_pieces<E_, true>(up, beside) : rows_of_pieces<E_, false>(up, beside)))
            return cols ? launch_small<E_, true>(st, down, up, beside) : launch_small<E_, false>(st, down, up, beside);
        KN_TRY(launch_down<E_>(st, down, cols));
        if (padded && !cols) {
            Beside whole = beside;
            whole.b = padded;
            whole.rank = whole.b_j = beside.rp;
            whole.b_group = (int64_t)up.J * beside.rp;
            if (rows_of_pieces<E_, false>(up, whole)) {
                const int64_t blocks = kn_div_up((int64_t)up.J * beside.rp * (int64_t)sizeof(E_), 256 * 16);
                KN_TRY(kn_launch(blocks * down.E, 256, [&](dim3 grid, int32_t first) {
                    hipLaunchKernelGGL((k_adapt_pad<E_>), grid, dim3(256), 0, st, (const E_ *)beside.b, (E_ *)padded, down.offsets, up.M, up.J, beside.rank, beside.rp, (int32_t)blocks, first);
                }));
                return launch_up<E_, false>(st, up, whole);
            }
        }
        return cols && up.b_c != 1 ? launch_up<E_, true>(st, up, beside) : launch_up<E_, false>(st, up, beside);
    });
}

int32_t padded_rank(int32_t dtype, int32_t rank) { return (int32_t)kn_align_up(rank, 16 / kn_item(dtype)); }
int check(const kn_linear_desc *d, int32_t rank)
{
    KN_TRY(kn_linear_check(d));
    if (rank < 1) return KN_E_INVALID_ARG;
    return rank > KN_MAX_WIDTH ? KN_E_UNSUPPORTED : KN_OK;
}
// networks of the rows, and which networks are left out
int64_t net_bytes(const kn_linear_desc *d) { return kn_align_up(d->rows * 4, 256) + kn_align_up(d->experts * 4, 256); }
int32_t *apart_of(const kn_linear_desc *d, void *workspace) { return (int32_t *)((char *)workspace + kn_align_up(d->rows * 4, 256)); }
int64_t h_bytes(const kn_linear_desc *d, int32_t rank) { return kn_align_up(d->rows * (int64_t)padded_rank(d->dtype, rank) * kn_item(d->dtype), 256); }
// Room for the g of few rows in 32 bits
int64_t wide_bytes(const kn_linear_desc *d, int32_t rank)
{
    return d->rows > FEW_ROWS || d->dtype == KN_F32 ? 0 : kn_align_up(d->rows * (int64_t)padded_rank(d->dtype, rank) * 4, 256);
}
// Room for a factor of J rows of `rank` in rows of whole pieces, where its rows are contiguous and not that already (not beyond 256 MiB: then as they are)
int64_t padded_bytes(const kn_linear_desc *d, int32_t rank, bool cols, int32_t J)
{
    const int32_t rp = padded_rank(d->dtype, rank);
    const int64_t bytes = kn_align_up((int64_t)d->experts * J * rp * kn_item(d->dtype), 256);
    return cols || rp == rank || d->rows <= FEW_ROWS || bytes > 1 << 28 ? 0 : bytes;
}
// The gradients of A and B as those of a grouped layer
kn_linear_desc layer_of(const kn_linear_desc *d, int32_t n_in, int32_t n_out, int64_t x_rows, int64_t ldx)
{
    kn_linear_desc l = *d;
    l.n_in = n_in; l.n_out = n_out; l.x_rows = x_rows; l.ldx = ldx;
    return l;
}
int dw_bytes(const kn_linear_desc *d, int32_t rank, int64_t *out)
{
    const kn_linear_desc a = layer_of(d, d->n_in, rank, d->x_rows, d->ldx), b = layer_of(d, rank, d->n_out, d->rows, padded_rank(d->dtype, rank));
    int64_t na = 0, nb = 0;
    KN_TRY(kn_linear_dw_bytes(&a, true, &na));
    KN_TRY(kn_linear_dw_bytes(&b, true, &nb));
    const int64_t few = few_bytes(d->rows, d->n_in, d->n_out, kn_item(d->dtype)) + wide_bytes(d, rank); // (done with before the others begin)
    *out = na + nb;
    *out = few > *out ? few : *out;
    const int64_t padded = padded_bytes(d, rank, d->w_layout == KN_W_OUT_IN, d->n_in);
    *out = padded > *out ? padded : *out;
    return KN_OK;
}
bool bad_workspace(const void *ws, int64_t have, int64_t need) { return need > 0 && (!ws || ((uintptr_t)ws & 255) || have < need); }

} // namespace

extern "C" int kn_adapted_linear_workspace_bytes(const kn_linear_desc *d, int32_t rank, int64_t *out_bytes)
{
    KN_TRY(check(d, rank));
    if (!out_bytes) return KN_E_INVALID_ARG;
    *out_bytes = net_bytes(d) + h_bytes(d, rank) + few_bytes(d->rows, d->n_out, d->n_in, kn_item(d->dtype)) + padded_bytes(d, rank, d->w_layout == KN_W_IN_OUT, d->n_out);
    return KN_OK;
}

extern "C" int kn_adapted_linear(void *stream, const kn_linear_desc *d, int32_t rank, const void *x, const void *w, const void *a, const void *b,
                                 const float *scales, const void *bias, const int32_t *offsets, const int32_t *rows, int32_t relu, void *y, void *h,
                                 void *workspace, int64_t workspace_bytes)
{
    KN_TRY(check(d, rank));
    if (d->rows == 0) return KN_OK;
    if (!w || !a || !b || !offsets || !y || (d->x_rows > 0 && !x) || (!rows && d->x_rows < d->rows) || ((uintptr_t)h & 15)) return KN_E_INVALID_ARG;
    int64_t need = 0;
    KN_TRY(kn_adapted_linear_workspace_bytes(d, rank, &need));
    if (bad_workspace(workspace, workspace_bytes, need)) return KN_E_WORKSPACE;
    const bool io = d->w_layout == KN_W_IN_OUT;
    const int64_t K = d->n_in, N = d->n_out, R = rank;
    Down down = {x, a, scales, h ? h : (char *)workspace + net_bytes(d), (int32_t *)workspace, offsets, rows, d->ldx, K * R, io ? R : 1, io ? 1 : K,
                 (int32_t)d->rows, d->experts, d->n_in, rank, padded_rank(d->dtype, rank), (int32_t)d->x_rows, 0, b, R * N, apart_of(d, workspace), nullptr};
    Beside beside = {down.h, b, down.net, down.apart, nullptr, R * N, io ? N : 1, io ? 1 : R, d->experts, rank, down.rp};
    KnProduct p = {};
    p.a = x; p.b = w; p.bias = bias; p.out = y; p.rows = rows;
    p.lda = d->ldx; p.b_c = io ? N : 1; p.b_j = io ? 1 : K; p.o_i = N;
    p.M = down.M; p.J = d->n_out; p.C = d->n_in; p.a_rows = down.a_rows; p.relu = relu != 0;
    char *more = (char *)workspace + net_bytes(d) + h_bytes(d, rank); // (few rows' sums, or a padded factor)
    return run((hipStream_t)stream, d->dtype, io, down, p, beside, (float *)more, padded_bytes(d, rank, io, d->n_out) > 0 ? more : nullptr);
}

extern "C" int kn_adapted_linear_backward_workspace_bytes(const kn_linear_desc *d, int32_t rank, int64_t *out_bytes)
{
    KN_TRY(check(d, rank));
    if (!out_bytes) return KN_E_INVALID_ARG;
    int64_t dw = 0;
    KN_TRY(dw_bytes(d, rank, &dw));
    *out_bytes = net_bytes(d) + h_bytes(d, rank) + dw;
    return KN_OK;
}

extern "C" int kn_adapted_linear_backward(void *stream, const kn_linear_desc *d, int32_t rank, const void *dy, const void *x, const void *h, const void *w,
                                          const void *a, const void *b, const float *scales, const int32_t *offsets, const int32_t *rows, int32_t relu_in,
                                          void *dx, void *da, void *db, void *workspace, int64_t workspace_bytes)
{
    KN_TRY(check(d, rank));
    if (!offsets || !da || !db ||
        (d->rows > 0 && (!dy || !h || !w || !a || !b || !dx || (d->x_rows > 0 && !x) || (!rows && d->x_rows < d->rows) || ((uintptr_t)h & 15))))
        return KN_E_INVALID_ARG;
    int64_t dw = 0;
    KN_TRY(dw_bytes(d, rank, &dw));
    if (bad_workspace(workspace, workspace_bytes, net_bytes(d) + h_bytes(d, rank) + dw)) return KN_E_WORKSPACE;
    const bool io = d->w_layout == KN_W_IN_OUT;
    const int64_t K = d->n_in, N = d->n_out, R = rank;
    char *g = (char *)workspace + net_bytes(d), *sums = g + h_bytes(d, rank);
    const int32_t rp = padded_rank(d->dtype, rank);
    if (d->rows > 0) {
        float *wide = wide_bytes(d, rank) > 0 ? (float *)(sums + few_bytes(d->rows, d->n_in, d->n_out, kn_item(d->dtype))) : nullptr;
        Down down = {dy, b, scales, g, (int32_t *)workspace, offsets, nullptr, N, R * N, io ? 1 : R, io ? N : 1,
                     (int32_t)d->rows, d->experts, d->n_out, rank, rp, (int32_t)d->rows, 0, a, K * R, apart_of(d, workspace), wide};
        Beside beside = {g, a, down.net, down.apart, wide, K * R, io ? 1 : K, io ? R : 1, d->experts, rank, rp};
        KnProduct p = {};
        p.a = dy; p.b = w; p.mask = relu_in ? (x ? x : w) : nullptr; p.out = dx; // (an x without rows may have no address)
        p.lda = N; p.ldm = d->ldx; p.b_c = io ? 1 : K; p.b_j = io ? N : 1; p.o_i = K;
        p.M = down.M; p.J = d->n_in; p.C = d->n_out; p.a_rows = p.M; p.m_rows = (int32_t)d->x_rows;
        p.mask_rows = relu_in ? rows : nullptr;
        KN_TRY(run((hipStream_t)stream, d->dtype, !io, down, p, beside, (float *)sums, padded_bytes(d, rank, !io, d->n_in) > 0 ? sums : nullptr));
    }
    const kn_linear_desc la = layer_of(d, d->n_in, rank, d->x_rows, d->ldx), lb = layer_of(d, rank, d->n_out, d->rows, rp);
    return kn_linear_dw_low_rank(stream, &la, x, g, rp, rows, da, &lb, h, dy, N, db, offsets, sums, dw);
}
