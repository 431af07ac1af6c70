// Gradients of the weights and biases of a layer of all networks: kn_grouped_linear_dw.
#include "kn_tile.h"

namespace {

// A network's rows are cut into parts of at most `len`: a network of one part has its sums written at once, of several, each
// part's go to the workspace in fp32 and k_reduce_join adds them in order, so that the result does not depend on who was first.  Part c
// of a network whose rows begin at o has place 2 (o / len) + c: a network of several parts has more than len rows, so these
// places do not meet, and there are at most 2 (M / len) + 2.
struct Parts {
    int32_t len;
    float *sums, *bias_sums; // (places, I, J) and (places, columns of dy)
};
__host__ __device__ inline int64_t part_places(int64_t M, int64_t len) { return 2 * (M / len) + 2; }

// Tiles of BM x BN of a network's out(i, j) = sum over rows r of a(r, i) b(r, j): both operands column-wise, the contraction is the
// rows, 128 bytes' worth a stage.  The columns' sums (gradient of the biases) are products with ones of the fragments that are
// there anyway, in the workgroups of the first tile: SUM_B the columns of b, SUM_A those of a.
// Measured: 32,768 rows through an index, 32 networks 1024 x 2048 in bf16: 231 us, 595 TFLOP/s.  The transposing read brings 8 bytes a
// lane, so that fragments cost twice the reads of the forward product's, and the LDS bounds it (128 x 128 by four wavefronts of 64 x
// 64: 230 against 219 on even networks; 256 x 128: 230; 128 x 256: 246).  64 x 64 tiles: 524,291 rows, 4,096 networks 64 x 64 in fp16: 34
// us, 4.9 TB/s (47 with 128 x 128).
// SAVED: a, or b, is what kn_save_f8 left of x (its exponents beside it), and goes through registers: the 32,768 rows 250 us, 524,291 rows 64 x 64 in fp16 33.  Of small layers, too,
// whose x as it was would be k_reduce_small's: widths far below a tile's cost what the tile does.
enum { SUM_NONE, SUM_A, SUM_B };
enum { SAVED_NONE, SAVED_A, SAVED_B };
template <typename T, bool DIRECT, int BM, int BN, int WR, int WC, int SAVED = SAVED_NONE>
__global__ void __launch_bounds__(WR * WC * 64) k_product_reduce(KnProduct p, int32_t sum, Parts parts, const uint8_t *exponents)
{
    constexpr int NW = WR * WC, STAGE = (BM + BN) * 128, U = BM / WR / 16, V = BN / WC / 16, CS = 128 / sizeof(T);
    typedef typename KnFrag<T>::Type Frag;
    __shared__ __align__(16) char lds_[2 * STAGE];
    KN_LDS char *lds = (KN_LDS char *)lds_;
    const int tid = kn_thread(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int jtiles = (p.J + BN - 1) / BN, itiles = (p.I + BM - 1) / BM;
    // (a part's tiles go to all XCDs, neighbours among them to one: networks differ in rows, XCDs should not)
    const int32_t tiles = itiles * jtiles, block = p.first + kn_block(), number = kn_xcd_order(block % tiles, tiles);
    const int32_t part = block / tiles;
    const KnPiece piece = kn_find_piece(p.offsets, p.E, p.M, parts.len, part);
    const int32_t group = piece.group;
    if (group >= p.E) return;
    const int32_t o = kn_offset(p.offsets, group, p.M), c0 = piece.begin, cend = max(c0, min(piece.end, c0 + parts.len));
    if (c0 >= cend && c0 != o) return; // (the first part of a network without rows writes zeros)
    const bool several = piece.end - o > parts.len;
    const int64_t place = 2 * (o / parts.len) + (c0 - o) / parts.len;
    const int j0 = number % jtiles * BN, i0 = number / jtiles * BM;
    const int32_t steps = (cend - c0 + CS - 1) / CS;
    const bool sum_a = sum == SUM_A && j0 == 0, sum_b = sum == SUM_B && i0 == 0;
    typename std::conditional<SAVED == SAVED_A, KnSavedLoader<T, BM, NW>, KnGroupLoader<T, BM, NW, DIRECT>>::type la;
    typename std::conditional<SAVED == SAVED_B, KnSavedLoader<T, BN, NW>, KnGroupLoader<T, BN, NW, DIRECT>>::type lb;
    const int wi = (wave / WC) * (BM / WR), wj = (wave % WC) * (BN / WC);
    kn_f32x4 acc[U][V] = {}, side[U > V ? U : V] = {};
    Frag ones;
#pragma unroll
    for (int q = 0; q < (int)(sizeof(Frag) / sizeof(T)); ++q) ones[q] = (T)1.0f;
    Frag fa[2][U], fb[2][V];
    auto fetch = [&](int s) {
        KN_LDS char *tile = lds + (s & 1) * STAGE;
        la.fetch(tile, wave, lane, c0 + s * CS);
        lb.fetch(tile + BM * 128, wave, lane, c0 + s * CS);
    };
    auto read = [&](int s, int kk) {
        const KN_LDS char *ta = lds + (s & 1) * STAGE, *tb = ta + BM * 128;
#pragma unroll
        for (int u = 0; u < U; ++u) fa[kk][u] = kn_col_frag<T, BM>(ta, wi + 16 * u, kk, lane);
#pragma unroll
        for (int v = 0; v < V; ++v) fb[kk][v] = kn_col_frag<T, BN>(tb, wj + 16 * v, kk, lane);
    };
    auto multiply = [&](int kk) {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int v = 0; v < V; ++v) acc[u][v] = kn_mfma(fb[kk][v], fa[kk][u], acc[u][v]);
    };
    auto add_up = [&](int kk) {
        if (sum_a && wj == 0) {
#pragma unroll
            for (int u = 0; u < U; ++u) side[u] = kn_mfma(ones, fa[kk][u], side[u]);
        }
        if (sum_b && wi == 0) {
#pragma unroll
            for (int v = 0; v < V; ++v) side[v] = kn_mfma(fb[kk][v], ones, side[v]);
        }
    };
    if (steps > 0) {
        if constexpr (SAVED == SAVED_A) la.start(wave, lane, (const uint8_t *)p.a, exponents, i0, p.I, p.rows, p.a_rows, c0, cend);
        else la.start(wave, lane, (const T *)p.a + i0, p.lda, p.I - i0, p.rows, p.a_rows, c0, cend);
        if constexpr (SAVED == SAVED_B) lb.start(wave, lane, (const uint8_t *)p.b, exponents, j0, p.J, p.b_index, p.b_rows, c0, cend);
        else lb.start(wave, lane, (const T *)p.b + j0, p.ldb, p.J - j0, p.b_index, p.b_rows, c0, cend);
        fetch(0);
        if (!DIRECT && steps > 1) fetch(1);
        kn_stage_barrier();
        if (DIRECT && steps > 1) fetch(1);
        read(0, 0);
        for (int s = 0; s < steps; ++s) {
            add_up(0);
            read(s, 1);
            multiply(0);
            kn_interleave<U, V, T, true, true>();
            kn_stage_barrier<DIRECT ? 0 : 63>(); // (loads into registers are waited for where they are put down)
            if (s + 2 < steps) fetch(s + 2);
            add_up(1);
            read(s + 1, 0); // (behind the last stage: what happens to lie there, unused)
            multiply(1);
            kn_interleave<U, V, T, true, true>();
        }
    }
    kn_stage_barrier(); // (the tiles' LDS is used again)
    auto put_bias = [&](int j, int n, float v) {
        if (j >= n) return;
        if (several) parts.bias_sums[place * n + j] = v;
        else ((T *)p.out_bias)[(int64_t)group * n + j] = (T)v;
    };
    if (sum_a && wj == 0 && lane < 16) { // (each column of the product is alike: its 16 rows are the sums of 16 columns of a)
#pragma unroll
        for (int u = 0; u < U; ++u) put_bias(i0 + wi + 16 * u + lane, p.I, side[u][0]);
    }
    if (sum_b && wi == 0 && (lane & 15) == 0) {
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int r = 0; r < 4; ++r) put_bias(j0 + wj + 16 * v + (lane >> 4) * 4 + r, p.J, side[v][r]);
    }
    constexpr int WN = BN / WC, LD = WN + 4, LR = WN / 8;
    static_assert(64 % LR == 0, "");
    KN_LDS float *mine = (KN_LDS float *)(lds + wave * (16 * LD * 4));
    const int cj = lane % LR * 8;
    const int32_t j = j0 + wj + cj;
    float *sums = parts.sums + place * p.I * p.J;
    T *out = (T *)p.out + (int64_t)group * p.o_group;
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int v = 0; v < V; ++v) *(KN_LDS kn_f32x4 *)(mine + (lane & 15) * LD + 16 * v + (lane >> 4) * 4) = acc[u][v];
        kn_lanes_meet();
#pragma unroll
        for (int h = 0; h < (16 * LR + 63) / 64; ++h) {
            const int r = h * (64 / LR) + lane / LR;
            const int32_t i = i0 + wi + 16 * u + r;
            if (r >= 16 || i >= p.I || j >= p.J) continue;
            const kn_f32x4 lo = *(const KN_LDS kn_f32x4 *)(mine + r * LD + cj), hi = *(const KN_LDS kn_f32x4 *)(mine + r * LD + cj + 4);
            if (several) {
                KnEight<float>::store(sums + (int64_t)i * p.J, j, p.J, typename KnEight<float>::Piece{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
            } else {
                const typename KnEight<T>::Piece v = {(T)lo[0], (T)lo[1], (T)lo[2], (T)lo[3], (T)hi[0], (T)hi[1], (T)hi[2], (T)hi[3]};
                KnEight<T>::store(out + (int64_t)i * p.o_i, j, p.J, v);
            }
        }
        kn_lanes_meet();
    }
}

// Layers of the small networks' kind whose rows are not whole pieces: a workgroup of WAVES wavefronts per part, 16 U x 16 V results at
// most; a wavefront takes every WAVES-th step of rows, straight into fragments, value by value (16 neighbouring lanes, 16 neighbouring
// values), and they are summed in the order of their numbers.  Nothing is staged and nothing waits until then: a part of a few
// hundred rows is one chain of look-up, index, values, and the chains in flight are what counts.  Measured: 684,936 rows of 126 bytes
// through an index, 4,096 networks 63 x 3 in bf16: 75 us (103 with tiles staged in the LDS).  Where networks have fewer rows than a step
// on average, or a few steps' and are enough to fill the chip, WAVES is 1: 27,000 rows of 4,096 networks 63 x 33 in fp16: 25 us, with
// four wavefronts 43; 262,145 rows of 32 x 33 in bf16 (with the join) 30 and 41, 524,291 rows of 63 x 32: 57 and 57.
template <typename T, int U, int V, int WAVES>
__global__ void __launch_bounds__(WAVES * 64) k_reduce_small(KnProduct p, int32_t sum, Parts parts)
{
    constexpr int W = 16 / sizeof(T), RS = 4 * W, BM = 16 * U, BN = 16 * V, LD = BN + 4;
    typedef typename KnFrag<T>::Type Frag;
    __shared__ __align__(16) float red[BM * LD];
    __shared__ float side_a[BM], side_b[BN];
    const int tid = kn_thread(), lane = tid & 63, col = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const KnPiece piece = kn_find_piece(p.offsets, p.E, p.M, parts.len, p.first + kn_block());
    const int32_t group = piece.group;
    if (group >= p.E) return;
    const int32_t o = kn_offset(p.offsets, group, p.M), c0 = piece.begin, cend = max(c0, min(piece.end, c0 + parts.len));
    if (c0 >= cend && c0 != o) return; // (the first part of a network without rows writes zeros)
    const bool several = piece.end - o > parts.len;
    const int64_t place = 2 * (o / parts.len) + (c0 - o) / parts.len;
    const bool sum_a = sum == SUM_A, sum_b = sum == SUM_B;
    int32_t ai[U], bj[V];
#pragma unroll
    for (int u = 0; u < U; ++u) ai[u] = min(16 * u + col, p.I - 1);
#pragma unroll
    for (int v = 0; v < V; ++v) bj[v] = min(16 * v + col, p.J - 1);
    kn_f32x4 acc[U][V] = {}, sa[U] = {}, sb[V] = {};
    Frag ones;
#pragma unroll
    for (int q = 0; q < W; ++q) ones[q] = (T)1.0f;
    for (int32_t c = c0 + wave * RS; c < cend; c += WAVES * RS) {
        Frag fa[U], fb[V];
#pragma unroll
        for (int q = 0; q < W; ++q) { // (rows behind the part, and rows that a matrix does not have: zeros)
            const int32_t r = min(c + g * W + q, cend - 1), ra = p.rows ? p.rows[r] : r, rb = p.b_index ? p.b_index[r] : r;
            const bool in = c + g * W + q < cend, in_a = in && (uint32_t)ra < (uint32_t)p.a_rows, in_b = in && (uint32_t)rb < (uint32_t)p.b_rows;
            const T *a = (const T *)p.a + (int64_t)(in_a ? ra : 0) * p.lda, *b = (const T *)p.b + (int64_t)(in_b ? rb : 0) * p.ldb;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const T x = p.a_rows > 0 ? a[ai[u]] : (T)0.0f;
                fa[u][q] = in_a ? x : (T)0.0f;
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const T x = p.b_rows > 0 ? b[bj[v]] : (T)0.0f;
                fb[v][q] = in_b ? x : (T)0.0f;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int v = 0; v < V; ++v) acc[u][v] = kn_mfma(fb[v], fa[u], acc[u][v]);
        if (sum_a)
#pragma unroll
            for (int u = 0; u < U; ++u) sa[u] = kn_mfma(ones, fa[u], sa[u]);
        if (sum_b)
#pragma unroll
            for (int v = 0; v < V; ++v) sb[v] = kn_mfma(fb[v], ones, sb[v]);
    }
    const int busy = max(1, min(WAVES, (cend - c0 + RS - 1) / RS));
    for (int w = 0; w < busy; ++w) { // (a lane's four results are neighbours in a row)
        if (wave == w) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    kn_f32x4 *at = (kn_f32x4 *)(red + (16 * u + col) * LD + 16 * v + 4 * g);
                    *at = w ? *at + acc[u][v] : acc[u][v];
                }
                if (sum_a && g == 0) side_a[16 * u + col] = w ? side_a[16 * u + col] + sa[u][0] : sa[u][0];
            }
            if (sum_b && col == 0)
#pragma unroll
                for (int v = 0; v < V; ++v)
#pragma unroll
                    for (int r = 0; r < 4; ++r) side_b[16 * v + 4 * g + r] = w ? side_b[16 * v + 4 * g + r] + sb[v][r] : sb[v][r];
        }
        __syncthreads();
    }
    float *sums = parts.sums + place * p.I * p.J;
    T *out = (T *)p.out + (int64_t)group * p.o_group; // (its rows follow one another)
    for (int q = tid; q < p.I * p.J; q += WAVES * 64) {
        const float y = red[q / p.J * LD + q % p.J];
        if (several) sums[q] = y;
        else out[q] = (T)y;
    }
    const int n = sum_a ? p.I : sum_b ? p.J : 0;
    if (tid < n) {
        const float y = sum_a ? side_a[tid] : side_b[tid];
        if (several) parts.bias_sums[place * n + tid] = y;
        else ((T *)p.out_bias)[(int64_t)group * n + tid] = (T)y;
    }
}

// One side of up to 64 values (a low-rank product's), the other long: a workgroup of WAVES wavefronts per part and tile of 16 FI x 16 FJ results; a wavefront
// takes every WAVES-th step of rows by itself, asked for while another is multiplied, and they are summed in the order of their numbers.  TURN: 16-bit rows
// in pieces, wherever they lie, which an LDS of the wavefront's own turns into columns; else (fp32, and rows of less than a piece) value by value, 16 neighbouring
// lanes, 16 neighbouring values.  Bound by the long side's bytes.  Rows that are not whole pieces, 20,000 of 100 networks 515 x 300, rank 10 in bf16: 20 us, value by value 45.
// (In fp32 nothing but value by value has been measured.)
constexpr int thin_bytes(int fi, int fj) { return 16 * fi * (16 * fj + 4) * 4 > (fi + fj) * 1024 ? 16 * fi * (16 * fj + 4) * 4 : (fi + fj) * 1024; } // of a wavefront
template <typename T, int FI, int FJ, bool TURN, int WAVES>
__device__ __forceinline__ void reduce_thin(const KnProduct &p, const Parts &parts, int32_t width_a, int32_t width_b, int32_t block, char *lds_)
{
    constexpr int W = 16 / sizeof(T), RS = 4 * W, LD = 16 * FJ + 4, OWN = thin_bytes(FI, FJ);
    typedef typename KnFrag<T>::Type Frag;
    const int tid = kn_thread(), lane = tid & 63, col = lane & 15, g = lane >> 4, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    KN_LDS char *own = (KN_LDS char *)lds_ + wave * OWN;
    const int jtiles = (p.J + 16 * FJ - 1) / (16 * FJ), itiles = (p.I + 16 * FI - 1) / (16 * FI), tiles = itiles * jtiles;
    const int32_t number = block % tiles;
    const KnPiece piece = kn_find_piece(p.offsets, p.E, p.M, parts.len, block / tiles);
    const int32_t group = piece.group;
    if (group >= p.E) return;
    const int32_t o = kn_offset(p.offsets, group, p.M), c0 = piece.begin, cend = max(c0, min(piece.end, c0 + parts.len));
    if (c0 >= cend && c0 != o) return; // (the first part of a network without rows writes zeros)
    const bool several = piece.end - o > parts.len;
    const int64_t place = 2 * (o / parts.len) + (c0 - o) / parts.len;
    const int j0 = number % jtiles * 16 * FJ, i0 = number / jtiles * 16 * FI;
    kn_f32x4 acc[FI][FJ] = {};
    // F fragments' worth of a step's rows of one side
    auto ask = [&](auto count, const T *at, int64_t ld, const int32_t *index, int32_t rows, int32_t width, int32_t c, Frag *to, uint32_t &none) {
        constexpr int F = decltype(count)::value;
        none = 0; // a bit for each fragment (TURN) or value of a fragment: rows that are not there
#pragma unroll
        for (int f = 0; f < (TURN ? F : W); ++f) {
            const int32_t r = c + (TURN ? (lane + 64 * f) / (2 * F) : g * W + f);
            const int32_t src = index ? index[min(r, cend - 1)] : min(r, cend - 1);
            const bool there = r < cend && (uint32_t)src < (uint32_t)rows;
            none |= there ? 0u : 1u << f;
            const T *row = at + (int64_t)(there ? src : 0) * ld;
            if constexpr (TURN) to[f] = *(const typename KnAny<T>::Piece *)(row + min((lane + 64 * f) % (2 * F) * W, width - W));
            else
#pragma unroll
                for (int v = 0; v < F; ++v) to[v][f] = row[min(16 * v + col, width - 1)];
        }
    };
    auto turn = [&](auto count, Frag *to, uint32_t none, KN_LDS char *lds) {
        constexpr int F = decltype(count)::value;
        if constexpr (TURN) {
#pragma unroll
            for (int f = 0; f < F; ++f) *(KN_LDS Frag *)(lds + kn_turned_byte<F>((lane + 64 * f) / (2 * F), (lane + 64 * f) % (2 * F))) = none >> f & 1 ? Frag{} : to[f];
        } else {
#pragma unroll
            for (int v = 0; v < F; ++v)
#pragma unroll
                for (int f = 0; f < W; ++f) to[v][f] = none >> f & 1 ? (T)0.0f : to[v][f];
        }
    };
    struct Step { Frag a[FI], b[FJ]; uint32_t none_a, none_b; };
    std::integral_constant<int, FI> fi;
    std::integral_constant<int, FJ> fj;
    auto load = [&](Step &x, int32_t c) {
        ask(fi, (const T *)p.a + i0, p.lda, p.rows, p.a_rows, width_a - i0, c, x.a, x.none_a);
        ask(fj, (const T *)p.b + j0, p.ldb, p.b_index, p.b_rows, width_b - j0, c, x.b, x.none_b);
    };
    auto multiply = [&](Step &x, int32_t c) {
        if (c >= cend) return;
        turn(fi, x.a, x.none_a, own);
        turn(fj, x.b, x.none_b, own + FI * 1024);
        if constexpr (TURN) {
            kn_lanes_meet();
#pragma unroll
            for (int u = 0; u < FI; ++u) x.a[u] = __builtin_bit_cast(Frag, kn_turned_frag<FI>(own, u, lane));
#pragma unroll
            for (int v = 0; v < FJ; ++v) x.b[v] = __builtin_bit_cast(Frag, kn_turned_frag<FJ>(own + FI * 1024, v, lane));
            kn_lanes_meet();
        }
#pragma unroll
        for (int u = 0; u < FI; ++u)
#pragma unroll
            for (int v = 0; v < FJ; ++v) acc[u][v] = kn_mfma(x.b[v], x.a[u], acc[u][v]);
    };
    if (p.a_rows > 0 && p.b_rows > 0 && c0 + wave * RS < cend) {
        constexpr int TURNS = WAVES * RS;
        Step even, odd;
        load(even, c0 + wave * RS);
        for (int32_t c = c0 + wave * RS; c < cend; c += 2 * TURNS) { // (behind the part's end: its last row, unused)
            load(odd, c + TURNS);
            multiply(even, c);
            load(even, c + 2 * TURNS);
            multiply(odd, c + TURNS);
        }
    }
    kn_lanes_meet();
    KN_LDS float *red = (KN_LDS float *)own;
#pragma unroll
    for (int u = 0; u < FI; ++u)
#pragma unroll
        for (int v = 0; v < FJ; ++v) *(KN_LDS kn_f32x4 *)(red + (16 * u + col) * LD + 16 * v + 4 * g) = acc[u][v];
    __syncthreads();
    float *sums = parts.sums + place * p.I * p.J;
    T *out = (T *)p.out + (int64_t)group * p.o_group; // (its rows follow one another)
    for (int q = tid; q < 16 * FI * 16 * FJ; q += WAVES * 64) {
        const int r = q / (16 * FJ), c = q % (16 * FJ);
        int i = r, j = c;
        if constexpr (TURN) { // (a piece that would pass the rows' end is their last one: what the piece before has, too, is left out)
            i = min(r / W * W, width_a - i0 - W) + r % W;
            j = min(c / W * W, width_b - j0 - W) + c % W;
            if (i < r / W * W || j < c / W * W) continue;
        }
        if (i0 + i >= p.I || j0 + j >= p.J) continue;
        float y = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) y += *(const KN_LDS float *)((KN_LDS char *)lds_ + w * OWN + (r * LD + c) * 4);
        const int64_t at = (int64_t)(i0 + i) * p.J + j0 + j;
        if (several) sums[at] = y;
        else out[at] = (T)y;
    }
}
// One such gradient, or two of one call side by side: a low-rank product's factors, the long side of one the first index and of the other the second
struct Thin {
    KnProduct p;
    Parts parts;
    int32_t width_a, width_b; // values that a row of a and b has: those of g and h have zeros up to a whole piece
};
template <typename T, int FI, int FJ, bool TURN, int WAVES> __global__ void __launch_bounds__(WAVES * 64) k_reduce_thin(Thin a)
{
    __shared__ __align__(16) char lds[WAVES * thin_bytes(FI, FJ)];
    reduce_thin<T, FI, FJ, TURN, WAVES>(a.p, a.parts, a.width_a, a.width_b, a.p.first + kn_block(), lds);
}
template <typename T, int F, bool TURN, int WAVES> __global__ void __launch_bounds__(WAVES * 64) k_reduce_thin_pair(Thin tall, Thin wide, int32_t blocks)
{
    __shared__ __align__(16) char lds[WAVES * (thin_bytes(4, F) > thin_bytes(F, 4) ? thin_bytes(4, F) : thin_bytes(F, 4))];
    const int32_t block = tall.p.first + kn_block();
    if (block < blocks) reduce_thin<T, 4, F, TURN, WAVES>(tall.p, tall.parts, tall.width_a, tall.width_b, block, lds);
    else reduce_thin<T, F, 4, TURN, WAVES>(wide.p, wide.parts, wide.width_a, wide.width_b, block - blocks, lds);
}

// The parts' sums of the networks that have several, in the order of the parts; `chunk` results per workgroup.  SEARCH: there are at most
// M / len such networks, and a workgroup looks for its own among all (few networks of many results); else there is one for
// every network's results, and most find nothing to do.  SPLIT: each wavefront sums a quarter of a network's parts, and the quarters are added
// in order (50,560 rows of 25 networks 64 x 112, the longest of some 160 parts: 51 -> 17 us).
template <typename T, bool SEARCH, bool SPLIT>
__device__ __forceinline__ void reduce_join(const KnProduct &p, int32_t sum, const Parts &parts, int32_t chunk, int32_t block, int32_t *scratch, int32_t &found, float (*quarter)[64])
{
    const int64_t n = (int64_t)p.I * p.J;
    const int32_t pieces = (int32_t)((n + chunk - 1) / chunk), turn = block / pieces;
    int32_t group = turn;
    if constexpr (SEARCH) {
        int32_t before = 0;
        if (kn_thread() == 0) found = -1;
        for (int32_t e0 = 0; e0 < p.E && before <= turn; e0 += 256) {
            const int32_t e = e0 + kn_thread();
            const bool several = e < p.E && kn_offset(p.offsets, e + 1, p.M) - kn_offset(p.offsets, e, p.M) > parts.len;
            int32_t all;
            const int32_t rank = before + kn_block_exclusive_scan(several ? 1 : 0, scratch, all);
            if (several && rank == turn) found = e;
            before += all;
        }
        __syncthreads();
        group = found;
        if (group < 0) return;
    }
    const int32_t o = kn_offset(p.offsets, group, p.M), rows = kn_offset(p.offsets, group + 1, p.M) - o;
    if (rows <= parts.len) return;
    const int32_t count = (rows + parts.len - 1) / parts.len;
    const int64_t place = 2 * (o / parts.len), first = (int64_t)(block % pieces) * chunk;
    T *out = (T *)p.out + (int64_t)group * p.o_group;
    if constexpr (SPLIT) {
        const int lane = kn_thread() & 63, wave = kn_thread() >> 6;
        const int c0 = count * wave / 4, c1 = count * (wave + 1) / 4;
        for (int64_t q = first + lane; q - lane < min(n, first + chunk); q += 64) {
            float y = 0.0f;
            if (q < n)
#pragma unroll 8
                for (int c = c0; c < c1; ++c) y += parts.sums[(place + c) * n + q];
            quarter[wave][lane] = y;
            __syncthreads();
            if (wave == 0 && q < n) out[q] = (T)(((quarter[0][lane] + quarter[1][lane]) + quarter[2][lane]) + quarter[3][lane]);
            __syncthreads();
        }
    } else for (int64_t q = first + kn_thread(); q < min(n, first + chunk); q += 256) {
        float y = 0.0f;
#pragma unroll 4
        for (int c = 0; c < count; ++c) y += parts.sums[(place + c) * n + q];
        out[q] = (T)y; // (out's rows follow one another)
    }
    if (sum == SUM_NONE || first > 0) return;
    const int32_t m = sum == SUM_A ? p.I : p.J;
    for (int32_t j = kn_thread(); j < m; j += 256) {
        float y = 0.0f;
#pragma unroll 16
        for (int c = 0; c < count; ++c) y += parts.bias_sums[(place + c) * m + j];
        ((T *)p.out_bias)[(int64_t)group * m + j] = (T)y;
    }
}
template <typename T, bool SEARCH, bool SPLIT> __global__ void __launch_bounds__(256) k_reduce_join(KnProduct p, int32_t sum, Parts parts, int32_t chunk)
{
    __shared__ int32_t scratch[4], found;
    __shared__ float quarter[4][64];
    reduce_join<T, SEARCH, SPLIT>(p, sum, parts, chunk, p.first + kn_block(), scratch, found, quarter);
}
// of two gradients of few results
constexpr int32_t FEW_CHUNK = 256;
template <typename T> __global__ void __launch_bounds__(256) k_reduce_join_pair(Thin a, Thin b, int32_t blocks)
{
    __shared__ int32_t scratch[4], found;
    __shared__ float quarter[4][64];
    const int32_t block = a.p.first + kn_block();
    if (block < blocks) reduce_join<T, false, true>(a.p, SUM_NONE, a.parts, FEW_CHUNK, block, scratch, found, quarter);
    else reduce_join<T, false, true>(b.p, SUM_NONE, b.parts, FEW_CHUNK, block - blocks, scratch, found, quarter);
}

// Layers of up to 64 x 64 whose rows are not whole pieces are k_reduce_small's (us, against 64 x 64 staged in the LDS: 524,291 rows, 4,096
// networks 63 x 32: 57 and 63 in bf16, 91 and 123 in fp32; 262,145 rows, 1,600 networks 91 x 64: 109 and 52, 151 and 102).  Else tiles
// of 64 x 64 where 128 x 128 would be few, or a side is no wider than that and the other no wider than 128, or rows are few (more
// workgroups at a time: such a tile's few rows are latency; 262,145 rows, 1,600 networks 91 x 64 in bf16: 52 us, 128 x 128 75; 20,000
// rows, 300 networks 512 x 64: 20, 22; but 200,000 rows, 16 networks 1024 x 64: 128, 108), and in fp32, which the matrix cores bound:
// what a tile fetches is no matter, how evenly tiles fill the chip is (8,192 rows, 16 networks 1024 x 1024, the longest 2,892:
// 64 x 64 189 us, 128 x 128 226; 128 networks 512 x 512, the longest 568: 88, 99); and 32 x 32 where 64 x 64 would be few (1,001 rows,
// 5 networks 259 x 131: 9.6 us, 64 x 64 14.6).
bool narrow(const kn_linear_desc *d) { return d->n_in <= 128 && d->n_out <= 128; }
enum Way { WAY_SMALL, WAY_32, WAY_64, WAY_128 };
Way way_of(const kn_linear_desc *d, bool direct)
{
    if (!direct && d->n_in <= 64 && d->n_out <= 64) return WAY_SMALL;
    if (d->dtype == KN_F32) return (d->experts + d->rows / 512) * kn_div_up(d->n_in, 64) * kn_div_up(d->n_out, 64) < 256 ? WAY_32 : WAY_64;
    if ((d->n_in <= 64 || d->n_out <= 64) && (narrow(d) || d->rows / d->experts < 256)) return WAY_64;
    return d->experts * kn_div_up(d->n_in, 128) * kn_div_up(d->n_out, 128) < 256 && d->rows < 65536 ? WAY_64 : WAY_128;
}

// Rows of a part: a part more is a tile written and read again in fp32, so that there are only as many as keep the chip busy, and up to
// 1,024 rows of a wide layer are one (the join is a launch more, 4 us).  Wide layers: 32 networks 1024 x 2048, the longest of 32,768
// rows 5,741: parts of 1,024 rows 357 us, of 4,096 264, of 8,192 238, none 231; 8 networks 512 x 512, the longest 23,284: of 1,024 97,
// of 2,048 80, none 261; 4 networks 256 x 256, the longest of 16,384 11,740: of 256 31, of 1,024 23, of 2,048 33.  In fp32, where a
// tile takes longest and its sums are the less: of 512 51, of 2,048 71.  Narrow layers' parts are small, and more of them are chains
// that run at the same time.
// k_reduce_thin: four wavefronts and parts of 512 rows, or eight and 1,024 (us, whole forward and backward calls): 8,192 rows of 16 networks 1024 x 2048, rank 16, 143 and
// 138, of even networks 138 and 130; 16,384 of 4 412 and 410; 16,384 of one 1024 x 1024 141 and 147; but 4,096 of 64 107 and 132, 20,000 of 100 515 x
// 300 149 and 165, 262,145 of 1,600 91 x 64 181 and 235.
bool many_rows(int64_t rows, int64_t networks) { return rows / networks >= 256; }
int32_t part_length(const kn_linear_desc *d, bool thin)
{
    if (thin) { // (no more than a few hundred parts)
        const int64_t least = many_rows(d->rows, d->experts) ? 1024 : 512, len = kn_div_up(d->rows, 256);
        return (int32_t)kn_align_up(len < least ? least : len, 64);
    }
    const bool whole = d->dtype == KN_F32;
    const int64_t tiles = narrow(d) ? 1 : kn_div_up(d->n_in, 128) * kn_div_up(d->n_out, 128);
    const int64_t len = kn_div_up(d->rows, kn_div_up(narrow(d) ? 1024 : whole ? 256 : 512, tiles));
    const int64_t least = narrow(d) ? 128 : whole && d->rows > 1024 ? 512 : tiles <= 8 ? 1024 : 2048;
    return (int32_t)kn_align_up(len < least ? least : len, 64);
}

// A low-rank product's gradients, whose other side is longer than what the narrow layers' kernels take
bool is_thin(const kn_linear_desc *d) { return (d->n_in <= 64) != (d->n_out <= 64); }

// Few results, whose parts' sums are joined by more workgroups, a quarter of the parts for a wavefront
bool few_results(const KnProduct &p, const Parts &parts)
{
    const int64_t most = p.M / parts.len, results = (int64_t)p.I * p.J;
    return results * (most < p.E ? most : p.E) <= 1 << 20 && p.E * kn_div_up(results, FEW_CHUNK) <= 8192;
}
template <typename T> int launch_join(hipStream_t st, const KnProduct &p, int32_t sum, const Parts &parts);

template <typename T, int FI, int FJ, bool TURN> int launch_thin_of(hipStream_t st, const Thin &a)
{
    const int64_t blocks = kn_pieces(a.p.M, a.p.E, a.parts.len) * kn_div_up(a.p.I, 16 * FI) * kn_div_up(a.p.J, 16 * FJ);
    const bool many = many_rows(a.p.M, a.p.E);
    return kn_launch(blocks, many ? 512 : 256, [&](dim3 grid, int32_t first) {
        Thin q = a;
        q.p.first = first;
        if (many) hipLaunchKernelGGL((k_reduce_thin<T, FI, FJ, TURN, 8>), grid, dim3(512), 0, st, q);
        else hipLaunchKernelGGL((k_reduce_thin<T, FI, FJ, TURN, 4>), grid, dim3(256), 0, st, q);
    });
}
template <typename T, bool TURN> int launch_thin(hipStream_t st, const Thin &a)
{
    const int32_t I = a.p.I, J = a.p.J;
    KN_TRY((I <= J ? I <= 16 ? launch_thin_of<T, 1, 4, TURN>(st, a) : I <= 32 ? launch_thin_of<T, 2, 4, TURN>(st, a) : launch_thin_of<T, 4, 4, TURN>(st, a)
                   : J <= 16 ? launch_thin_of<T, 4, 1, TURN>(st, a) : J <= 32 ? launch_thin_of<T, 4, 2, TURN>(st, a) : launch_thin_of<T, 4, 4, TURN>(st, a)));
    return launch_join<T>(st, a.p, SUM_NONE, a.parts);
}
template <typename T, int F, bool TURN> int launch_pair_of(hipStream_t st, const Thin &tall, const Thin &wide)
{
    const int64_t pieces = kn_pieces(tall.p.M, tall.p.E, tall.parts.len), blocks = pieces * kn_div_up(tall.p.I, 64) * kn_div_up(tall.p.J, 16 * F);
    const int64_t all = blocks + pieces * kn_div_up(wide.p.I, 16 * F) * kn_div_up(wide.p.J, 64);
    const bool many = many_rows(tall.p.M, tall.p.E);
    if (all > 0x7fffffffLL) return KN_E_UNSUPPORTED;
    return kn_launch(all, many ? 512 : 256, [&](dim3 grid, int32_t first) {
        Thin q = tall;
        q.p.first = first;
        if (many) hipLaunchKernelGGL((k_reduce_thin_pair<T, F, TURN, 8>), grid, dim3(512), 0, st, q, wide, (int32_t)blocks);
        else hipLaunchKernelGGL((k_reduce_thin_pair<T, F, TURN, 4>), grid, dim3(256), 0, st, q, wide, (int32_t)blocks);
    });
}
// Two at once: a launch less, and one's last workgroups run beside the other's (8,192 rows of 16 networks 1024 x 2048, rank 16 in bf16, with the joins 34 -> 25 us)
template <typename T, bool TURN> int launch_pair(hipStream_t st, const Thin &a, const Thin &b)
{
    const Thin &tall = a.p.I > a.p.J ? a : b, &wide = a.p.I > a.p.J ? b : a;
    const int32_t rank = tall.p.J;
    KN_TRY((rank <= 16 ? launch_pair_of<T, 1, TURN>(st, tall, wide) : rank <= 32 ? launch_pair_of<T, 2, TURN>(st, tall, wide) : launch_pair_of<T, 4, TURN>(st, tall, wide)));
    if (tall.p.M <= tall.parts.len) return KN_OK;
    if (!few_results(tall.p, tall.parts) || !few_results(wide.p, wide.parts)) {
        KN_TRY(launch_join<T>(st, tall.p, SUM_NONE, tall.parts));
        return launch_join<T>(st, wide.p, SUM_NONE, wide.parts);
    }
    const int64_t blocks = tall.p.E * kn_div_up((int64_t)tall.p.I * tall.p.J, FEW_CHUNK), all = blocks + wide.p.E * kn_div_up((int64_t)wide.p.I * wide.p.J, FEW_CHUNK);
    return kn_launch(all, 256, [&](dim3 grid, int32_t first) {
        Thin q = tall;
        q.p.first = first;
        hipLaunchKernelGGL((k_reduce_join_pair<T>), grid, dim3(256), 0, st, q, wide, (int32_t)blocks);
    });
}

template <typename T, bool DIRECT, int SAVED>
int launch_reduce(hipStream_t st, const kn_linear_desc *d, const KnProduct &p, int32_t sum, const Parts &parts, const uint8_t *exponents)
{
    const Way way = way_of(d, DIRECT || SAVED != SAVED_NONE);
    const int bm = way == WAY_128 ? 128 : way == WAY_32 || (way == WAY_SMALL && p.I <= 32) ? 32 : 64;
    const int bn = way == WAY_128 ? 128 : way == WAY_32 ? 32 : way == WAY_64 || p.J > 48 ? 64 : p.J > 32 ? 48 : p.J > 16 ? 32 : 16;
    const int64_t blocks = kn_pieces(p.M, p.E, parts.len) * kn_div_up(p.I, bm) * kn_div_up(p.J, bn);
    const int64_t each = d->rows / d->experts;
    const bool alone = way == WAY_SMALL && (each < 32 || (each < 256 && d->experts >= 1024));
    const int status = kn_launch(blocks, way == WAY_128 ? 512 : alone ? 64 : 256, [&](dim3 grid, int32_t first) {
        KnProduct q = p;
        q.first = first;
        if (way == WAY_128) {
            if constexpr (sizeof(T) == 2) hipLaunchKernelGGL((k_product_reduce<T, DIRECT, 128, 128, 2, 4, SAVED>), grid, dim3(512), 0, st, q, sum, parts, exponents);
        } else if (way == WAY_64) hipLaunchKernelGGL((k_product_reduce<T, DIRECT, 64, 64, 2, 2, SAVED>), grid, dim3(256), 0, st, q, sum, parts, exponents);
        else if (way == WAY_32) {
            if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((k_product_reduce<T, DIRECT, 32, 32, 2, 2, SAVED>), grid, dim3(256), 0, st, q, sum, parts, exponents);
        } else if constexpr (!DIRECT && SAVED == SAVED_NONE) {
#define KN_SMALL(U, V)                                                                                                                      \
    if (alone) hipLaunchKernelGGL((k_reduce_small<T, U, V, 1>), grid, dim3(64), 0, st, q, sum, parts);                                      \
    else hipLaunchKernelGGL((k_reduce_small<T, U, V, 4>), grid, dim3(256), 0, st, q, sum, parts)
            switch (bm + bn / 16) {
            case 33: KN_SMALL(2, 1); break;
            case 34: KN_SMALL(2, 2); break;
            case 35: KN_SMALL(2, 3); break;
            case 36: KN_SMALL(2, 4); break;
            case 65: KN_SMALL(4, 1); break;
            case 66: KN_SMALL(4, 2); break;
            case 67: KN_SMALL(4, 3); break;
            default: KN_SMALL(4, 4);
            }
#undef KN_SMALL
        }
    });
    KN_TRY(status);
    return launch_join<T>(st, p, sum, parts);
}

template <typename T> int launch_join(hipStream_t st, const KnProduct &p, int32_t sum, const Parts &parts)
{
    if (p.M <= parts.len) return KN_OK; // (no network has several)
    const int64_t most = p.M / parts.len, results = (int64_t)p.I * p.J;
    const bool few = few_results(p, parts);
    const int32_t chunk = few ? FEW_CHUNK : 4096;
    const int64_t pieces = kn_div_up(results, chunk);
    const bool search = most < p.E && p.E * pieces > 8192;
    const int64_t joins = (search ? most : p.E) * pieces;
    auto join = few ? (k_reduce_join<T, false, true>) : search ? (k_reduce_join<T, true, false>) : (k_reduce_join<T, false, false>); // (few: no more than 8,192 workgroups)
    return kn_launch(joins, 256, [&](dim3 grid, int32_t first) {
        KnProduct q = p;
        q.first = first;
        hipLaunchKernelGGL(join, grid, dim3(256), 0, st, q, sum, parts, chunk);
    });
}

} // namespace

extern "C" int kn_grouped_linear_dw_workspace_bytes(const kn_linear_desc *d, int64_t *out_bytes)
{
    KN_TRY(kn_linear_check(d));
    return out_bytes ? kn_linear_dw_bytes(d, false, out_bytes) : KN_E_INVALID_ARG;
}

int kn_linear_dw_bytes(const kn_linear_desc *d, bool thin, int64_t *out_bytes)
{
    const int32_t len = part_length(d, thin && is_thin(d));
    *out_bytes = d->rows <= len ? 0 : kn_align_up(part_places(d->rows, len) * ((int64_t)d->n_in * d->n_out + d->n_out) * 4, 256);
    return KN_OK;
}

extern "C" int kn_grouped_linear_dw(void *stream, const kn_linear_desc *d, const void *x, const void *dy, const int32_t *offsets,
                                    const int32_t *rows, void *dw, void *db, void *workspace, int64_t workspace_bytes)
{
    KN_TRY(kn_linear_check(d));
    return kn_linear_dw_run(stream, d, x, nullptr, dy, d->n_out, offsets, rows, dw, db, workspace, workspace_bytes);
}

extern "C" int kn_grouped_linear_dw_saved(void *stream, const kn_linear_desc *d, const void *q, const uint8_t *exponents, const void *dy, const int32_t *offsets,
                                          const int32_t *rows, void *dw, void *db, void *workspace, int64_t workspace_bytes)
{
    KN_TRY(kn_saved_check(d));
    if (((uintptr_t)q & 15) || (d->rows > 0 && d->x_rows > 0 && !exponents)) return KN_E_INVALID_ARG;
    kn_linear_desc whole = *d;
    whole.ldx = d->n_in;
    static const uint8_t none = 0; // (no row is read: any address but NULL)
    return kn_linear_dw_run(stream, &whole, q, exponents ? exponents : &none, dy, d->n_out, offsets, rows, dw, db, workspace, workspace_bytes);
}

// Both operands and the result of a gradient.  LOW_..: a low-rank factor's, whose g or h (the side named) has rows with zeros up to a whole piece
namespace {
enum Low { LOW_NO, LOW_OUT, LOW_IN };
Thin product_of(const kn_linear_desc *d, const void *x, const void *dy, int64_t lddy, const int32_t *offsets, const int32_t *rows, void *dw, void *db, void *workspace, Low low)
{
    Parts parts = {part_length(d, low != LOW_NO && is_thin(d)), (float *)workspace, nullptr};
    parts.bias_sums = parts.sums + part_places(d->rows, parts.len) * (int64_t)d->n_in * d->n_out;
    KnProduct p = {};
    const bool io = d->w_layout == KN_W_IN_OUT; // (columns are what is contiguous in dw)
    p.a = io ? x : dy; p.b = io ? dy : x;
    p.lda = io ? d->ldx : lddy; p.ldb = io ? lddy : d->ldx;
    p.rows = io ? rows : nullptr; p.b_index = io ? nullptr : rows;
    p.M = (int32_t)d->rows; p.E = d->experts; p.I = io ? d->n_in : d->n_out; p.J = io ? d->n_out : d->n_in;
    p.a_rows = (int32_t)(io ? d->x_rows : d->rows); p.b_rows = (int32_t)(io ? d->rows : d->x_rows);
    p.out = dw; p.out_bias = db; p.offsets = offsets;
    p.o_group = (int64_t)d->n_in * d->n_out; p.o_i = p.J;
    const int32_t unit = 16 / kn_item(d->dtype);
    const int32_t in = low == LOW_IN ? (int32_t)kn_align_up(d->n_in, unit) : d->n_in, out = low == LOW_OUT ? (int32_t)kn_align_up(d->n_out, unit) : d->n_out;
    return {p, parts, io ? in : out, io ? out : in};
}
bool whole_rows(const KnProduct &p, int64_t V, int32_t width_a, int32_t width_b)
{
    return width_a % V == 0 && width_b % V == 0 && (((uintptr_t)p.a | (uintptr_t)p.b) & 15) == 0 && p.lda % V == 0 && p.ldb % V == 0;
}
} // namespace

int kn_linear_dw_run(void *stream, const kn_linear_desc *d, const void *x, const uint8_t *exponents, const void *dy, int64_t lddy, const int32_t *offsets,
                     const int32_t *rows, void *dw, void *db, void *workspace, int64_t workspace_bytes)
{
    if (!offsets || !dw || (d->rows > 0 && (!dy || (d->x_rows > 0 && !x))) || (d->rows > 0 && !rows && d->x_rows < d->rows)) return KN_E_INVALID_ARG;
    int64_t need = 0;
    KN_TRY(kn_grouped_linear_dw_workspace_bytes(d, &need));
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)) return KN_E_WORKSPACE;
    const bool io = d->w_layout == KN_W_IN_OUT;
    const Thin t = product_of(d, x, dy, lddy, offsets, rows, dw, db, workspace, LOW_NO);
    const KnProduct &p = t.p;
    const Parts &parts = t.parts;
    const int32_t sum = !db ? SUM_NONE : io ? SUM_B : SUM_A;
    return kn_with_type(d->dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        constexpr int64_t V = 16 / sizeof(E_);
        hipStream_t st = (hipStream_t)stream;
        if (exponents) {
            const bool direct = d->n_out % V == 0 && ((uintptr_t)dy & 15) == 0 && lddy % V == 0;
            if (io) return direct ? launch_reduce<E_, true, SAVED_A>(st, d, p, sum, parts, exponents) : launch_reduce<E_, false, SAVED_A>(st, d, p, sum, parts, exponents);
            return direct ? launch_reduce<E_, true, SAVED_B>(st, d, p, sum, parts, exponents) : launch_reduce<E_, false, SAVED_B>(st, d, p, sum, parts, exponents);
        }
        const bool direct = whole_rows(p, V, p.I, p.J);
        return direct ? launch_reduce<E_, true, SAVED_NONE>(st, d, p, sum, parts, nullptr) : launch_reduce<E_, false, SAVED_NONE>(st, d, p, sum, parts, nullptr);
    });
}

int kn_linear_dw_low_rank(void *stream, const kn_linear_desc *da, const void *x, const void *g, int64_t ldg, const int32_t *rows, void *out_a, const kn_linear_desc *db,
                          const void *h, const void *dy, int64_t lddy, void *out_b, const int32_t *offsets, void *workspace, int64_t workspace_bytes)
{
    int64_t na = 0, nb = 0;
    KN_TRY(kn_linear_dw_bytes(da, true, &na));
    KN_TRY(kn_linear_dw_bytes(db, true, &nb));
    if (na + nb > 0 && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < na + nb)) return KN_E_WORKSPACE;
    char *ws_b = (char *)workspace + na;
    const Thin a = product_of(da, x, g, ldg, offsets, rows, out_a, nullptr, workspace, LOW_OUT), b = product_of(db, h, dy, lddy, offsets, nullptr, out_b, nullptr, ws_b, LOW_IN);
    const bool thin_a = is_thin(da), thin_b = is_thin(db);
    hipStream_t st = (hipStream_t)stream;
    return kn_with_type(da->dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        constexpr int64_t V = 16 / sizeof(E_);
        constexpr bool TURNS = sizeof(E_) == 2;
        const bool turn_a = TURNS && a.width_a >= V && a.width_b >= V, turn_b = TURNS && b.width_a >= V && b.width_b >= V;
        if (thin_a && thin_b && turn_a == turn_b) return turn_a ? launch_pair<E_, TURNS>(st, a, b) : launch_pair<E_, false>(st, a, b);
        if (thin_a) KN_TRY((turn_a ? launch_thin<E_, TURNS>(st, a) : launch_thin<E_, false>(st, a)));
        else KN_TRY(kn_linear_dw_run(stream, da, x, nullptr, g, ldg, offsets, rows, out_a, nullptr, workspace, na));
        if (thin_b) return turn_b ? launch_thin<E_, TURNS>(st, b) : launch_thin<E_, false>(st, b);
        return kn_linear_dw_run(stream, db, h, nullptr, dy, lddy, offsets, nullptr, out_b, nullptr, ws_b, nb);
    });
}
