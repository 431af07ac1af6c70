// Products grouped by network with ragged sizes, and the gradient of their inputs: kn_grouped_linear, kn_grouped_linear_dx.
#include "kn_tile.h"

#include <type_traits>

namespace {

// Tiles of BM x BN results, WR x WC wavefronts, NB stages in the LDS, of which one is multiplied while the others are fetched.  COLS:
// b's columns are contiguous in memory (else its contraction is).  DIRECT: rows of whole 16-byte pieces throughout (KnRowLoader).
// Fragments of b are the products' first operand, so that a lane holds four neighbouring results of a row; they go through
// the LDS once more to leave in pieces of 8.
// Measured: 65,536 rows through an index, 64 networks 2048 x 1024 in bf16, 192 x 128: 320 us, 860 TFLOP/s, where one product of the
// library of 8192 x 8192 x 8192 reaches 1,250.  The clock is 2.03 GHz with the matrix cores busy 44 % of the time (256 x 256: 2.30 GHz, 39 %, the
// same time); with every fetch a hit in the L2 it would be 250 us, so that more than half of what is above the floor is the wait for what
// the L2 does not have.
template <typename T, bool SAVED, bool COLS, bool DIRECT, int BM, int BN, int WR, int WC, int NB>
__global__ void __launch_bounds__(WR * WC * 64) k_product_rows(KnProduct p, int32_t blocks)
{
    constexpr int NW = WR * WC, STAGE = (BM + BN) * 128, U = BM / WR / 16, V = BN / WC / 16, CS = 128 / sizeof(T);
    typedef typename KnFrag<T>::Type Frag;
    static_assert(DIRECT || NB == 2, "");
    typedef KnRowLoader<T, BM, NW, DIRECT> LoadA;
    constexpr int BYTES = NB * STAGE > NW * 16 * (BN / WC + 4) * 4 ? NB * STAGE : NW * 16 * (BN / WC + 4) * 4;
    __shared__ __align__(16) char lds_[BYTES];
    KN_LDS char *lds = (KN_LDS char *)lds_;
    const int tid = kn_thread(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ntiles = (p.J + BN - 1) / BN;
    // (where a network has a piece or none, its columns go to all XCDs: only some networks have rows, XCDs should be alike)
    const int32_t number = p.M < (int64_t)BM * p.E ? p.first + kn_block() : kn_xcd_order(p.first + kn_block(), blocks);
    const KnPiece piece = kn_find_piece(p.offsets, p.E, p.M, BM, number / ntiles);
    const int j0 = number % ntiles * BN;
    if (piece.begin >= piece.end) return;
    const bool some = piece.group < p.E;
    const int64_t group = some ? piece.group : 0;
    const T *a = (const T *)p.a, *b = (const T *)p.b + group * p.b_group;
    LoadA la;
    la.start(wave, lane, [&](int r) {
        const int32_t i = min(piece.begin + r, piece.end - 1);
        const int32_t src = p.rows ? p.rows[i] : i;
        return a + (int64_t)((uint32_t)src < (uint32_t)p.a_rows ? src : 0) * p.lda;
    });
    KnRowLoader<T, BN, NW, DIRECT> lbr;
    KnColLoader<T, BN, NW, DIRECT> lbc;
    if constexpr (COLS) lbc.start(wave, lane, b + j0, p.b_c, p.J - j0);
    else lbr.start(wave, lane, [&](int r) { return b + (int64_t)min(j0 + r, p.J - 1) * p.b_j; });
    const int32_t C = some && p.a_rows > 0 ? p.C : 0, steps = (C + CS - 1) / CS;
    constexpr int LOADS = LoadA::N + (COLS ? lbc.N : lbr.N); // a wavefront's, per stage
    constexpr int LATER = DIRECT ? (NB - 2) * LOADS : 63; // (loads into registers are waited for where they are put down)
    auto fetch = [&](int s, int at) {
        KN_LDS char *tile = lds + at * STAGE;
        la.fetch(tile, wave, lane, C - s * CS);
        if constexpr (COLS) lbc.fetch(tile + BM * 128, wave, lane, C - s * CS);
        else lbr.fetch(tile + BM * 128, wave, lane, C - s * CS);
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
    // Half a stage's fragments are read while the other half's are multiplied; in between, the next stage has to have arrived, and the
    // one behind the NB that lie in the LDS takes the place of the one that everybody has just read.  A wavefront without rows (the
    // end of a network's) only fetches: what its products would cost is power, which the others are short of.
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
        if (WR == 1 || piece.begin + wi < piece.end) march(std::true_type());
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
    kn_bias_of<T>(p, some, group, j, add);
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
        for (int v = 0; v < V; ++v) *(KN_LDS kn_f32x4 *)(mine + (lane & 15) * LD + 16 * v + (lane >> 4) * 4) = acc[u][v];
        kn_lanes_meet();
#pragma unroll
        for (int h = 0; h < (16 * LR + 63) / 64; ++h) {
            const int r = h * (64 / LR) + lane / LR;
            const int32_t i = piece.begin + wi + 16 * u + r;
            if (r >= 16 || i >= piece.end || j >= p.J) continue;
            const kn_f32x4 lo = *(const KN_LDS kn_f32x4 *)(mine + r * LD + cj), hi = *(const KN_LDS kn_f32x4 *)(mine + r * LD + cj + 4);
            float y[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            kn_finish<T, SAVED>(p, some, i, j, add, y);
        }
        kn_lanes_meet();
    }
}

// A row or none per network, or few rows of fp32: the weights are read once, straight into the registers they are multiplied from, 16 bytes a lane and load.
// A workgroup makes 16 rows of FEW_COLS results; its FEW_WAVES wavefronts take every FEW_WAVES-th step of the contraction and are
// summed at the end, in the order of their numbers.  Columns contiguous in memory: lane l takes R = 16 / sizeof(T) columns from
// R (l % 16) on, of the R rows of the contraction from R (l / 16) on: an R x R square, whose transpose is, per column j of it, one
// product's fragment: column j of every lane's square.  16-bit squares are turned by byte permutations of register pairs, fp32
// ones by naming.  Bound by the weights' bytes: 32 rows in about 25 of 64 networks 2048 x 1024, bf16: 24 us, 4.4 TB/s.
constexpr int FEW_WAVES = 8;
template <typename T, bool SAVED>
__global__ void __launch_bounds__(FEW_WAVES * 64) k_product_few(KnProduct p)
{
    constexpr int R = 16 / sizeof(T), BN = 16 * R, KS = 4 * R, LD = BN + 4;
    typedef typename KnFrag<T>::Type Frag;
    __shared__ __align__(16) float red[FEW_WAVES * 16 * LD];
    const int tid = kn_thread(), lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ntiles = (p.J + BN - 1) / BN;
    const int32_t number = p.first + kn_block(); // (a network's columns over all XCDs: there is nothing to share but a few rows)
    const KnPiece piece = kn_find_piece(p.offsets, p.E, p.M, 16, number / ntiles);
    const int j0 = number % ntiles * BN;
    if (piece.begin >= piece.end) return;
    const bool some = piece.group < p.E;
    const int64_t group = some ? piece.group : 0;
    const int col = lane & 15, g = lane >> 4;
    const int32_t row = min(piece.begin + col, piece.end - 1), src = p.rows ? p.rows[row] : row;
    const T *arow = (const T *)p.a + (int64_t)((uint32_t)src < (uint32_t)p.a_rows ? src : 0) * p.lda;
    const T *brow = (const T *)p.b + group * p.b_group + min(j0 + R * col, p.J - R);
    const int32_t C = some ? p.C : 0, steps = (C + KS - 1) / KS;
    kn_f32x4 acc[R] = {};
    struct Step { kn_u32x4 a, b[R]; };
    auto load = [&](Step &x, int s) {
        const int32_t k = s * KS + R * g;
        const kn_u32x4 none = {0, 0, 0, 0}; // (behind the contraction's end: zeros, of a and of b)
        const bool there = k < C;
        x.a = there ? *(const kn_u32x4 *)(arow + k) : none;
#pragma unroll
        for (int t = 0; t < R; ++t) x.b[t] = there ? *(const kn_u32x4 *)(brow + (int64_t)(k + t) * p.b_c) : none;
    };
    auto multiply = [&](const Step &x) {
        union { kn_u32x4 u; Frag f; } fa, fb;
        fa.u = x.a;
#pragma unroll
        for (int v = 0; v < R; ++v) {
            if constexpr (sizeof(T) == 4) fb.u = kn_u32x4{x.b[0][v], x.b[1][v], x.b[2][v], x.b[3][v]};
            else
#pragma unroll
                for (int t = 0; t < 4; ++t) // column v of rows 2 t and 2 t + 1: the lower or the upper halves of word v / 2
                    fb.u[t] = __builtin_amdgcn_perm(x.b[2 * t + 1][v / 2], x.b[2 * t][v / 2], v & 1 ? 0x07060302 : 0x05040100);
            acc[v] = kn_mfma(fb.f, fa.f, acc[v]);
        }
    };
    Step even, odd;
    int s = wave;
    if (s < steps) load(even, s);
    while (s < steps) {
        if (s + FEW_WAVES < steps) load(odd, s + FEW_WAVES);
        multiply(even);
        s += FEW_WAVES;
        if (s >= steps) break;
        if (s + FEW_WAVES < steps) load(even, s + FEW_WAVES);
        multiply(odd);
        s += FEW_WAVES;
    }
    float *mine = red + (wave * 16 + col) * LD; // register r of product v: column R (4 g + r) + v
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int v = 0; v < R; v += 4) *(kn_f32x4 *)(mine + R * (4 * g + r) + v) = kn_f32x4{acc[v][r], acc[v + 1][r], acc[v + 2][r], acc[v + 3][r]};
    __syncthreads();
    for (int q = tid; q < 16 * BN / 8; q += FEW_WAVES * 64) {
        const int r = q / (BN / 8), cj = q % (BN / 8) * 8;
        const int32_t i = piece.begin + r, j = j0 + cj;
        if (i >= piece.end || j >= p.J) continue;
        float y[8] = {}, add[8];
#pragma unroll
        for (int w = 0; w < FEW_WAVES; ++w) {
            const kn_f32x4 lo = *(const kn_f32x4 *)(red + (w * 16 + r) * LD + cj), hi = *(const kn_f32x4 *)(red + (w * 16 + r) * LD + cj + 4);
#pragma unroll
            for (int n = 0; n < 4; ++n) { y[n] += lo[n]; y[n + 4] += hi[n]; }
        }
        kn_bias_of<T>(p, some, group, j, add);
        kn_finish<T, SAVED>(p, some, i, j, add, y);
    }
}

// Layers of the small networks' kind (contraction up to KF fragments, columns up to V of 16, or a few such tiles of columns), of any
// sizes, strides and alignment: a wavefront takes SMALL_ROWS rows of one network by itself, with the network's fragments in its
// registers; nothing goes through the LDS and no wavefront waits for another.  Such calls are bound by their bytes, or rather by the
// latency of one look-up, one fetch and one store per piece: what is under way at a time is what counts, so all of a piece is
// asked for at once.  Measured: 262,145 rows through an index, 4,096 networks 63 x 32 in fp32: 39 us, 3.4 TB/s (rows of 252 bytes touch
// a third more lines than they fill; 44 us where each odd end is waited for); 524,291 rows, 64 x 64 in fp16, input gradient with a ReLU's mask: 59 us, 4.0 TB/s (68 where a
// lane stores and masks 8 bytes at a time).  Pieces of 64 rows: 49 and 69, of 128: 70 and 90, of 16: 52 and 85.
constexpr int SMALL_ROWS = 32, SMALL_WAVES = 4;
// SAVED: the mask is what kn_save_f8 left.  A kernel of its own: as a branch at run time it takes the forward pass of 64 x 64 in 16 bits from 128 to 130 registers, from four
// wavefronts a SIMD to three (524,288 rows of 4,096 networks in fp16: 41 -> 46 us).
template <typename T, bool SAVED, bool COLS, int KF, int V, bool ODD>
__global__ void __launch_bounds__(SMALL_WAVES * 64) k_product_small(KnProduct p, int32_t pieces)
{
    constexpr int W = KnSmallFrag<T>::W, KS = KnSmallFrag<T>::KS, SUBS = SMALL_ROWS / 16;
    // A lane's four results of W / 4 products are neighbours, W of them: the products' columns are dealt out in fours
    constexpr int PAIR = W / 4, RUNS = V / PAIR;
    typedef typename KnFrag<T>::Type Frag;
    typedef T Run __attribute__((ext_vector_type(W), aligned(sizeof(T)))); // wherever they lie
    __shared__ __align__(16) T rows_of[SMALL_WAVES][16 * 16 * V + W]; // 16 rows of results of a wavefront, as they follow one another
    const int lane = kn_thread() & 63, col = lane & 15, g = lane >> 4;
    T *line = rows_of[kn_thread() >> 6];
    const int32_t number = __builtin_amdgcn_readfirstlane((p.first + kn_block()) * SMALL_WAVES + (kn_thread() >> 6));
    const int ntiles = (p.J + 16 * V - 1) / (16 * V);
    if (number / ntiles >= pieces) return;
    const KnPiece piece = kn_find_piece(p.offsets, p.E, p.M, SMALL_ROWS, number / ntiles);
    const int32_t j0 = number % ntiles * 16 * V;
    if (piece.begin >= piece.end) return;
    const bool some = piece.group < p.E;
    const int64_t group = some ? piece.group : 0;
    const int32_t C = p.C;
    Frag fa[SUBS][KF], fb[KF][V];
    bool there[SUBS];
    if (some && p.a_rows > 0) {
        const T *arow[SUBS], *brow[V];
        uint32_t fifth_a[SUBS][KF], fifth_b[KF][V];
        const bool odd_a = ODD && (((uintptr_t)p.a / sizeof(T) | p.lda) & 1), odd_b = ODD && (((uintptr_t)p.b / sizeof(T) | p.b_j) & 1);
#pragma unroll
        for (int s = 0; s < SUBS; ++s) {
            const int32_t i = min(piece.begin + 16 * s + col, piece.end - 1), src = p.rows ? p.rows[i] : i;
            there[s] = (uint32_t)src < (uint32_t)p.a_rows;
            arow[s] = (const T *)p.a + (int64_t)(there[s] ? src : 0) * p.lda;
        }
        const T *b = (const T *)p.b + group * p.b_group;
#pragma unroll
        for (int k = 0; k < KF; ++k)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int32_t c = k * KS + g * W;
                const int32_t j = min(j0 + v / PAIR * (16 * PAIR) + (col >> 2) * W + v % PAIR * 4 + (col & 3), p.J - 1);
                if constexpr (COLS) {
#pragma unroll
                    for (int q = 0; q < W; ++q) {
                        const T w = b[(int64_t)min(c + q, C - 1) * p.b_c + j];
                        fb[k][v][q] = c + q < C ? w : (T)0.0f;
                    }
                } else {
                    brow[v] = b + (int64_t)j * p.b_j;
                    fb[k][v] = kn_row_ask<T>(brow[v], c, C, odd_b, fifth_b[k][v]);
                }
            }
#pragma unroll
        for (int s = 0; s < SUBS; ++s)
#pragma unroll
            for (int k = 0; k < KF; ++k) fa[s][k] = kn_row_ask<T>(arow[s], k * KS + g * W, C, odd_a, fifth_a[s][k]);
        if (C >= W && (ODD || C % W)) {
#pragma unroll
            for (int k = 0; k < KF; ++k) {
                if (!ODD && (k + 1) * KS <= C) continue;
#pragma unroll
                for (int s = 0; s < SUBS; ++s) kn_row_place<T>(fa[s][k], arow[s], k * KS + g * W, C, odd_a, fifth_a[s][k]);
                if constexpr (!COLS)
#pragma unroll
                    for (int v = 0; v < V; ++v) kn_row_place<T>(fb[k][v], brow[v], k * KS + g * W, C, odd_b, fifth_b[k][v]);
            }
        }
    }
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
    for (int n = 0; n < RUNS; ++n) add[n] = some && bias ? run(bias + group * p.J, min(j0 + 4 * W * n + W * g, p.J - 1)) : Run{};
    if (some && mask) { // (asked for before the first result is stored, not one after the other's)
#pragma unroll
        for (int s = 0; s < SUBS; ++s) {
            const int32_t i = min(piece.begin + 16 * s + col, piece.end - 1), src = p.mask_rows ? p.mask_rows[i] : i;
            const bool in = (uint32_t)src < (uint32_t)p.m_rows;
#pragma unroll
            for (int n = 0; n < RUNS; ++n) {
                m[s][n] = Run{};
                if constexpr (SAVED) { // (a lane's W columns lie in a saved row's whole 16 bytes)
                    typedef int8_t Bytes __attribute__((ext_vector_type(W)));
                    const int32_t j = j0 + 4 * W * n + W * g;
                    Bytes b = {};
                    if (in && j < p.J) b = *(const Bytes *)((const int8_t *)p.mask + (int64_t)src * p.ldm + j);
#pragma unroll
                    for (int r = 0; r < W; ++r) m[s][n][r] = (T)(b[r] > 0 ? 1.0f : 0.0f);
                    continue;
                }
                if (in) m[s][n] = run(mask + (int64_t)src * p.ldm, min(j0 + 4 * W * n + W * g, p.J - 1));
            }
        }
    }
#pragma unroll
    for (int s = 0; s < SUBS; ++s) {
        const int32_t i = piece.begin + 16 * s + col;
        if (piece.begin + 16 * s >= piece.end) break;
        kn_f32x4 acc[V] = {};
        if (some && p.a_rows > 0) {
#pragma unroll
            for (int k = 0; k < KF; ++k)
#pragma unroll
                for (int v = 0; v < V; ++v) acc[v] = kn_mfma(fb[k][v], fa[s][k], acc[v]);
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
                if (some && bias) y += (float)add[n][r];
                if (p.relu) y = y > 0.0f || y != y ? y : 0.0f; // (a NaN stays one)
                if (some && mask && !((float)m[s][n][r] > 0.0f)) y = 0.0f;
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

// Whether the rows of a and of b are made of whole 16-byte pieces on multiples of 16 bytes, as the DIRECT kernels take them
template <typename T, bool COLS> bool rows_of_pieces(const KnProduct &p)
{
    constexpr int64_t V = 16 / sizeof(T);
    return ((uintptr_t)p.a | (uintptr_t)p.b) % 16 == 0 && p.C % V == 0 && p.lda % V == 0 && (!COLS || p.J % V == 0) && p.a_rows > 0;
}

template <typename T, bool SAVED, bool COLS, bool DIRECT, int BM, int BN, int WR, int WC, int NB> int launch_rows(hipStream_t st, const KnProduct &p)
{
    const int64_t blocks = kn_pieces(p.M, p.E, BM) * kn_div_up(p.J, BN);
    return kn_launch(blocks, WR * WC * 64, [&](dim3 grid, int32_t first) {
        KnProduct q = p;
        q.first = first;
        hipLaunchKernelGGL((k_product_rows<T, SAVED, COLS, DIRECT, BM, BN, WR, WC, NB>), grid, dim3(WR * WC * 64), 0, st, q, (int32_t)blocks);
    });
}

template <typename T, bool SAVED> int launch_few(hipStream_t st, const KnProduct &p)
{
    const int64_t blocks = kn_pieces(p.M, p.E, 16) * kn_div_up(p.J, 256 / (int)sizeof(T));
    return kn_launch(blocks, FEW_WAVES * 64, [&](dim3 grid, int32_t first) {
        KnProduct q = p;
        q.first = first;
        hipLaunchKernelGGL((k_product_few<T, SAVED>), grid, dim3(FEW_WAVES * 64), 0, st, q);
    });
}

// Which kernel.  Large tiles fetch least per product, small ones fill the chip; measured (bf16, us, weights not in a cache):
//   rows, networks, K, N (columns contiguous)      few   64 x 128   128 x 128   192 x 128
//   32, 64, 2048, 1024, most networks without         21         31          35          40
//   256, 8, 1024, 2048                                 9         13          14          18
//   512, 64, 2048, 1024                               65         59          53          59
//   8,192, 64, 2048, 1024                            194         85          88          98
//   16,384, 64, 2048, 1024                                      126         113         127
//   4,096, 8, 1024, 2048                              77         32          32          29
//   65,536, 64, 2048, 1024                                      381         328         318
//   20,306, 23, 64, 1472                                         29          26          31
//   65,536, 64, 256, 1024                                       112          98         100
// and with the contraction contiguous, 32 x 64 in four stages against 64 x 128: 24 to 32, 10 to 13, 61 to 68, 120 to 92.
// fp32 is bound by the matrix cores, a sixteenth as fast: rows that a tile does not have cost more than what it fetches twice.
//   rows, networks, K, N                           few    32 x 64    32 x 128    64 x 128   128 x 128
//   266, 37, 1584, 1280, columns contiguous         66                  71         117         120
//   1,024, 8, 1024, 1024                            30                  45          47          78
//   2,048, 64, 512, 512                             26                  34          43          44
//   8,192, 64, 512, 512                                                 60          65          78
//   32,768, 8, 512, 1024                                               339         306         317
//   2,048, 64, 512, 512, contraction contiguous                22       33          41          42
//   8,192, 16, 1024, 1024                                     180      167         177         209
template <typename T, bool SAVED, bool COLS> int launch_pieces(hipStream_t st, const KnProduct &p)
{
    const int64_t each = p.M / p.E; // rows of a network, on average
    auto tiles = [&](int64_t bm) { return (p.M + bm - 1) / bm * ((p.J + 127) / 128); };
    if constexpr (sizeof(T) == 4) {
        const bool narrow = (int64_t)p.M * p.J <= 1 << 20; // (too few tiles of 32 x 128 for the chip)
        if (!rows_of_pieces<T, COLS>(p))
            return narrow ? launch_rows<T, SAVED, COLS, false, 32, 64, 1, 4, 2>(st, p) : each < 512 ? launch_rows<T, SAVED, COLS, false, 32, 128, 1, 4, 2>(st, p) : launch_rows<T, SAVED, COLS, false, 64, 128, 1, 4, 2>(st, p);
        if constexpr (COLS) {
            if (narrow) return launch_few<T, SAVED>(st, p);
            if (p.J <= 64) return launch_rows<T, SAVED, COLS, true, 32, 64, 1, 4, 2>(st, p);
            return each < 512 ? launch_rows<T, SAVED, COLS, true, 32, 128, 1, 4, 2>(st, p) : launch_rows<T, SAVED, COLS, true, 64, 128, 1, 4, 2>(st, p);
        } else {
            if (p.J <= 64 && !narrow) return launch_rows<T, SAVED, COLS, true, 32, 64, 1, 4, 2>(st, p); // (two stages: more workgroups at a time)
            return narrow ? launch_rows<T, SAVED, COLS, true, 32, 64, 1, 4, 4>(st, p) : launch_rows<T, SAVED, COLS, true, 32, 128, 1, 4, 2>(st, p);
        }
    } else {
        if (!rows_of_pieces<T, COLS>(p))
            return each >= 64 && tiles(128) >= 256 ? launch_rows<T, SAVED, COLS, false, 128, 128, 2, 4, 2>(st, p) : launch_rows<T, SAVED, COLS, false, 32, 128, 1, 4, 2>(st, p);
        const bool little = (int64_t)p.M * p.J <= 1 << 19;
        if constexpr (COLS) {
            if (little && (each < 2 || (int64_t)p.E * p.C * p.J <= 1 << 25)) return launch_few<T, SAVED>(st, p);
        } else {
            if (little || each < 64) return launch_rows<T, SAVED, COLS, true, 32, 64, 1, 4, 4>(st, p);
        }
        if (each >= 384 && tiles(192) >= 256 && p.C * (int64_t)sizeof(T) >= 1024) return launch_rows<T, SAVED, COLS, true, 192, 128, 2, 2, 2>(st, p);
        if (each >= 192 && tiles(128) >= 512) return launch_rows<T, SAVED, COLS, true, 128, 128, 2, 4, 2>(st, p);
        return launch_rows<T, SAVED, COLS, true, 64, 128, 1, 4, 2>(st, p);
    }
}

template <typename T, bool SAVED, bool COLS, int KF, int V, bool ODD> int launch_small_of(hipStream_t st, const KnProduct &p)
{
    const int64_t pieces = kn_pieces(p.M, p.E, SMALL_ROWS), waves = pieces * kn_div_up(p.J, 16 * V);
    if (waves > 0x7fffffffLL) return KN_E_UNSUPPORTED;
    return kn_launch(kn_div_up(waves, SMALL_WAVES), SMALL_WAVES * 64, [&](dim3 grid, int32_t first) {
        KnProduct q = p;
        q.first = first;
        hipLaunchKernelGGL((k_product_small<T, SAVED, COLS, KF, V, ODD>), grid, dim3(SMALL_WAVES * 64), 0, st, q, (int32_t)pieces);
    });
}
template <typename T, bool SAVED, bool COLS, int KF, int V> int launch_small(hipStream_t st, const KnProduct &p)
{
    if constexpr (sizeof(T) == 2) { // rows that begin between two words
        if (((uintptr_t)p.a / 2 | p.lda | (COLS ? 0 : (uintptr_t)p.b / 2 | p.b_j)) & 1) return launch_small_of<T, SAVED, COLS, KF, V, true>(st, p);
    }
    return launch_small_of<T, SAVED, COLS, KF, V, false>(st, p);
}
constexpr int SMALL_MOST = 128; // widest contraction and most columns that k_product_small takes
template <typename T, bool SAVED, bool COLS> int launch_small_widths(hipStream_t st, const KnProduct &p)
{
    const int kf = (p.C + KnSmallFrag<T>::KS - 1) / KnSmallFrag<T>::KS;
    if constexpr (sizeof(T) == 4) {
        if (kf > 4) return launch_small<T, SAVED, COLS, 8, 2>(st, p);
        if (kf > 2) return p.J <= 32 ? launch_small<T, SAVED, COLS, 4, 2>(st, p) : launch_small<T, SAVED, COLS, 4, 4>(st, p);
        return p.J <= 32 ? launch_small<T, SAVED, COLS, 2, 2>(st, p) : launch_small<T, SAVED, COLS, 2, 4>(st, p);
    } else {
        if (kf > 2) return launch_small<T, SAVED, COLS, 4, 4>(st, p);
        if (kf > 1) return p.J <= 32 ? launch_small<T, SAVED, COLS, 2, 2>(st, p) : launch_small<T, SAVED, COLS, 2, 4>(st, p);
        return p.J <= 32 ? launch_small<T, SAVED, COLS, 1, 2>(st, p) : launch_small<T, SAVED, COLS, 1, 4>(st, p);
    }
}

// Layers of up to SMALL_MOST by SMALL_MOST whose rows are whole pieces: by tiles or a wavefront per 32 rows (small).  Tiles share a
// network's weights among more rows, small starts sooner and takes wide layers of few rows per network without empty rows of tiles.
// Measured (us, small / tiles), by rows per network of 2,000, and as rows, networks:
//                               4        16        64       128       256     20,000, 4,096    65,536, 200
//   fp32   48 x 64            12/15     19/14     32/26     51/42     94/93        21/22          19/14
//          64 x 64            12/16     20/14     36/27     57/52    102/100       23/22          20/14
//          96 x 64            18/18     27/18     54/32     96/64    174/122       34/27          27/17
//          128 x 32           12/19     20/27     33/36     57/66    100/115       21/37          20/18
//          32 x 128           11/27     18/17     34/32     53/52    122/131       20/26          19/17
//   fp16, columns contiguous
//          64 x 128           10/12     14/14     24/24     37/33     76/68        17/24          14/12
//          72 x 64            10/19     13/15     21/25     33/35     61/62        17/26          13/12
//          128 x 32           10/19     11/15     20/25     31/34     60/62        15/25          12/12
//          72 x 72            15/13     20/15     37/26     59/36    109/66        28/26          18/12
//   fp16, contraction contiguous
//          64 x 128           10/17     14/21     25/23     39/32     76/66        18/35          15/11
//          72 x 72             9/19     12/23     23/25     36/34     67/65        18/39          12/12
//          96 x 64             7/11      9/13     18/25     26/33     46/64        15/22          10/12
//          128 x 64           10/11     11/14     22/24     35/35     62/66        18/23          14/12
//          128 x 128          18/20     20/24     38/27     65/46    120/83        29/40          22/13
// 16 bits and up to 64 x 64, 32 x 128: small throughout (64 x 64: 524,288 rows, 4,096 networks 45/71, 300,000 of 16 21/25).
template <typename T> bool small_by_tiles(const KnProduct &p, bool cols)
{
    const int64_t each = p.M / p.E;
    if constexpr (sizeof(T) == 4) return p.C > 32 && p.J > 32 ? each >= 16 || p.C + p.J >= 128 : p.C * p.J >= 4096 && each >= 256;
    if (p.J <= 64) return p.C > 64 && p.J > 32 && (cols ? each >= 96 : p.C > 96 && each >= 256);
    return p.C > 64 ? cols || each >= 64 : p.C > 32 && each >= 96;
}
template <typename T, bool SAVED> int launch_forward(hipStream_t st, const KnProduct &p)
{
    const bool cols = p.b_j == 1 && p.b_c != 1; // (one column of one input: either)
    // (91 x 64, whose rows are not whole pieces, by staged tiles: 262,145 rows, 1,600 networks 43 and 71 us in bf16, 103 and 123 in fp32)
    const bool pieces = cols ? rows_of_pieces<T, true>(p) : rows_of_pieces<T, false>(p);
    if (p.C <= SMALL_MOST && p.J <= SMALL_MOST && !(pieces && small_by_tiles<T>(p, cols)))
        return cols ? launch_small_widths<T, SAVED, true>(st, p) : launch_small_widths<T, SAVED, false>(st, p);
    return cols ? launch_pieces<T, SAVED, true>(st, p) : launch_pieces<T, SAVED, false>(st, p);
}

} // namespace

extern "C" int kn_grouped_linear(void *stream, const kn_linear_desc *d, const void *x, const void *w, const void *bias,
                                 const int32_t *offsets, const int32_t *rows, int32_t relu, void *y)
{
    KN_TRY(kn_linear_check(d));
    if (d->rows == 0) return KN_OK;
    if (!w || !offsets || !y || (d->x_rows > 0 && !x) || (!rows && d->x_rows < d->rows)) return KN_E_INVALID_ARG;
    KnProduct p = {};
    const bool io = d->w_layout == KN_W_IN_OUT;
    p.a = x; p.b = w; p.bias = bias; p.out = y; p.offsets = offsets; p.rows = rows;
    p.lda = d->ldx;
    p.b_group = (int64_t)d->n_in * d->n_out; p.b_c = io ? d->n_out : 1; p.b_j = io ? 1 : d->n_in;
    p.o_i = d->n_out;
    p.M = (int32_t)d->rows; p.E = d->experts; p.J = d->n_out; p.C = d->n_in;
    p.a_rows = (int32_t)d->x_rows; p.relu = relu != 0;
    return kn_with_type(d->dtype, [&](auto v) { return launch_forward<decltype(v), false>((hipStream_t)stream, p); });
}

namespace {
// The gradient of a layer's inputs; mask: of a ReLU before it (SAVED: what kn_save_f8 left of its results)
template <bool SAVED>
int linear_dx(void *stream, const kn_linear_desc *d, const void *dy, const void *w, const void *mask, const int32_t *offsets, const int32_t *rows, void *dx)
{
    if (!dy || !w || !offsets || !dx || (mask && !rows && d->x_rows < d->rows)) return KN_E_INVALID_ARG;
    KnProduct p = {};
    const bool io = d->w_layout == KN_W_IN_OUT;
    p.a = dy; p.b = w; p.mask = mask; p.out = dx; p.offsets = offsets; p.rows = nullptr;
    p.lda = d->n_out; p.ldm = SAVED ? kn_saved_bytes(d->n_in) : d->ldx;
    p.b_group = (int64_t)d->n_in * d->n_out; p.b_c = io ? 1 : d->n_in; p.b_j = io ? d->n_out : 1;
    p.o_i = d->n_in;
    p.M = (int32_t)d->rows; p.E = d->experts; p.J = d->n_in; p.C = d->n_out;
    p.a_rows = p.M; p.m_rows = (int32_t)d->x_rows;
    p.mask_rows = mask ? rows : nullptr;
    return kn_with_type(d->dtype, [&](auto v) { return launch_forward<decltype(v), SAVED>((hipStream_t)stream, p); });
}
} // namespace

extern "C" int kn_grouped_linear_dx(void *stream, const kn_linear_desc *d, const void *dy, const void *w, const void *x_relu,
                                    const int32_t *offsets, const int32_t *rows, void *dx)
{
    KN_TRY(kn_linear_check(d));
    return d->rows == 0 ? KN_OK : linear_dx<false>(stream, d, dy, w, x_relu, offsets, rows, dx);
}

extern "C" int kn_grouped_linear_dx_saved(void *stream, const kn_linear_desc *d, const void *dy, const void *w, const void *q, const int32_t *offsets,
                                          const int32_t *rows, void *dx)
{
    KN_TRY(kn_saved_check(d));
    if (d->rows == 0) return KN_OK;
    if (!q || ((uintptr_t)q & 15)) return KN_E_INVALID_ARG;
    return linear_dx<true>(stream, d, dy, w, q, offsets, rows, dx);
}
