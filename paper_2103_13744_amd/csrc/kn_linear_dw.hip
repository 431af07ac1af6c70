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
enum { SUM_NONE, SUM_A, SUM_B };
template <typename T, bool DIRECT, int BM, int BN, int WR, int WC>
__global__ void __launch_bounds__(WR * WC * 64) k_product_reduce(KnProduct p, int32_t sum, Parts parts)
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
    KnGroupLoader<T, BM, NW, DIRECT> la;
    KnGroupLoader<T, BN, NW, DIRECT> lb;
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
        la.start(wave, lane, (const T *)p.a + i0, p.lda, p.I - i0, p.rows, p.a_rows, c0, cend);
        lb.start(wave, lane, (const T *)p.b + j0, p.ldb, p.J - j0, p.b_index, p.b_rows, c0, cend);
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

// The parts' sums of the networks that have several, in the order of the parts; `chunk` results per workgroup.  SEARCH: there are at most
// M / len such networks, and a workgroup looks for its own among all (few networks of many results); else there is one for
// every network's results, and most find nothing to do.  SPLIT: each wavefront sums a quarter of a network's parts, and the quarters are added
// in order (50,560 rows of 25 networks 64 x 112, the longest of some 160 parts: 51 -> 17 us).
template <typename T, bool SEARCH, bool SPLIT> __global__ void __launch_bounds__(256) k_reduce_join(KnProduct p, int32_t sum, Parts parts, int32_t chunk)
{
    __shared__ int32_t scratch[4], found;
    __shared__ float quarter[4][64];
    const int64_t n = (int64_t)p.I * p.J;
    const int32_t pieces = (int32_t)((n + chunk - 1) / chunk), block = p.first + kn_block(), turn = block / pieces;
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
int32_t part_length(const kn_linear_desc *d)
{
    const bool whole = d->dtype == KN_F32;
    const int64_t tiles = narrow(d) ? 1 : kn_div_up(d->n_in, 128) * kn_div_up(d->n_out, 128);
    const int64_t len = kn_div_up(d->rows, kn_div_up(narrow(d) ? 1024 : whole ? 256 : 512, tiles));
    const int64_t least = narrow(d) ? 128 : whole && d->rows > 1024 ? 512 : tiles <= 8 ? 1024 : 2048;
    return (int32_t)kn_align_up(len < least ? least : len, 64);
}

template <typename T, bool DIRECT> int launch_reduce(hipStream_t st, const kn_linear_desc *d, const KnProduct &p, int32_t sum, const Parts &parts)
{
    const Way way = way_of(d, DIRECT);
    const int bm = way == WAY_128 ? 128 : way == WAY_32 || (way == WAY_SMALL && p.I <= 32) ? 32 : 64;
    const int bn = way == WAY_128 ? 128 : way == WAY_32 ? 32 : way == WAY_64 || p.J > 48 ? 64 : p.J > 32 ? 48 : p.J > 16 ? 32 : 16;
    const int64_t blocks = kn_pieces(p.M, p.E, parts.len) * kn_div_up(p.I, bm) * kn_div_up(p.J, bn);
    const int64_t each = d->rows / d->experts;
    const bool alone = way == WAY_SMALL && (each < 32 || (each < 256 && d->experts >= 1024));
    const int status = kn_launch(blocks, way == WAY_128 ? 512 : alone ? 64 : 256, [&](dim3 grid, int32_t first) {
        KnProduct q = p;
        q.first = first;
        if (way == WAY_128) {
            if constexpr (sizeof(T) == 2) hipLaunchKernelGGL((k_product_reduce<T, DIRECT, 128, 128, 2, 4>), grid, dim3(512), 0, st, q, sum, parts);
        } else if (way == WAY_64) hipLaunchKernelGGL((k_product_reduce<T, DIRECT, 64, 64, 2, 2>), grid, dim3(256), 0, st, q, sum, parts);
        else if (way == WAY_32) {
            if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((k_product_reduce<T, DIRECT, 32, 32, 2, 2>), grid, dim3(256), 0, st, q, sum, parts);
        } else if constexpr (!DIRECT) {
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
    if (p.M <= parts.len) return KN_OK; // (no network has several)
    const int64_t most = p.M / parts.len, results = (int64_t)p.I * p.J;
    const bool few = results * (most < p.E ? most : p.E) <= 1 << 20 && p.E * kn_div_up(results, 256) <= 8192;
    const int32_t chunk = few ? 256 : 4096; // (few results: more workgroups, whose wavefronts take a quarter of the parts each)
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
    if (!out_bytes) return KN_E_INVALID_ARG;
    const int32_t len = part_length(d);
    *out_bytes = d->rows <= len ? 0 : kn_align_up(part_places(d->rows, len) * ((int64_t)d->n_in * d->n_out + d->n_out) * 4, 256);
    return KN_OK;
}

extern "C" int kn_grouped_linear_dw(void *stream, const kn_linear_desc *d, const void *x, const void *dy, const int32_t *offsets,
                                    const int32_t *rows, void *dw, void *db, void *workspace, int64_t workspace_bytes)
{
    KN_TRY(kn_linear_check(d));
    if (!offsets || !dw || (d->rows > 0 && (!dy || (d->x_rows > 0 && !x))) || (d->rows > 0 && !rows && d->x_rows < d->rows)) return KN_E_INVALID_ARG;
    int64_t need = 0;
    KN_TRY(kn_grouped_linear_dw_workspace_bytes(d, &need));
    if (need > 0 && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need)) return KN_E_WORKSPACE;
    Parts parts = {part_length(d), (float *)workspace, nullptr};
    parts.bias_sums = parts.sums + part_places(d->rows, parts.len) * (int64_t)d->n_in * d->n_out;
    KnProduct p = {};
    const bool io = d->w_layout == KN_W_IN_OUT; // (columns are what is contiguous in dw)
    p.a = io ? x : dy; p.b = io ? dy : x;
    p.lda = io ? d->ldx : d->n_out; p.ldb = io ? d->n_out : d->ldx;
    p.rows = io ? rows : nullptr; p.b_index = io ? nullptr : rows;
    p.M = (int32_t)d->rows; p.E = d->experts; p.I = io ? d->n_in : d->n_out; p.J = io ? d->n_out : d->n_in;
    p.a_rows = (int32_t)(io ? d->x_rows : d->rows); p.b_rows = (int32_t)(io ? d->rows : d->x_rows);
    p.out = dw; p.out_bias = db; p.offsets = offsets;
    p.o_group = (int64_t)d->n_in * d->n_out; p.o_i = p.J;
    const int32_t sum = !db ? SUM_NONE : io ? SUM_B : SUM_A;
    return kn_with_type(d->dtype, [&](auto v) -> int {
        typedef decltype(v) E_;
        constexpr int64_t V = 16 / sizeof(E_);
        const bool direct = p.I % V == 0 && p.J % V == 0 && (((uintptr_t)p.a | (uintptr_t)p.b) & 15) == 0 && p.lda % V == 0 && p.ldb % V == 0;
        return direct ? launch_reduce<E_, true>((hipStream_t)stream, d, p, sum, parts) : launch_reduce<E_, false>((hipStream_t)stream, d, p, sum, parts);
    });
}
