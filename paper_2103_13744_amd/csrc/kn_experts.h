// What the operators of per-row networks share (router, grouped products, weighted sum): element types, the look-up of a
// workgroup's rows among groups of ragged sizes, the description of a grouped product.
#pragma once

#include "kn_common.h"

typedef float kn_f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 kn_f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 kn_bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t kn_u32x4 __attribute__((ext_vector_type(4)));

constexpr int32_t KN_MAX_EXPERTS = 65535;
constexpr int32_t KN_MAX_WIDTH = 1 << 20;
constexpr int64_t KN_MAX_ROWS = 1ll << 30;

static inline int kn_item(int32_t dtype) { return dtype == KN_F32 ? 4 : 2; }
static inline bool kn_dtype_ok(int32_t dtype) { return dtype == KN_F32 || dtype == KN_F16 || dtype == KN_BF16; }

// Calls `f` with a value of the element type that `dtype` names (which has been checked).
template <typename F> static inline int kn_with_type(int32_t dtype, F &&f)
{
    if (dtype == KN_F32) return f(float());
    if (dtype == KN_F16) return f((_Float16)0);
    return f((__bf16)0.0f);
}

// Calls f(workgroups, number of the first) for so many workgroups.  A launch holds less than 2^32 threads: the runtime takes more without a
// word and runs what is left of them modulo 2^32.  (Launches begin at a multiple of eight: a workgroup's XCD goes by its number.)
template <typename F> static inline int kn_launch(int64_t blocks, int threads, F &&f)
{
    if (blocks > 0x7fffffffLL) return KN_E_UNSUPPORTED;
    const int64_t most = (0xffffffffLL / threads) & ~7LL;
    for (int64_t first = 0; first < blocks; first += most) {
        f(dim3((unsigned)(blocks - first < most ? blocks - first : most)), (int32_t)first);
        KN_CHECK_LAUNCH();
    }
    return KN_OK;
}

// Largest value among the 16 lanes of a row of the wavefront, in all of them: rotations inside the row.
__device__ __forceinline__ float kn_row_max(float v)
{
    constexpr int ROW_ROR = 0x120; // dpp_ctrl encoding
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 8, 0xf, 0xf, true)));
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 4, 0xf, 0xf, true)));
    v = fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 2, 0xf, 0xf, true)));
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ROW_ROR + 1, 0xf, 0xf, true)));
}

// Between what a wavefront's lanes write to the LDS and what others of its lanes read there, and before that place is written again.  The
// hardware keeps a wavefront's accesses in order; this holds the compiler to it.  No instruction comes of it.
__device__ __forceinline__ void kn_lanes_meet() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// Rows of one network among the sorted rows: where a workgroup's piece lies.
struct KnPiece {
    int32_t group;   // the network, or E: rows of no network
    int32_t begin;   // first row of the piece
    int32_t end;     // end of the group's rows (begin >= end: nothing to do)
};

// offsets[e] as far as it can be used: callers' arrays are not looked at on the host
__device__ __forceinline__ int32_t kn_offset(const int32_t *__restrict__ offsets, int32_t e, int32_t M)
{
    return min(max(offsets[e], 0), M);
}

// Group e gets the pieces of `len` rows numbered from offsets[e] / len + e on: these first numbers grow strictly with e and
// leave every group room for all its pieces, so a workgroup finds its group by a search in the offsets alone, with no list
// of pieces to be made before.  64 offsets a step, one per lane: one step for up to 64 groups, three for 65,535.
// Piece numbers run from 0 to M / len + E (the last group, E, is that of the rows without a network).
__device__ __forceinline__ KnPiece kn_find_piece(const int32_t *__restrict__ offsets, int32_t E, int32_t M, int32_t len, int32_t number)
{
    const int lane = kn_thread() & (KN_WAVE - 1);
    int32_t lo = 0, n = E + 1; // the group lies in [lo, lo + n)
    while (n > 1) {
        const int32_t step = (n + KN_WAVE - 1) / KN_WAVE;
        const int32_t e = lo + lane * step;
        const bool there = lane * step < n;
        const bool upto = there && kn_offset(offsets, min(e, E), M) / len + e <= number;
        const int32_t hits = __popcll(__ballot(upto)); // (the first is always one: number >= first number of lo)
        const int32_t at = max(hits, 1) - 1;
        lo += at * step;
        n = min(step, n - at * step);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const int32_t o = kn_offset(offsets, lo, M);
    KnPiece p;
    p.group = lo;
    const int32_t first = o / len + lo;
    p.end = lo < E ? kn_offset(offsets, lo + 1, M) : M;
    p.begin = number >= first ? o + (number - first) * len : p.end; // (always, where offsets start at 0 and do not fall)
    return p;
}
static inline int64_t kn_pieces(int64_t M, int64_t E, int64_t len) { return M / len + E + 1; }

// 16 x 16 products of fragments of 8 values a lane: lane l holds row (or column) l % 16 and the contraction's 8 (l / 16) .. + 7
// of 32; results: column l % 16, rows 4 (l / 16) .. + 3.
__device__ __forceinline__ kn_f32x4 kn_mfma(kn_f16x8 a, kn_f16x8 b, kn_f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ kn_f32x4 kn_mfma(kn_bf16x8 a, kn_bf16x8 b, kn_f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
// the same for 4 values a lane of fp32: four products over 4 each, contraction 4 (l / 16) + j in the order j = 0 .. 3.  The 16 terms
// are summed by themselves and then added: a long sum rounds at its own size once per 16 terms.
__device__ __forceinline__ kn_f32x4 kn_mfma(kn_f32x4 a, kn_f32x4 b, kn_f32x4 c)
{
    kn_f32x4 sum = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], sum, 0, 0, 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] += sum[j];
    return c;
}

// A grouped product as the kernels see it.
//   forward:         out(i, j) = sum over c of a(i, c) b_e(c, j), a = x (rows through `rows`), b_e = w[e], out = y, c < K
//   input gradient:  the same with a = dy, b_e = w[e] transposed, out = dx, c < N
//   weight gradient: out_e(i, j) = sum over the network's rows r of a(r, i) b(r, j), a = x (rows through `rows`), b = dy
struct KnProduct {
    const void *a, *b, *bias, *mask; // mask: out(i, j) becomes 0 where mask(row i, j) <= 0 (a ReLU's result)
    void *out, *out_bias;            // out_bias (weight gradient): sum over the rows r of b(r, j)
    const int32_t *offsets, *rows, *b_index, *mask_rows; // rows: of a, b_index: of b, mask_rows: of the mask; nullable
    int64_t lda, ldb, ldm;           // row strides in elements: a, b (weight gradient), mask
    int64_t b_group, b_c, b_j;       // strides of b_e: network, contraction, column
    int64_t o_group, o_i;            // strides of out: network (weight gradient), row (columns are neighbours)
    int32_t M, E, I, J, C;           // rows, networks; weight gradient: rows of out_e; columns of out; contraction
    int32_t a_rows, b_rows, m_rows;  // rows that a, b (weight gradient) and the mask have (an index outside is a row of zeros)
    int32_t relu;
    int32_t first;                   // number of the launch's first workgroup
};

// What kn_save_f8 leaves of K values of a row
constexpr int KN_SAVED_BLOCK = 128;
static inline int64_t kn_saved_bytes(int64_t K) { return kn_align_up(K, 16); }

// kn_grouped_linear_dw, with rows of dy that may lie apart; exponents: x is what kn_save_f8 left
int kn_linear_dw_run(void *stream, const kn_linear_desc *d, const void *x, const uint8_t *exponents, const void *dy, int64_t lddy, const int32_t *offsets, const int32_t *rows,
                     void *dw, void *db, void *workspace, int64_t workspace_bytes);
// Workspace of one of the two below (low_rank: whatever kernel it is)
int kn_linear_dw_bytes(const kn_linear_desc *d, bool low_rank, int64_t *out_bytes);
// The gradients of a low-rank product's factors, as layers of their own: a (n_in, rank) from x and g, b (rank, n_out) from h and dy
int kn_linear_dw_low_rank(void *stream, const kn_linear_desc *da, const void *x, const void *g, int64_t ldg, const int32_t *rows, void *out_a, const kn_linear_desc *db,
                          const void *h, const void *dy, int64_t lddy, void *out_b, const int32_t *offsets, void *workspace, int64_t workspace_bytes);

// What the grouped products check alike
static inline int kn_linear_check(const kn_linear_desc *d)
{
    if (!d || d->rows < 0 || d->x_rows < 0 || d->experts < 1 || d->n_in < 1 || d->n_out < 1 || !kn_dtype_ok(d->dtype) ||
        (d->w_layout != KN_W_IN_OUT && d->w_layout != KN_W_OUT_IN) || d->ldx < d->n_in)
        return KN_E_INVALID_ARG;
    if (d->rows > KN_MAX_ROWS || d->x_rows > KN_MAX_ROWS || d->experts > KN_MAX_EXPERTS || d->n_in > KN_MAX_WIDTH || d->n_out > KN_MAX_WIDTH)
        return KN_E_UNSUPPORTED;
    return KN_OK;
}
// ldx is not looked at where x is what kn_save_f8 left
static inline int kn_saved_check(const kn_linear_desc *d)
{
    if (!d) return KN_E_INVALID_ARG;
    kn_linear_desc whole = *d;
    whole.ldx = d->n_in;
    return kn_linear_check(&whole);
}

