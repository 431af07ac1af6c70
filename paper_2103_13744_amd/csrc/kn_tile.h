// Tiles of a product in the LDS: how they get there (16 bytes a lane, straight from memory), how they lie, how fragments are read.
//
// A stage holds 128 bytes of the contraction (64 values of 16 bits, 32 of fp32) of every row or column of the workgroup's tile.
//  - rows: the contraction is contiguous in memory.  A row is 128 bytes, its 16-byte piece c lies at c ^ (r & 7): the 16 rows of a
//    fragment read the same piece from all banks.
//  - columns: the tile's other index is contiguous in memory.  Row c of the contraction holds W values, W * sizeof(T) bytes;
//    pieces of 16 bytes are moved by an exclusive or with bits of c, so that the rows of a fragment lie in different banks.  16-bit
//    fragments are read with the transposing LDS read (4 x 16 values per 16 lanes), fp32 ones value by value.
#pragma once

#include "kn_experts.h"

#define KN_LDS __attribute__((address_space(3)))
#define KN_GLOBAL __attribute__((address_space(1)))

// 16 bytes of zeros: what lanes fetch whose piece lies outside
static __device__ const kn_u32x4 kn_zeros = {0, 0, 0, 0};

// 64 lanes x 16 bytes from each lane's address to 1 KiB of the LDS at `lds` (the same in all lanes)
__device__ __forceinline__ void kn_fetch(const void *src, KN_LDS char *lds)
{
    __builtin_amdgcn_global_load_lds((const KN_GLOBAL uint32_t *)src, (KN_LDS uint32_t *)lds, 16, 0, 0);
}

template <typename T> struct KnFrag; // 16 bytes of values
template <> struct KnFrag<uint8_t> { typedef kn_u32x4 Type; };
template <> struct KnFrag<_Float16> { typedef kn_f16x8 Type; };
template <> struct KnFrag<__bf16> { typedef kn_bf16x8 Type; };
template <> struct KnFrag<float> { typedef kn_f32x4 Type; };

// byte in a row-wise tile
__device__ __forceinline__ int kn_row_byte(int r, int piece) { return r * 128 + ((piece ^ (r & 7)) << 4); }
// exclusive or on the piece's number in row c of a column-wise tile W wide: 16-bit fragments read rows 8 g + 0..3 of two g at a time,
// 32 bytes of each (rows of 128 bytes lie two to a line of the banks); fp32 fragments rows 4 g of four g, 64 bytes of each
template <typename T, int W> __device__ __forceinline__ int kn_col_swizzle(int c)
{
    if constexpr (sizeof(T) == 4) return (c >> 2 & (W == 32 ? 1 : 3)) << 2;
    else if constexpr (W == 64) return ((c >> 1 & 1) | (c >> 3 & 1) << 1) << 1;
    else return ((c & 3) | (c >> 3 & 1) << 2) << 1;
}

typedef short kn_s16x4 __attribute__((ext_vector_type(4)));

// Fragment kk (of two) of the 16 rows from r0 on (r0 a multiple of 16) in a row-wise tile
template <typename T> __device__ __forceinline__ typename KnFrag<T>::Type kn_row_frag(const KN_LDS char *tile, int r0, int kk, int lane)
{
    const int r = r0 + (lane & 15);
    return *(const KN_LDS typename KnFrag<T>::Type *)(tile + kn_row_byte(r, kk * 4 + (lane >> 4)));
}
// the same of the 16 columns from j0 on in a column-wise tile W wide
template <typename T, int W> __device__ __forceinline__ typename KnFrag<T>::Type kn_col_frag(const KN_LDS char *__restrict tile, int j0, int kk, int lane)
{
    if constexpr (sizeof(T) == 2) {
        const int g = lane >> 4, i = lane & 15, c = kk * 32 + 8 * g + (i >> 2);
        const int piece = (j0 >> 3) + (i >> 1 & 1);
        const KN_LDS char *at = tile + c * (W * 2) + ((piece ^ kn_col_swizzle<T, W>(c)) << 4) + (i & 1) * 8;
        union { kn_s16x4 h[2]; typename KnFrag<T>::Type v; } f;
        f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((KN_LDS kn_s16x4 *)at);
        f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((KN_LDS kn_s16x4 *)(at + 4 * W * 2)); // (the same swizzle)
        return f.v;
    } else {
        typename KnFrag<T>::Type v;
        const int c = kk * 16 + 4 * (lane >> 4), j = j0 + (lane & 15);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            v[q] = *(const KN_LDS float *)(tile + (c + q) * (W * 4) + (((j >> 2) ^ kn_col_swizzle<T, W>(c + q)) << 4) + (j & 3) * 4);
        return v;
    }
}

// Values k .. k + W - 1 of a row of C wherever it lies, W = 16 bytes' worth; zeros behind its end.  k is a multiple of W.
template <typename T> struct KnAny {
    typedef T Piece __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
    typedef T Words __attribute__((ext_vector_type(16 / sizeof(T)), aligned(4)));
};
template <typename T> __device__ __forceinline__ typename KnFrag<T>::Type kn_any_piece(const T *row, int32_t k, int32_t C)
{
    constexpr int W = 16 / sizeof(T);
    typename KnFrag<T>::Type f;
    if (k + W <= C) {
        f = *(const typename KnAny<T>::Piece *)(row + k);
    } else {
        f = typename KnFrag<T>::Type{};
        if (k < C)
#pragma unroll
            for (int q = 0; q < W; ++q) {
                const T v = row[min(k + q, C - 1)];
                f[q] = k + q < C ? v : (T)0.0f;
            }
    }
    return f;
}

// Eight neighbouring values of a row of J from j on, wherever they lie (behind its end: the last one / nothing)
template <typename T> struct KnEight {
    typedef T Piece __attribute__((ext_vector_type(8), aligned(sizeof(T))));
    static __device__ __forceinline__ Piece load(const T *row, int32_t j, int32_t J)
    {
        Piece f;
        if (j + 8 <= J) f = *(const Piece *)(row + j);
        else
#pragma unroll
            for (int q = 0; q < 8; ++q) f[q] = row[min(j + q, J - 1)];
        return f;
    }
    static __device__ __forceinline__ void store(T *row, int32_t j, int32_t J, Piece f)
    {
        if (j + 8 <= J) *(Piece *)(row + j) = f;
        else
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (j + q < J) row[j + q] = f[q];
    }
};

// What a wavefront brings of each stage of a tile (NW wavefronts in the workgroup).  DIRECT: rows are made of whole 16-byte pieces on
// multiples of 16 bytes, which go straight from memory to the LDS.  Else pieces that start anywhere and may end inside go through
// registers: `fetch` puts down the stage that is there and asks for the one after it, so that `ask_first` comes before the first.
//
// A row-wise tile of R rows: N times 8 rows.  row(r): where row r begins (a row that does not exist: any valid one, its results
// are not used).
template <typename T, int R, int NW, bool DIRECT> struct KnRowLoader {
    static constexpr int N = R / 8 / NW, CS = 128 / sizeof(T), W = 16 / sizeof(T);
    const T *at[N];
    typename KnFrag<T>::Type held[DIRECT ? 1 : N];
    int piece; // this lane's piece of a row
    template <typename F> __device__ __forceinline__ void start(int wave, int lane, F &&row)
    {
        piece = (lane & 7) ^ (lane >> 3);
#pragma unroll
        for (int t = 0; t < N; ++t) at[t] = row((wave * N + t) * 8 + (lane >> 3)) + (DIRECT ? piece * W : 0);
    }
    // left: values of the contraction from the stage on; what lies behind them becomes zeros
    __device__ __forceinline__ void ask(int32_t left)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            held[t] = typename KnFrag<T>::Type{};
            if (piece * W < left) held[t] = kn_any_piece(at[t], piece * W, left);
            at[t] += CS;
        }
    }
    __device__ __forceinline__ void ask_first(int32_t left) { if constexpr (!DIRECT) ask(left); }
    __device__ __forceinline__ void fetch(KN_LDS char *tile, int wave, int lane, int32_t left)
    {
        if constexpr (DIRECT) {
            const bool none = left < CS && piece * W >= left;
#pragma unroll
            for (int t = 0; t < N; ++t) {
                kn_fetch(none ? (const void *)&kn_zeros : at[t], tile + (wave * N + t) * 1024);
                at[t] += CS;
            }
        } else {
#pragma unroll
            for (int t = 0; t < N; ++t) *(KN_LDS typename KnFrag<T>::Type *)(tile + (wave * N + t) * 1024 + lane * 16) = held[t];
            if (left > CS) ask(left - CS);
        }
    }
};
// A column-wise tile W wide: N times 1024 / (W sizeof(T)) rows of the contraction, `stride` values apart; `columns`: those that are
// there from the tile's first on.  (DIRECT: a lane behind them fetches the last whole piece.)
template <typename T, int W, int NW, bool DIRECT> struct KnColLoader {
    static constexpr int CS = 128 / sizeof(T), PW = 16 / sizeof(T), PR = W / PW, RP = 64 / PR, N = CS / RP / NW;
    const T *at[N];
    typename KnFrag<T>::Type held[DIRECT ? 1 : N];
    int64_t step;
    int32_t columns;
    __device__ __forceinline__ int row(int wave, int lane, int t) const { return (wave * N + t) * RP + lane / PR; }
    __device__ __forceinline__ int first_column(int wave, int lane, int t) const
    {
        const int k = ((lane % PR) ^ kn_col_swizzle<T, W>(row(wave, lane, t))) * PW;
        return DIRECT ? min(k, columns - PW) : k;
    }
    __device__ __forceinline__ void start(int wave, int lane, const T *first, int64_t stride, int32_t n)
    {
        columns = n;
        step = stride * CS;
#pragma unroll
        for (int t = 0; t < N; ++t) at[t] = first + row(wave, lane, t) * stride + (DIRECT ? first_column(wave, lane, t) : 0);
    }
    __device__ __forceinline__ void ask(int wave, int lane, int32_t left)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int k = first_column(wave, lane, t);
            held[t] = typename KnFrag<T>::Type{};
            if (row(wave, lane, t) < left && k < columns) held[t] = kn_any_piece(at[t], k, columns);
            at[t] += step;
        }
    }
    __device__ __forceinline__ void ask_first(int wave, int lane, int32_t left) { if constexpr (!DIRECT) ask(wave, lane, left); }
    __device__ __forceinline__ void fetch(KN_LDS char *tile, int wave, int lane, int32_t left)
    {
        if constexpr (DIRECT) {
#pragma unroll
            for (int t = 0; t < N; ++t) {
                kn_fetch(row(wave, lane, t) < left ? (const void *)at[t] : (const void *)&kn_zeros, tile + (wave * N + t) * 1024);
                at[t] += step;
            }
        } else {
#pragma unroll
            for (int t = 0; t < N; ++t) *(KN_LDS typename KnFrag<T>::Type *)(tile + (wave * N + t) * 1024 + lane * 16) = held[t];
            if (left > CS) ask(wave, lane, left - CS);
        }
    }
};
// A column-wise tile whose rows are rows c0 .. last of a matrix of `rows`, through an index or (nullptr) not; the numbers of a
// stage's rows are asked for a stage before its values.
template <typename T, int W, int NW, bool DIRECT> struct KnGroupLoader {
    static constexpr int CS = 128 / sizeof(T), PW = 16 / sizeof(T), PR = W / PW, RP = 64 / PR, N = CS / RP / NW;
    int32_t next[N];
    typename KnFrag<T>::Type held[DIRECT ? 1 : N];
    const T *base;
    const int32_t *index;
    int64_t stride;
    int32_t rows, last, columns;
    __device__ __forceinline__ int row(int wave, int lane, int t) const { return (wave * N + t) * RP + lane / PR; }
    __device__ __forceinline__ int first_column(int wave, int lane, int t) const
    {
        const int k = ((lane % PR) ^ kn_col_swizzle<T, W>(row(wave, lane, t))) * PW;
        return DIRECT ? min(k, columns - PW) : k;
    }
    __device__ __forceinline__ void ask_rows(int wave, int lane, int32_t c0)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int32_t c = min(c0 + row(wave, lane, t), last);
            next[t] = index ? index[c] : c;
        }
    }
    __device__ __forceinline__ void start(int wave, int lane, const T *first, int64_t ld, int32_t n_columns, const int32_t *idx, int32_t n_rows, int32_t c0,
                                          int32_t cend)
    {
        base = first;
        stride = ld;
        index = idx;
        rows = n_rows;
        last = cend - 1;
        columns = n_columns;
        ask_rows(wave, lane, c0);
        if constexpr (!DIRECT) ask(wave, lane, c0);
    }
    __device__ __forceinline__ void ask(int wave, int lane, int32_t c0)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int k = first_column(wave, lane, t);
            const bool there = c0 + row(wave, lane, t) <= last && (uint32_t)next[t] < (uint32_t)rows && k < columns;
            held[t] = typename KnFrag<T>::Type{};
            if (there) held[t] = kn_any_piece(base + next[t] * stride, k, columns);
        }
        ask_rows(wave, lane, c0 + CS);
    }
    // the stage whose first row is c0
    __device__ __forceinline__ void fetch(KN_LDS char *tile, int wave, int lane, int32_t c0)
    {
        if constexpr (DIRECT) {
            int32_t now[N];
#pragma unroll
            for (int t = 0; t < N; ++t) now[t] = next[t];
            ask_rows(wave, lane, c0 + CS);
#pragma unroll
            for (int t = 0; t < N; ++t) {
                const bool there = c0 + row(wave, lane, t) <= last && (uint32_t)now[t] < (uint32_t)rows;
                kn_fetch(there ? (const void *)(base + now[t] * stride + first_column(wave, lane, t)) : (const void *)&kn_zeros, tile + (wave * N + t) * 1024);
            }
        } else {
#pragma unroll
            for (int t = 0; t < N; ++t) *(KN_LDS typename KnFrag<T>::Type *)(tile + (wave * N + t) * 1024 + lane * 16) = held[t];
            if (c0 + CS <= last) ask(wave, lane, c0 + CS);
        }
    }
};

// Between two stages: what this wavefront asked for has arrived in the LDS, what it read there has arrived in registers, and so for every
// wavefront of the workgroup.  The buffer read before may be fetched into again, the one fetched may be read.
// LATER: so many of the loads that this wavefront asked for last need not have arrived.
template <int LATER = 0> __device__ __forceinline__ void kn_stage_barrier()
{
    static_assert(LATER < 64, "");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((LATER & 15) | (LATER >> 4) << 14 | 7 << 4); // vmcnt(LATER), lgkmcnt(0); expcnt is not waited for
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Order of the instructions since the last such mark: the fragments' reads spread among the products.
template <int U, int V, typename T, bool COLS_B, bool COLS_A = false> __device__ __forceinline__ void kn_interleave()
{
    constexpr int PER_COL = sizeof(T) == 2 ? 2 : 4, READS = U * (COLS_A ? PER_COL : 1) + V * (COLS_B ? PER_COL : 1);
    constexpr int PRODUCTS = U * V * (sizeof(T) == 2 ? 1 : 4), EACH = PRODUCTS / READS > 0 ? PRODUCTS / READS : 1;
    __builtin_amdgcn_sched_group_barrier(0x008, EACH, 0); // (a product first: what it waits for is not asked for behind a new read)
#pragma unroll
    for (int i = 0; i < READS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0); // an LDS read
        __builtin_amdgcn_sched_group_barrier(0x008, EACH, 0); // products
    }
}

// A workgroup's number such that those of one XCD (every eighth) are neighbours and share what they read in its L2
__device__ __forceinline__ int32_t kn_xcd_order(int32_t b, int32_t n)
{
    const int32_t each = n >> 3, more = n & 7, x = b & 7;
    return x * each + min(x, more) + (b >> 3);
}
