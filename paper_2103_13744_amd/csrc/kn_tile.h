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

template <typename T> struct KnFrag;
template <> struct KnFrag<_Float16> { typedef kn_f16x8 Type; };
template <> struct KnFrag<__bf16> { typedef kn_bf16x8 Type; };
template <> struct KnFrag<float> { typedef kn_f32x4 Type; };

// byte in a row-wise tile
__device__ __forceinline__ int kn_row_byte(int r, int piece) { return r * 128 + ((piece ^ (r & 7)) << 4); }
// exclusive or on the piece's number in row c of a column-wise tile: 16-bit fragments read rows 8 g + 0..3 of two g at a time, 32
// bytes of each; fp32 fragments rows 4 g of four g, 64 bytes of each
template <typename T> __device__ __forceinline__ int kn_col_swizzle(int c)
{
    if constexpr (sizeof(T) == 2) return ((c & 3) | ((c >> 3 & 1) << 2)) << 1;
    else return (c >> 2 & 3) << 2;
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
        const KN_LDS char *at = tile + c * (W * 2) + ((piece ^ kn_col_swizzle<T>(c)) << 4) + (i & 1) * 8;
        union { kn_s16x4 h[2]; typename KnFrag<T>::Type v; } f;
        f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((KN_LDS kn_s16x4 *)at);
        f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((KN_LDS kn_s16x4 *)(at + 4 * W * 2)); // (the same swizzle)
        return f.v;
    } else {
        typename KnFrag<T>::Type v;
        const int c = kk * 16 + 4 * (lane >> 4), j = j0 + (lane & 15);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            v[q] = *(const KN_LDS float *)(tile + (c + q) * (W * 4) + (((j >> 2) ^ kn_col_swizzle<T>(c + q)) << 4) + (j & 3) * 4);
        return v;
    }
}

// What a wavefront fetches of each stage of a row-wise tile of R rows (NW wavefronts in the workgroup): N times 8 rows.
// row(r): address of row r's first value (any valid one for a row that does not exist: its results are not used).
template <typename T, int R, int NW> struct KnRowLoader {
    static constexpr int N = R / 8 / NW, CS = 128 / sizeof(T);
    const char *at[N];
    int piece; // this lane's piece of a row
    template <typename F> __device__ __forceinline__ void start(int wave, int lane, F &&row)
    {
        piece = (lane & 7) ^ (lane >> 3);
#pragma unroll
        for (int t = 0; t < N; ++t) at[t] = (const char *)row((wave * N + t) * 8 + (lane >> 3)) + (piece << 4);
    }
    // left: values of the contraction from this stage on; the stage's pieces behind them are zeros
    __device__ __forceinline__ void fetch(KN_LDS char *tile, int wave, int32_t left)
    {
        const bool none = left < CS && piece * 16 >= left * (int)sizeof(T);
#pragma unroll
        for (int t = 0; t < N; ++t) {
            kn_fetch(none ? (const char *)&kn_zeros : at[t], tile + (wave * N + t) * 1024);
            at[t] += 128;
        }
    }
};
// The same of a column-wise tile W wide: N times 1024 / (W sizeof(T)) rows of the contraction.  `pieces`: 16-byte pieces of a row
// that are there (from the tile's first column on); a lane behind them fetches the last one.
template <typename T, int W, int NW> struct KnColLoader {
    static constexpr int CS = 128 / sizeof(T), PR = W * sizeof(T) / 16, RP = 64 / PR, N = CS / RP / NW;
    const char *at[N];
    int64_t step;
    __device__ __forceinline__ int row(int wave, int lane, int t) const { return (wave * N + t) * RP + lane / PR; }
    __device__ __forceinline__ int piece(int wave, int lane, int t, int pieces) const
    {
        return min((lane % PR) ^ kn_col_swizzle<T>(row(wave, lane, t)), pieces - 1);
    }
    __device__ __forceinline__ void start(int wave, int lane, const T *first, int64_t stride, int pieces)
    {
        step = stride * (int64_t)sizeof(T) * CS;
#pragma unroll
        for (int t = 0; t < N; ++t) at[t] = (const char *)(first + row(wave, lane, t) * stride) + piece(wave, lane, t, pieces) * 16;
    }
    __device__ __forceinline__ void fetch(KN_LDS char *tile, int wave, int lane, int32_t left)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            kn_fetch(row(wave, lane, t) < left ? at[t] : (const char *)&kn_zeros, tile + (wave * N + t) * 1024);
            at[t] += step;
        }
    }
};

// A column-wise tile whose rows are those of one network, through an index or not: the numbers of the next stage's rows are
// asked for before this stage's values, so that they are there when that stage is fetched.
template <typename T, int W, int NW, bool INDEX> struct KnGroupLoader {
    static constexpr int CS = 128 / sizeof(T), PR = W * sizeof(T) / 16, RP = 64 / PR, N = CS / RP / NW;
    int32_t next[N];
    int at[N]; // bytes of this lane's piece in a row
    const char *base;
    const int32_t *index;
    int64_t stride;
    int32_t rows, last; // rows that there are; the network's last
    __device__ __forceinline__ int row(int wave, int lane, int t) const { return (wave * N + t) * RP + lane / PR; }
    __device__ __forceinline__ void ask(int wave, int lane, int32_t c0)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int32_t c = min(c0 + row(wave, lane, t), last);
            next[t] = INDEX ? index[c] : c;
        }
    }
    // first: the tile's first column; c0: the network's first row
    __device__ __forceinline__ void start(int wave, int lane, const T *first, int64_t ld, int pieces, const int32_t *idx, int32_t n, int32_t c0, int32_t cend)
    {
        base = (const char *)first;
        stride = ld * (int64_t)sizeof(T);
        index = idx;
        rows = n;
        last = cend - 1;
#pragma unroll
        for (int t = 0; t < N; ++t) at[t] = min((lane % PR) ^ kn_col_swizzle<T>(row(wave, lane, t)), pieces - 1) * 16;
        ask(wave, lane, c0);
    }
    __device__ __forceinline__ void fetch(KN_LDS char *tile, int wave, int lane, int32_t c0)
    {
        int32_t now[N];
#pragma unroll
        for (int t = 0; t < N; ++t) now[t] = next[t];
        ask(wave, lane, c0 + CS);
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const bool there = c0 + row(wave, lane, t) <= last && (uint32_t)now[t] < (uint32_t)rows;
            kn_fetch(there ? base + (int64_t)now[t] * stride + at[t] : (const char *)&kn_zeros, tile + (wave * N + t) * 1024);
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
