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

#include <type_traits>

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

template <typename T> struct KnSmallFrag {
    static constexpr int W = 16 / sizeof(T), KS = 4 * W;
};
// kn_any_piece in two parts, so that nothing waits for a fetch before all are under way: a piece that ends behind the row is fetched from
// its last 16 bytes, and shifted to its place at the end.  `odd`: 16-bit rows may begin between two words, where a fetch of 16 bytes is
// several times as slow: the words that the piece lies in are fetched (five; each holds a value of the piece, so that no more than the other
// half of a word of the row's is read beside it, and shifted out) and joined at the end
// (524,291 rows, 4,096 networks 63 x 32 in bf16: 50 -> 40 us, with weights whose rows are 63 values 60 -> 35).
template <typename T> __device__ __forceinline__ typename KnFrag<T>::Type kn_row_ask(const T *row, int32_t k, int32_t C, bool odd, uint32_t &fifth)
{
    constexpr int W = KnSmallFrag<T>::W;
    if (C < W) return kn_any_piece<T>(row, k, C);
    typename KnFrag<T>::Type f = {};
    fifth = 0;
    if (k < C) {
        const T *at = row + min(k, C - W);
        if (sizeof(T) == 2 && odd) {
            const uintptr_t word = ~(uintptr_t)3;
            f = *(const typename KnAny<T>::Words *)((uintptr_t)at & word);
            fifth = *(const uint32_t *)(((uintptr_t)at + 14) & word);
        } else {
            f = *(const typename KnAny<T>::Piece *)at;
        }
    }
    return f;
}
template <typename T>
__device__ __forceinline__ void kn_row_place(typename KnFrag<T>::Type &f, const T *row, int32_t k, int32_t C, bool odd, uint32_t fifth)
{
    constexpr int W = KnSmallFrag<T>::W;
    kn_u32x4 d = __builtin_bit_cast(kn_u32x4, f);
    if (sizeof(T) == 2 && odd) {
        const uint32_t low = (uint32_t)(uintptr_t)(row + min(k, C - W)) & 2;
        d = kn_u32x4{__builtin_amdgcn_alignbyte(d[1], d[0], low), __builtin_amdgcn_alignbyte(d[2], d[1], low), __builtin_amdgcn_alignbyte(d[3], d[2], low),
                     __builtin_amdgcn_alignbyte(fifth, d[3], low)};
    }
    const kn_u32x4 whole = d;
    const int bytes = (W - C % W) % W * (int)sizeof(T); // alike for all lanes
    if (bytes & 2) d = kn_u32x4{d[0] >> 16 | d[1] << 16, d[1] >> 16 | d[2] << 16, d[2] >> 16 | d[3] << 16, d[3] >> 16};
    if (bytes & 4) d = kn_u32x4{d[1], d[2], d[3], 0};
    if (bytes & 8) d = kn_u32x4{d[2], d[3], 0, 0};
    f = __builtin_bit_cast(typename KnFrag<T>::Type, k < C && k + W > C ? d : whole);
}
// 32 rows of 16 V values of 16 bits in an LDS that one wavefront has for itself, to be read column by column: where row r and its piece lie, so that the 4 x 4 rows
// of a transposing read are spread over all banks.
template <int V> __device__ __forceinline__ int kn_turned_byte(int r, int piece)
{
    if constexpr (V == 1) return (r ^ (r >> 3 & 1) << 2) * 32 + piece * 16;
    else if constexpr (V == 2) return r * 64 + (piece ^ (r >> 3 & 1) << 1) * 16;
    else return r * 128 + (piece ^ ((r >> 1 & 1) | (r >> 3 & 1) << 1) << 1) * 16;
}
// Column 16 v + l % 16 of rows 8 (l / 16) .. + 7
template <int V> __device__ __forceinline__ kn_f16x8 kn_turned_frag(KN_LDS char *turn, int v, int lane)
{
    const int g = lane >> 4, i = lane & 15;
    union { kn_s16x4 h[2]; kn_f16x8 f; } t;
#pragma unroll
    for (int h = 0; h < 2; ++h)
        t.h[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((KN_LDS kn_s16x4 *)(turn + kn_turned_byte<V>(8 * g + 4 * h + (i >> 2), 2 * v + (i >> 1 & 1)) + (i & 1) * 8));
    return t.f;
}

// What is added to columns j .. j + 7 of a network's results (j a multiple of 8)
template <typename T> __device__ __forceinline__ void kn_bias_of(const KnProduct &p, bool some, int64_t group, int32_t j, float add[8])
{
    const bool any = p.bias && some && j < p.J;
    typename KnEight<T>::Piece v = {};
    if (any) v = KnEight<T>::load((const T *)p.bias + group * p.J, j, p.J);
#pragma unroll
    for (int q = 0; q < 8; ++q) add[q] = any ? (float)v[q] : 0.0f;
}
// The end of 8 neighbouring results of row i: zeros for a row that x does not have, bias, ReLU, the mask of a ReLU before (SAVED: from what kn_save_f8 left, where a
// positive byte is a positive value, in rows of ldm bytes); one rounding
template <typename T, bool SAVED = false>
__device__ __forceinline__ void kn_finish(const KnProduct &p, bool some, int32_t i, int32_t j, const float add[8], float y[8])
{
    if (p.rows && (uint32_t)p.rows[i] >= (uint32_t)p.a_rows) {
#pragma unroll
        for (int q = 0; q < 8; ++q) y[q] = 0.0f;
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        y[q] += add[q];
        if (p.relu) y[q] = y[q] > 0.0f || y[q] != y[q] ? y[q] : 0.0f; // (a NaN stays one)
    }
    if (p.mask && some) {
        const int32_t src = p.mask_rows ? p.mask_rows[i] : i;
        const bool in = (uint32_t)src < (uint32_t)p.m_rows;
        if constexpr (SAVED) { // (j is a multiple of eight, and saved rows are of whole 16 bytes)
            typedef int8_t Eight __attribute__((ext_vector_type(8)));
            Eight m = {};
            if (in) m = *(const Eight *)((const int8_t *)p.mask + (int64_t)src * p.ldm + j);
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (m[q] <= 0) y[q] = 0.0f;
        } else {
            typename KnEight<T>::Piece m = {};
            if (in) m = KnEight<T>::load((const T *)p.mask + (int64_t)src * p.ldm, j, p.J);
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (!((float)m[q] > 0.0f)) y[q] = 0.0f;
        }
    }
    typename KnEight<T>::Piece o;
#pragma unroll
    for (int q = 0; q < 8; ++q) o[q] = (T)y[q];
    KnEight<T>::store((T *)p.out + (int64_t)i * p.o_i, j, p.J, o);
}

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

// Four values of 8 bits times a power of two, in T: exact in bf16 and fp32, and in fp16 where the values came from there
template <typename T> __device__ __forceinline__ void kn_widen_saved(uint32_t v, float power, T to[4])
{
    if constexpr (std::is_same<T, __bf16>::value) {
        const auto a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, power, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v, power, true);
        to[0] = a[0]; to[1] = a[1]; to[2] = b[0]; to[3] = b[1];
    } else if constexpr (std::is_same<T, _Float16>::value) {
        const auto a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, power, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(v, power, true);
        to[0] = a[0]; to[1] = a[1]; to[2] = b[0]; to[3] = b[1];
    } else {
        const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v, power, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(v, power, true);
        to[0] = a[0]; to[1] = a[1]; to[2] = b[0]; to[3] = b[1];
    }
}
__device__ __forceinline__ float kn_power(uint8_t exponent) { return __int_as_float((int)exponent << 23); }

// KnGroupLoader for rows that kn_save_f8 left, widened on their way through the registers.  Values and exponents of a stage are asked for a stage before they
// are put down, the numbers of its rows two.
template <typename T, int W, int NW> struct KnSavedLoader {
    static constexpr int CS = 128 / sizeof(T), PW = 16 / sizeof(T), PR = W / PW, RP = 64 / PR, N = CS / RP / NW;
    int32_t next[N];
    uint32_t held[N][PW / 4];
    uint8_t power[N];
    const uint8_t *base, *exponents;
    const int32_t *index;
    int64_t stride;
    int32_t rows, last, columns, blocks;
    __device__ __forceinline__ int row(int wave, int lane, int t) const { return (wave * N + t) * RP + lane / PR; }
    __device__ __forceinline__ int first_column(int wave, int lane, int t) const { return ((lane % PR) ^ kn_col_swizzle<T, W>(row(wave, lane, t))) * PW; }
    __device__ __forceinline__ void ask_rows(int wave, int lane, int32_t c0)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int32_t c = min(c0 + row(wave, lane, t), last);
            next[t] = index ? index[c] : c;
        }
    }
    // first: column of the tile's first value, of `width` in a row
    __device__ __forceinline__ void start(int wave, int lane, const uint8_t *q, const uint8_t *exps, int32_t first, int32_t width, const int32_t *idx, int32_t n_rows,
                                          int32_t c0, int32_t cend)
    {
        stride = (width + 15) & ~15;
        blocks = (width + KN_SAVED_BLOCK - 1) / KN_SAVED_BLOCK;
        base = q + first;
        exponents = exps + first / KN_SAVED_BLOCK; // (a tile is no wider than a block, and lies in one)
        columns = (int32_t)stride - first;
        index = idx;
        rows = n_rows;
        last = cend - 1;
        ask_rows(wave, lane, c0);
        ask(wave, lane, c0);
    }
    __device__ __forceinline__ void ask(int wave, int lane, int32_t c0)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const int k = first_column(wave, lane, t);
            const bool there = c0 + row(wave, lane, t) <= last && (uint32_t)next[t] < (uint32_t)rows && k < columns;
#pragma unroll
            for (int q = 0; q < PW / 4; ++q) held[t][q] = 0;
            power[t] = 0;
            if (there) {
                const uint32_t *v = (const uint32_t *)(base + next[t] * stride + k);
#pragma unroll
                for (int q = 0; q < PW / 4; ++q) held[t][q] = v[q];
                power[t] = exponents[(int64_t)next[t] * blocks];
            }
        }
        ask_rows(wave, lane, c0 + CS);
    }
    // the stage whose first row is c0
    __device__ __forceinline__ void fetch(KN_LDS char *tile, int wave, int lane, int32_t c0)
    {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            union { T v[PW]; typename KnFrag<T>::Type f; } wide;
#pragma unroll
            for (int q = 0; q < PW / 4; ++q) kn_widen_saved<T>(held[t][q], kn_power(power[t]), wide.v + 4 * q);
            *(KN_LDS typename KnFrag<T>::Type *)(tile + (wave * N + t) * 1024 + lane * 16) = wide.f;
        }
        if (c0 + CS <= last) ask(wave, lane, c0 + CS);
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
