// Rows of 32- or 16-bit numbers, as the training step's kernels read and write them: numbers are worked on in 32 bits and rounded
// once, to the nearest (halves to even), where a 16-bit result is stored.
#pragma once

#include "rg_internal.h"

// Rows start where their stride puts them, so vectors are declared with their elements' alignment only: the device's memory
// instructions take 16 bytes from any element's address.
template <typename T, int N> struct RgPack;
template <int N> struct RgPack<float, N> { typedef float type __attribute__((ext_vector_type(N), aligned(4))); };
template <int N> struct RgPack<__bf16, N> { typedef __bf16 type __attribute__((ext_vector_type(N), aligned(2))); };
template <int N> struct RgPack<_Float16, N> { typedef _Float16 type __attribute__((ext_vector_type(N), aligned(2))); };
typedef uint32_t rg_u32x4 __attribute__((ext_vector_type(4), aligned(4)));

// The first `live` numbers of N from p as they are, the others 0.  (Where not all are there, loads of the last one stand in for those that are
// not, so that none waits for another.)
template <int N, typename T>
__device__ __forceinline__ typename RgPack<T, N>::type rg_load_raw(const T* p, int live) {
    if (live >= N) return *(const typename RgPack<T, N>::type*)p;
    typename RgPack<T, N>::type a;
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = (T)0.0f;
    if (live > 0) {
        T v[N];
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = p[i < live ? i : live - 1];
#pragma unroll
        for (int i = 0; i < N; ++i) a[i] = i < live ? v[i] : (T)0.0f;
    }
    return a;
}

// The same, in 32 bits.
template <int N, typename T>
__device__ __forceinline__ void rg_load_head(const T* p, int live, float (&v)[N]) {
    const typename RgPack<T, N>::type a = rg_load_raw<N>(p, live);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (float)a[i];
}

// Numbers col .. col + N - 1 of a row of `dim` >= N by one load without a branch: where the row ends before them they are loaded from further left,
// and rg_row_end puts them (those behind the end as 0) in place once they are there.
template <int N, typename T>
__device__ __forceinline__ typename RgPack<T, N>::type rg_load_row(const T* row, int col, int dim) {
    return *(const typename RgPack<T, N>::type*)(row + min(col, dim - N));
}
template <int N, typename T>
__device__ __forceinline__ void rg_row_end(T (&a)[N], int col, int dim) {
    const int over = col - min(col, dim - N);
    if (dim % N != 0) {                                    // (rows of whole vectors: all there, or none)
#pragma unroll
        for (int step = 1; step < N; step *= 2)
#pragma unroll
            for (int i = 0; i < N; ++i) a[i] = over & step ? (i + step < N ? a[(i + step) % N] : (T)0.0f) : a[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) a[i] = over < N ? a[i] : (T)0.0f;
}

// N numbers to p; ONCE: past the caches (see rg_store_once).
template <int N, bool ONCE = false, typename T>
__device__ __forceinline__ void rg_store(T* p, const float (&v)[N]) {
    constexpr int H = sizeof(T) * N <= 16 ? N : 16 / (int)sizeof(T);
#pragma unroll
    for (int h = 0; h < N / H; ++h) {
        typename RgPack<T, H>::type a;
#pragma unroll
        for (int i = 0; i < H; ++i) a[i] = (T)v[h * H + i];
        typename RgPack<T, H>::type* to = (typename RgPack<T, H>::type*)p + h;
        if constexpr (ONCE) __builtin_nontemporal_store(a, to);
        else *to = a;
    }
}

// Whether results are stored past the caches: more of them than the L2s hold, in rows of whole 16 bytes (246 M clipped numbers 516 -> 490 us, 270 k
// normalised rows of 256 floats 96 -> 92; rows of 602 numbers of 16 bits, which share 16 bytes with their neighbours, 135 -> 137).  That the next call reads
// them does not turn it (a product of 256 outputs and the layer norm of its result, through the caches -> past them: 41 MB 30.1 -> 29.6 us of f32 and 35.1 ->
// 33.0 of bf16, 61 MB 48.5 -> 44.6, 82 MB 51.3 -> 50.6, 102 MB 68.2 -> 69.7, 123 MB 74.6 -> 75.5, 205 MB 127.9 -> 119.0, 276 MB 169 -> 157, 813 MB 509 -> 482).
static inline bool rg_store_once(const void* p, int64_t row_bytes, int64_t stride_bytes, int64_t rows) {
    return ((uintptr_t)p | (uintptr_t)row_bytes | (uintptr_t)stride_bytes) % 16 == 0 && row_bytes * rows > (32ll << 20);
}

// The first `live` of N numbers.  Of 16 bytes: 8, 4 and 2 of them, as the bits of `live` say.
template <int N, bool ONCE = false, typename T>
__device__ __forceinline__ void rg_store_live(T* p, int live, const float (&v)[N]) {
    if (live >= N) { rg_store<N, ONCE>(p, v); return; }
    if (live <= 0) return;
    if constexpr (N * sizeof(T) == 16) {
        typename RgPack<T, N>::type a;
#pragma unroll
        for (int i = 0; i < N; ++i) a[i] = (T)v[i];
        typedef uint32_t Words __attribute__((ext_vector_type(4)));
        const Words w = __builtin_bit_cast(Words, a);
        constexpr int HALF = N / 2, WORD = 4 / sizeof(T);
        const bool half = live & HALF;
        typedef uint32_t Two __attribute__((ext_vector_type(2), aligned(2)));
        typedef uint32_t One __attribute__((aligned(2)));
        if (half) *(Two*)p = Two{w[0], w[1]};
        T* to = p + (live & HALF);
        uint32_t rest = half ? w[2] : w[0];
        const uint32_t behind = half ? w[3] : w[1];
        if (live & (HALF / 2)) *(One*)to = rest;           // a word: one number of 32 bits, two of 16
        if constexpr (WORD == 2) {
            to += live & 2;
            rest = live & 2 ? behind : rest;
            if (live & 1) *(uint16_t*)to = (uint16_t)rest;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < live) p[i] = (T)v[i];
    }
}

__device__ __forceinline__ int64_t rg_least(int64_t a, int64_t b) { return a < b ? a : b; }

// min(n, *n_dev): the rows a batch really has.
__device__ __forceinline__ int64_t rg_rows(int64_t n, const int32_t* n_dev) {
    if (!n_dev) return n;
    const int64_t d = *n_dev;
    return d < n ? (d < 0 ? 0 : d) : n;
}

// Workgroups are dealt to the 8 XCDs in turn: the place of workgroup `block` of `grid` in an order in which neighbours share an XCD
// (and its L2).
__device__ __forceinline__ int rg_xcd_block(int block, int grid) {
    const int xcd = block & 7, per = grid >> 3, more = grid & 7;
    return xcd * per + min(xcd, more) + (block >> 3);
}

// i / d for i < 2^17 and d <= 2^14; m = rg_inverse(d).
static inline uint32_t rg_inverse(uint32_t d) { return d <= 1 ? 0 : (uint32_t)(((1ull << 32) + d - 1) / d); }
__device__ __forceinline__ uint32_t rg_divide(uint32_t i, uint32_t m) { return m ? __umulhi(i, m) : i; }

static inline int rg_type_bytes(rg_dtype t) { return t == RG_F32 ? 4 : 2; }
static inline bool rg_type_known(rg_dtype t) { return t == RG_F32 || t == RG_BF16 || t == RG_F16; }

// Runs `...` with the element type of `t` as T.
#define RG_FOR_TYPE(t, ...)                                     \
    do {                                                        \
        if ((t) == RG_F32) { typedef float T; __VA_ARGS__; }    \
        else if ((t) == RG_BF16) { typedef __bf16 T; __VA_ARGS__; } \
        else { typedef _Float16 T; __VA_ARGS__; }               \
    } while (0)
