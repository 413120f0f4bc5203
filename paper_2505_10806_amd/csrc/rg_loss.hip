// Softmax cross entropy of rows against the rows of a weight, and its gradients, without the logits in memory.
#include <type_traits>

#include "rg_elements.h"

namespace {

// With z = x . weight^T (n rows, `classes` columns), lse_i = log sum_c exp z_ic:  loss_i = lse_i - z_i,label(i);  with g_ic = exp(z_ic - lse_i) - [c = label(i)]:
// dx_i = share_i sum_c g_ic weight_c,  dweight_c = sum_i share_i g_ic x_i.
// One kernel does all three.  A wavefront owns 32 OB rows of one operand (of x for the loss and dx, of the weight for dweight) and walks the rows of the other, 64
// at a time through LDS: z of 64 by 32 OB from the matrix units, with the owned row along the lanes, so that a row's maximum and sum stay in
// its lane; exponentials; then, for a gradient, z's registers are the right operand of the second product as they lie, and the left one is the staged tile
// again, read transposed.  dx and dweight each form z anew: that is one product in four, and nothing of size n by classes is ever stored.
//
// Numbers go through the matrix units as bf16 or f16 as they are; f32 in three parts of bf16 that add up to it (the six products of parts that reach
// above 2^-24).  Of g, sums are in 32 bits and the second product takes g rounded to the rows' type (bf16: half an ulp of 2^-9, as the result's own rounding; f32: three parts again).
// For f16, g is scaled by 2^14, which keeps g down to 2^-28 in f16's normal range.
typedef float Acc __attribute__((ext_vector_type(16)));
typedef uint32_t Words4 __attribute__((ext_vector_type(4)));
typedef uint32_t Words2 __attribute__((ext_vector_type(2)));
typedef short Short4 __attribute__((ext_vector_type(4)));

// The type that the matrix units take, the parts of a number, what g is scaled by, and the rows of a walked tile (of three parts half as many: registers).
template <typename T> struct Part { typedef T type; static constexpr int P = 1, BIAS = 0, ROWS = 64; };
template <> struct Part<float> { typedef __bf16 type; static constexpr int P = 3, BIAS = 0, ROWS = 32; };
template <> struct Part<_Float16> { typedef _Float16 type; static constexpr int P = 1, BIAS = 14, ROWS = 64; };

constexpr int kCols = 128, kRowBytes = kCols * 2;           // of a staged tile
constexpr int kSteps = kCols / 16;                          // matrix products to its columns
constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr float kLog2e = 1.44269504088896340736f;
enum { LOSS = 0, DX = 1, DW = 2 };

typedef __bf16 Bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 Half8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ Acc mma(Words4 a, Words4 b, Acc c, __bf16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(Bf8, a), __builtin_bit_cast(Bf8, b), c, 0, 0, 0);
}
__device__ __forceinline__ Acc mma(Words4 a, Words4 b, Acc c, _Float16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(Half8, a), __builtin_bit_cast(Half8, b), c, 0, 0, 0);
}
// The product of numbers in P parts, small ones first.
template <typename E, int P>
__device__ __forceinline__ Acc mma_parts(const Words4 (&a)[P], const Words4 (&b)[P], Acc c) {
    if constexpr (P == 3) {
        c = mma(a[2], b[0], c, E());
        c = mma(a[1], b[1], c, E());
        c = mma(a[0], b[2], c, E());
        c = mma(a[1], b[0], c, E());
        c = mma(a[0], b[1], c, E());
    }
    return mma(a[0], b[0], c, E());
}

// Eight numbers as P parts.  A part of an f32 is what the parts before leave, cut to eight bits: the three add up to it (what lies below 2^-133 is cut off; of
// a number that is not finite not all parts are, and what it adds to is a NaN).
template <typename T>
__device__ __forceinline__ void cut(const float (&v)[8], Words4 (&w)[Part<T>::P]) {
    if constexpr (Part<T>::P == 1) {
        typedef T Eight __attribute__((ext_vector_type(8)));
        Eight e;
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = (T)v[j];
        w[0] = __builtin_bit_cast(Words4, e);
    } else {
        float rest[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) rest[j] = v[j];
#pragma unroll
        for (int p = 0; p < 3; ++p) {
#pragma unroll
            for (int j = 0; j < 8; j += 2) w[p][j / 2] = __builtin_amdgcn_perm(__float_as_uint(rest[j + 1]), __float_as_uint(rest[j]), 0x07060302u);
#pragma unroll
            for (int j = 0; j < 8; ++j) rest[j] -= __uint_as_float(__float_as_uint(rest[j]) & 0xFFFF0000u);
        }
    }
}

// Eight numbers of a row from `col`, as they lie; behind the row's end they are put right by row_parts.  SHORT: of rows that may be shorter.
template <bool SHORT, typename T>
__device__ __forceinline__ typename RgPack<T, 8>::type load_eight(const T* row, int col, int dim) {
    if (!SHORT || dim >= 8) return rg_load_row<8>(row, col, dim);
    return rg_load_raw<8>(row + col, dim - col);
}
// Them as parts (zeros if the row does not count).
template <bool SHORT, typename T>
__device__ __forceinline__ void row_parts(const typename RgPack<T, 8>::type& raw, int col, int dim, bool counts, Words4 (&w)[Part<T>::P]) {
    if constexpr (Part<T>::P == 1) {
        T v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = raw[j];
        if (!SHORT || dim >= 8) rg_row_end<8>(v, col, dim);
        typedef T Eight __attribute__((ext_vector_type(8)));
        Eight e;
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = v[j];
        w[0] = __builtin_bit_cast(Words4, e);
    } else {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = raw[j];
        if (!SHORT || dim >= 8) rg_row_end<8>(v, col, dim);
        cut<T>(v, w);
    }
    if (!counts) {
#pragma unroll
        for (int p = 0; p < Part<T>::P; ++p) w[p] = Words4{0, 0, 0, 0};
    }
}

__device__ __forceinline__ bool has_label(int label, int classes) { return (uint32_t)label < (uint32_t)classes; }

// The owned rows as the matrix units take them: [block of 32 rows][16 columns][part][lane][8 numbers], lane l the row l % 32 and the columns 8 (l / 32) .. + 7.
// Rows that are not there, or (labels given) do not count, are zeros.
template <typename T>
__global__ void __launch_bounds__(256) k_pack_rows(const T* __restrict__ x, int64_t stride, int64_t first, int64_t n, const int32_t* __restrict__ n_dev, int dim,
                                                   int steps, const int32_t* __restrict__ labels, int classes, int64_t units, Words4* __restrict__ packed) {
    constexpr int P = Part<T>::P;
    const int64_t n_act = rg_rows(n, n_dev);
    const int lane = rg_lane();
    for (int64_t unit = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 6; unit < units; unit += (int64_t)gridDim.x * 4) {
        const int64_t block = unit / steps, row = first + block * 32 + (lane & 31);
        const int col = (int)(unit - block * steps) * 16 + (lane >> 5) * 8;
        const bool counts = row < n_act && (!labels || has_label(labels[row], classes));
        Words4 w[P];
        typename RgPack<T, 8>::type raw = {};
        if (counts) raw = rg_load_raw<8>(x + row * stride + col, dim - col);
        float v[8];
        if constexpr (P == 1) w[0] = __builtin_bit_cast(Words4, raw);
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = raw[j];
            cut<T>(v, w);
        }
#pragma unroll
        for (int p = 0; p < P; ++p) packed[(unit * P + p) * 64 + lane] = w[p];
    }
}

struct Job {
    const Words4* owned;       // k_pack_rows of the owned rows
    const void* walked;
    int64_t stride;            // of the walked rows
    int64_t owners, rows;      // owned rows; walked rows
    int64_t first;             // of the owned rows, which are taken in pieces: labels, lse, dloss, target and out begin there
    int64_t n;                 // rows of x, and their count on the device
    const int32_t* n_dev;
    int dim, steps, chunks, classes, tiles, splits;
    const int32_t* labels;
    const float* lse;
    const float* dloss;
    float scale;
    float2* stats;             // LOSS: [split][row]: maximum of z, sum of exp(z - maximum)
    float* target;             // LOSS: z at the label
    void* out;                 // DX, DW: the gradient, if there is one split
    int64_t out_stride;
    float* parts;              // else [split][owned row][dim]
};

// STEPS: 16 columns each, of rows of up to 256 numbers; 0: any, in chunks.  HOLD: the owned rows stay in registers.
template <typename T, int MODE, int OB, int NB, int STEPS, bool HOLD>
__global__ void __launch_bounds__(kThreads, 2) k_softmax_rows(const Job job) {
    typedef Part<T> S;
    typedef typename S::type E;
    constexpr int P = S::P, ROWS = S::ROWS, OWNERS = kWaves * 32 * OB, ITEMS = ROWS * 16 / kThreads, SB = ROWS / 32;
    __shared__ __attribute__((aligned(16))) char staged[2][P][ROWS * kRowBytes];
    __shared__ __attribute__((aligned(16))) float row_lse[2][ROWS], row_share[2][ROWS];
    __shared__ __attribute__((aligned(16))) int row_label[2][ROWS];
    __shared__ float largest[kWaves];
    const int lane = rg_lane(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5;
    const int order = rg_xcd_block(blockIdx.x, gridDim.x), split = order / job.tiles, tile = order - split * job.tiles;
    const int64_t n_act = rg_rows(job.n, job.n_dev);
    const int64_t rows = MODE == DW ? n_act : job.rows, owners = MODE == DW ? job.owners : rg_least(job.owners, n_act - job.first);
    const int64_t first_owner = (int64_t)tile * OWNERS;
    if (first_owner >= owners) return;
    const T* walked = (const T*)job.walked;
    const int dim = job.dim, steps = job.steps, chunks = job.chunks;

    // the walked tiles of this split, and the stages of a tile: its chunks of 128 columns for z, the last of them one of this workgroup's output columns, which it
    // serves at once; then the other output columns' chunk
    const int64_t all = (rows + ROWS - 1) / ROWS, per = (all + job.splits - 1) / job.splits, t0 = rg_least(split * per, all), t1 = rg_least(t0 + per, all);
    constexpr int SLICE = NB / 4;
    const int slice = blockIdx.y * SLICE;
    const int more = MODE == LOSS ? 0 : min(SLICE, chunks - slice) - 1;
    const auto chunk_of = [&](int stage) __attribute__((always_inline)) {
        if (MODE == LOSS) return stage;
        if (stage >= chunks) return slice + stage - chunks + 1;
        const int c = slice + 1 + stage;
        return c >= chunks ? c - chunks : c;
    };

    // dweight: shares are scaled by a power of two to at most 1, and the sums back
    int power = 0;
    if (MODE == DW && job.dloss) {
        float top = 0.0f;
        for (int64_t r = t0 * ROWS + threadIdx.x; r < rg_least(t1 * ROWS, rows); r += kThreads)
            if (has_label(job.labels[r], job.classes)) top = fmaxf(top, fabsf(job.dloss[r]));
        for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, RG_WAVE));
        if (lane == 0) largest[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, largest[w]);
        if (top > 0.0f && top < __builtin_inff()) (void)frexpf(top, &power);
    }

    // what a lane's owned rows bring
    int64_t owner[OB];
    int label[OB];
    float lse2[OB], m[OB], s[OB];
#pragma unroll
    for (int b = 0; b < OB; ++b) {
        owner[b] = first_owner + (wave * OB + b) * 32 + (lane & 31);
        label[b] = -1;
        lse2[b] = 0.0f;
        m[b] = -__builtin_inff();
        s[b] = 0.0f;
        if (MODE != DW && owner[b] < owners) {
            label[b] = job.labels[owner[b]];
            if (!has_label(label[b], job.classes)) label[b] = -1;
            if (MODE == DX && label[b] >= 0) lse2[b] = job.lse[owner[b]] * kLog2e - (float)S::BIAS;
        }
    }
    const Words4* owned[OB];
#pragma unroll
    for (int b = 0; b < OB; ++b) owned[b] = job.owned + ((first_owner / 32 + wave * OB + b) * steps) * (P * 64) + lane;
    Words4 held[OB][HOLD ? STEPS : 1][P];
    if constexpr (HOLD) {
#pragma unroll
        for (int b = 0; b < OB; ++b)
#pragma unroll
            for (int k = 0; k < STEPS; ++k)
#pragma unroll
                for (int p = 0; p < P; ++p) held[b][k][p] = owned[b][(k * P + p) * 64];
    }

    // staging: a thread's pieces of eight columns
    typename RgPack<T, 8>::type raw[ITEMS];
    bool counts[ITEMS];
    float next_lse = 0.0f, next_share = 0.0f;
    int next_label = -1;
    const auto load = [&](int64_t t, int stage) __attribute__((always_inline)) {
        const int chunk = chunk_of(stage);
#pragma unroll
        for (int u = 0; u < ITEMS; ++u) {
            const int i = threadIdx.x + u * kThreads;
            const int64_t r = t * ROWS + (i >> 4), from = rg_least(r, rows - 1);
            counts[u] = r < rows && (MODE != DW || has_label(job.labels[from], job.classes));
            raw[u] = load_eight<STEPS == 2>(walked + from * job.stride, chunk * kCols + (i & 15) * 8, dim);
        }
        if (MODE == DW && stage == 0 && threadIdx.x < ROWS) {
            const int64_t r = t * ROWS + threadIdx.x, from = rg_least(r, rows - 1);
            next_label = job.labels[from];
            const bool live = r < rows && has_label(next_label, job.classes);
            next_lse = live ? job.lse[from] * kLog2e : 0.0f;
            next_share = live ? ldexpf(job.dloss ? job.dloss[from] : 1.0f, S::BIAS - power) : 0.0f;
            if (!live) next_label = -1;
        }
    };
    const auto store = [&](int64_t t, int stage, int buffer) __attribute__((always_inline)) {
        const int chunk = chunk_of(stage);
        int dim = job.dim;
        asm volatile("" : "+s"(dim));                      // (else what depends on it is formed before the loop and takes registers through all of it)
#pragma unroll
        for (int u = 0; u < ITEMS; ++u) {
            const int i = threadIdx.x + u * kThreads, row = i >> 4, piece = (i & 15) ^ ((row & 3) << 1 | (row >> 2 & 1));
            Words4 w[P];
            row_parts<STEPS == 2, T>(raw[u], chunk * kCols + (i & 15) * 8, dim, counts[u], w);
#pragma unroll
            for (int p = 0; p < P; ++p) *(Words4*)(staged[buffer][p] + row * kRowBytes + piece * 16) = w[p];
        }
        if (MODE == DW && stage == 0 && threadIdx.x < ROWS) {
            row_lse[t & 1][threadIdx.x] = next_lse;
            row_share[t & 1][threadIdx.x] = next_share;
            row_label[t & 1][threadIdx.x] = next_label;
        }
    };

    Acc z[SB][OB], out[MODE == LOSS ? 1 : OB][MODE == LOSS ? 1 : NB];
    Words4 g[MODE == LOSS ? 1 : SB][2][MODE == LOSS ? 1 : OB][P];
    if (MODE != LOSS) {
#pragma unroll
        for (int b = 0; b < OB; ++b)
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) out[b][d][i] = 0.0f;
    }

    const int walk_row = lane & 31, twist = (walk_row & 3) << 1 | (walk_row >> 2 & 1);
    // z += the products of K steps of 16 columns, FROM the chunk's first step on.  Fragments of the walked rows are read RING - 1 products ahead, those of the owned
    // rows, where they are not held, two steps; the barriers keep the compiler from reading all of them at once, for which there are no registers.
    constexpr int RING = P == 1 ? 4 : 2;
    const auto products = [&](auto count, auto from, int chunk, int buffer) __attribute__((always_inline)) {
        constexpr int K = decltype(count)::value, FROM = decltype(from)::value, UNITS = K * SB, AHEAD = P == 1 ? 3 : 2;
        Words4 left[RING][P], right[AHEAD][OB][P];
        const auto read = [&](int u) __attribute__((always_inline)) {
            const int k = u / SB, q = u % SB;
#pragma unroll
            for (int p = 0; p < P; ++p) left[u % RING][p] = *(const Words4*)(staged[buffer][p] + (q * 32 + walk_row) * kRowBytes + (((2 * k + half) ^ twist) << 4));
        };
        const auto fetch = [&](int k) __attribute__((always_inline)) {
#pragma unroll
            for (int b = 0; b < OB; ++b)
#pragma unroll
                for (int p = 0; p < P; ++p) right[k % AHEAD][b][p] = owned[b][((int64_t)(chunk * kSteps + k) * P + p) * 64];
        };
        if constexpr (!HOLD) {
#pragma unroll
            for (int k = 0; k < AHEAD - 1; ++k)
                if (k < K) fetch(k);
        }
#pragma unroll
        for (int u = 0; u < RING - 1; ++u)
            if (u < UNITS) read(u);
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int k = u / SB, q = u % SB;
            if (u + RING - 1 < UNITS) read(u + RING - 1);
            if constexpr (!HOLD) {
                if (q == 0 && k + AHEAD - 1 < K) fetch(k + AHEAD - 1);
            }
#pragma unroll
            for (int b = 0; b < OB; ++b) {
                if constexpr (HOLD) z[q][b] = mma_parts<E, P>(left[u % RING], held[b][FROM + k], z[q][b]);
                else z[q][b] = mma_parts<E, P>(left[u % RING], right[k % AHEAD][b], z[q][b]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // out += g . the staged rows, for D blocks of 32 columns
    const auto second = [&](auto base, auto count, int buffer) __attribute__((always_inline)) {
        constexpr int D0 = decltype(base)::value, D = decltype(count)::value, UNITS = SB * 2 * D;
        const int i = lane & 15, row0 = 4 * half + (i >> 2), turn = (i >> 2) << 1 | half;
        Words4 left[RING][P];
        const auto read = [&](int u) __attribute__((always_inline)) {
            const int q = u / (2 * D), f = u / D % 2, d = u % D;
            const int piece = ((d * 4 + (lane >> 4 & 1) * 2 + (i >> 1 & 1)) ^ turn) * 16 + (i & 1) * 8;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const char* at = staged[buffer][p] + (q * 32 + f * 16 + row0) * kRowBytes + piece;
                typedef __attribute__((address_space(3))) Short4 Lds;
                const Words2 low = __builtin_bit_cast(Words2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)at));
                const Words2 high = __builtin_bit_cast(Words2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(at + 8 * kRowBytes)));
                left[u % RING][p] = Words4{low[0], low[1], high[0], high[1]};
            }
        };
#pragma unroll
        for (int u = 0; u < RING - 1; ++u)
            if (u < UNITS) read(u);
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int q = u / (2 * D), f = u / D % 2, d = u % D;
            if (u + RING - 1 < UNITS) read(u + RING - 1);
#pragma unroll
            for (int b = 0; b < OB; ++b) out[b][D0 + d] = mma_parts<E, P>(left[u % RING], g[q][f][b], out[b][D0 + d]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // z of a whole tile is there.  (What few tiles need, labels and the ends, stands in loops of its own behind barriers: mixed into the others it took 70 registers.)
    const auto finish = [&](int64_t t) __attribute__((always_inline)) {
        const int64_t first = t * ROWS;
        __builtin_amdgcn_sched_barrier(0);
        if (MODE == DW) {
            const int seen = row_label[t & 1][lane & (ROWS - 1)];
            const int64_t mine = job.first + first_owner + wave * OB * 32;
            const bool hits = __any(seen >= mine && seen < mine + OB * 32), idle = __any(row_share[t & 1][lane & (ROWS - 1)] == 0.0f);
#pragma unroll
            for (int q = 0; q < SB; ++q)
#pragma unroll
                for (int i = 0; i < 16; ++i)
#pragma unroll
                    for (int b = 0; b < OB; ++b)
                        z[q][b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[q][b][i], kLog2e, -row_lse[t & 1][q * 32 + 8 * (i >> 2) + 4 * half + (i & 3)]));
            __builtin_amdgcn_sched_barrier(0);
            if (hits) {
#pragma unroll
                for (int q = 0; q < SB; ++q)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
#pragma unroll
                        for (int b = 0; b < OB; ++b)
                            z[q][b][i] -= row_label[t & 1][q * 32 + 8 * (i >> 2) + 4 * half + (i & 3)] == (int)(job.first + owner[b]) ? 1.0f : 0.0f;
                __builtin_amdgcn_sched_barrier(0);
            }
            if (idle) {                                    // (nothing of a row that does not count, whatever its p is)
#pragma unroll
                for (int q = 0; q < SB; ++q)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
#pragma unroll
                        for (int b = 0; b < OB; ++b) z[q][b][i] = row_share[t & 1][q * 32 + 8 * (i >> 2) + 4 * half + (i & 3)] == 0.0f ? 0.0f : z[q][b][i];
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int q = 0; q < SB; ++q)
#pragma unroll
                for (int i = 0; i < 16; ++i)
#pragma unroll
                    for (int b = 0; b < OB; ++b) z[q][b][i] *= row_share[t & 1][q * 32 + 8 * (i >> 2) + 4 * half + (i & 3)];
        } else {
            if (first + ROWS > rows) {                    // (behind the last class)
                const int end = (int)(rows - first) - 4 * half;
#pragma unroll
                for (int q = 0; q < SB; ++q)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
#pragma unroll
                        for (int b = 0; b < OB; ++b) z[q][b][i] = q * 32 + 8 * (i >> 2) + (i & 3) >= end ? -__builtin_inff() : z[q][b][i];
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int b = 0; b < OB; ++b) {
                const bool here = label[b] >= first && label[b] < first + ROWS;
                const int at = (int)(label[b] - first) - 4 * half;           // (of this half's, if it equals one of them)
                const bool hits = __any(here);
                if (MODE == LOSS) {
                    if (hits) {
                        float told = 0.0f;
                        bool mine = false;
#pragma unroll
                        for (int q = 0; q < SB; ++q)
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const bool is = at == q * 32 + 8 * (i >> 2) + (i & 3);
                                told = is ? z[q][b][i] : told;
                                mine |= is;
                            }
                        if (here && mine) job.target[owner[b]] = told;
                        __builtin_amdgcn_sched_barrier(0);
                    }
                    float top = m[b];
#pragma unroll
                    for (int q = 0; q < SB; ++q)
#pragma unroll
                        for (int i = 0; i < 16; ++i) top = fmaxf(top, z[q][b][i]);
                    const float base = top == -__builtin_inff() ? 0.0f : top * kLog2e;
                    float sum[4] = {s[b] * __builtin_amdgcn_exp2f(__builtin_fmaf(m[b], kLog2e, -base)), 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int q = 0; q < SB; ++q)
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[i & 3] += __builtin_amdgcn_exp2f(__builtin_fmaf(z[q][b][i], kLog2e, -base));
                    m[b] = top;
                    s[b] = (sum[0] + sum[1]) + (sum[2] + sum[3]);
                } else {
#pragma unroll
                    for (int q = 0; q < SB; ++q)
#pragma unroll
                        for (int i = 0; i < 16; ++i) z[q][b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[q][b][i], kLog2e, -lse2[b]));
                    if (hits) {
                        __builtin_amdgcn_sched_barrier(0);
                        const int there = here ? at : -1000;
#pragma unroll
                        for (int q = 0; q < SB; ++q)
#pragma unroll
                            for (int i = 0; i < 16; ++i) z[q][b][i] -= there == q * 32 + 8 * (i >> 2) + (i & 3) ? (float)(1 << S::BIAS) : 0.0f;
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        }
        if constexpr (MODE != LOSS) {
#pragma unroll
            for (int q = 0; q < SB; ++q)
#pragma unroll
                for (int b = 0; b < OB; ++b)
#pragma unroll
                    for (int f = 0; f < 2; ++f) {
                        float v[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = z[q][b][f * 8 + j];
                        cut<T>(v, g[q][f][b]);
                    }
        }
        __builtin_amdgcn_sched_barrier(0);
    };

#define RG_INT(N) std::integral_constant<int, N>()
    constexpr int FIRST = STEPS == 0 || STEPS > kSteps ? 4 : STEPS / 2, SECOND = STEPS > kSteps ? (STEPS - kSteps) / 2 : 4;      // blocks of output columns
    const auto add_products = [&](int chunk, int buffer) __attribute__((always_inline)) {
        if constexpr (STEPS > kSteps) {
            if (chunk == 0) products(RG_INT(kSteps), RG_INT(0), chunk, buffer);
            else products(RG_INT(STEPS - kSteps), RG_INT(kSteps), chunk, buffer);
        } else if constexpr (STEPS > 0) {
            products(RG_INT(STEPS), RG_INT(0), chunk, buffer);
        } else {
            const int here = steps - chunk * kSteps;
            if (here > 6) products(RG_INT(8), RG_INT(0), chunk, buffer);
            else if (here > 4) products(RG_INT(6), RG_INT(0), chunk, buffer);
            else if (here > 2) products(RG_INT(4), RG_INT(0), chunk, buffer);
            else products(RG_INT(2), RG_INT(0), chunk, buffer);
        }
    };
    if (t0 < t1) {
        load(t0, 0);
        store(t0, 0, 0);
        __syncthreads();
    }
    int buffer = 0;
#pragma unroll 1
    for (int64_t t = t0; t < t1; ++t) {
#pragma unroll
        for (int q = 0; q < SB; ++q)
#pragma unroll
            for (int b = 0; b < OB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) z[q][b][i] = 0.0f;
        if (STEPS == 0 || STEPS > kSteps) {
#pragma unroll 1
            for (int stage = 0; stage < (STEPS > kSteps ? 1 : chunks - 1); ++stage) {
                load(t, stage + 1);
                add_products(MODE != LOSS && STEPS > kSteps ? 1 : chunk_of(stage), buffer);
                store(t, stage + 1, buffer ^ 1);
                __syncthreads();
                buffer ^= 1;
            }
        }
        // (the next rows are asked for behind the products of z, which leave no registers for them)
        add_products(STEPS > 0 && (MODE != LOSS || STEPS <= kSteps) ? 0 : STEPS > 0 ? 1 : chunk_of(chunks - 1), buffer);
        finish(t);
        const bool rest = NB > 4 && more > 0, go_on = t + 1 < t1;
        if (rest) load(t, chunks);
        else if (go_on) load(t + 1, 0);
        if constexpr (MODE != LOSS) second(RG_INT(0), RG_INT(FIRST), buffer);
        if (rest) store(t, chunks, buffer ^ 1);
        else if (go_on) store(t + 1, 0, buffer ^ 1);
        __syncthreads();
        buffer ^= 1;
        if constexpr (MODE != LOSS && NB > 4) {
            if (rest) {
                if (go_on) load(t + 1, 0);
                second(RG_INT(4), RG_INT(SECOND), buffer);
                if (go_on) store(t + 1, 0, buffer ^ 1);
                __syncthreads();
                buffer ^= 1;
            }
        }
    }
#undef RG_INT

    if constexpr (MODE == LOSS) {
#pragma unroll
        for (int b = 0; b < OB; ++b) {
            const float other_m = __shfl_xor(m[b], 32, RG_WAVE), other_s = __shfl_xor(s[b], 32, RG_WAVE);
            const float top = fmaxf(m[b], other_m), base = top == -__builtin_inff() ? 0.0f : top * kLog2e;
            const float sum = s[b] * __builtin_amdgcn_exp2f(__builtin_fmaf(m[b], kLog2e, -base)) + other_s * __builtin_amdgcn_exp2f(__builtin_fmaf(other_m, kLog2e, -base));
            if (half == 0 && owner[b] < owners) job.stats[split * job.owners + owner[b]] = make_float2(top, sum);
        }
    } else {
#pragma unroll
        for (int b = 0; b < OB; ++b) {
            if (owner[b] >= owners) continue;
            float factor = job.scale;
            const bool none = MODE == DX && label[b] < 0;
            if (MODE == DX && !none && job.dloss) factor *= job.dloss[owner[b]];
#pragma unroll
            for (int d = 0; d < NB; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int col = (slice * 4 + d) * 32 + i * 8 + half * 4;
                    if (col >= dim) continue;
                    float v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        v[j] = out[b][d][i * 4 + j] * factor;
                        if (MODE == DW || S::BIAS) v[j] = ldexpf(v[j], power - S::BIAS);
                        if (none) v[j] = 0.0f;
                    }
                    if (job.splits == 1) rg_store_live<4>((T*)job.out + owner[b] * job.out_stride + col, dim - col, v);
                    else rg_store_live<4>(job.parts + (split * job.owners + owner[b]) * dim + col, dim - col, v);
                }
        }
    }
}

// Each row's log-sum and loss from its splits.
__global__ void __launch_bounds__(256) k_loss_join(const float2* __restrict__ stats, int splits, int64_t first, int64_t count, int64_t n,
                                                   const int32_t* __restrict__ n_dev, const int32_t* __restrict__ labels, int classes, const float* __restrict__ target, float* __restrict__ loss,
                                                   float* __restrict__ lse) {
    // 16 lanes to a row
    const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 4;
    const int l = threadIdx.x & 15;
    if (row >= rg_least(count, rg_rows(n, n_dev) - first)) return;
    float m = -__builtin_inff(), s = 0.0f;
    const auto merge = [&](float other_m, float other_s) {
        const float top = fmaxf(m, other_m), base = top == -__builtin_inff() ? 0.0f : top;
        s = s * __builtin_amdgcn_exp2f((m - base) * kLog2e) + other_s * __builtin_amdgcn_exp2f((other_m - base) * kLog2e);
        m = top;
    };
    for (int k = l; k < splits; k += 16) {
        const float2 part = stats[(int64_t)k * count + row];
        merge(part.x, part.y);
    }
    for (int off = 8; off > 0; off >>= 1) merge(__shfl_xor(m, off, 16), __shfl_xor(s, off, 16));
    if (l != 0) return;
    const bool counts = has_label(labels[row], classes);
    const float sum = m + logf(s);
    if (lse) lse[row] = counts ? sum : 0.0f;
    if (loss) loss[row] = counts ? sum - target[row] : 0.0f;
}

// Sums of the splits' parts, in the order of the splits.
template <typename T>
__global__ void __launch_bounds__(256) k_grad_join(const float* __restrict__ parts, int splits, int64_t rows, int64_t first, int64_t n,
                                                   const int32_t* __restrict__ n_dev, int dim, int chunks, T* __restrict__ out, int64_t stride) {
    constexpr int V = 4;
    const int64_t total = rg_least(rows, rg_rows(n, n_dev) - first) * chunks, one = rows * dim;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / chunks;
        const int col = (int)(i - row * chunks) * V;
        float sum[V] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
        for (int k = 0; k < splits; ++k) {
            float v[V];
            rg_load_head<V>(parts + k * one + row * dim + col, dim - col, v);
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] += v[j];
        }
        rg_store_live<V>(out + row * stride + col, dim - col, sum);
    }
}

// Rows of zeros.
template <typename T>
__global__ void __launch_bounds__(256) k_zero_rows(T* __restrict__ out, int64_t stride, int64_t rows, int dim, int chunks) {
    constexpr int V = 16 / (int)sizeof(T);
    const float zero[V] = {};
    const int64_t total = rows * chunks;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / chunks;
        const int col = (int)(i - row * chunks) * V;
        rg_store_live<V>(out + row * stride + col, dim - col, zero);
    }
}

bool aligned(const void* p, int bytes) { return (uintptr_t)p % (uintptr_t)bytes == 0; }

constexpr int64_t kMostRows = (1ll << 31) - 1;

// Columns of a row as steps of 16, an even number of them (12 or 16 from 129 columns on, as the kernel holds them).
int steps_of(int dim) {
    const int steps = 2 * (int)rg_div_up(dim, 32);
    return steps <= 8 || steps > 16 ? steps : steps <= 12 ? 12 : 16;
}

int64_t packed_row(int steps, int parts) { return (int64_t)steps * parts * 32; }

constexpr int kOwners = 256;                                // packed rows come in so many

// Rows that are owned at a time: their packed form stays in the last level of cache.
int64_t piece_rows(int64_t rows, int steps, int parts) {
    const int64_t most = rg_max64(1, (128ll << 20) / packed_row(steps, parts) / kOwners) * kOwners;
    return rg_min64(most, rg_div_up(rows, kOwners) * kOwners);
}

template <typename T>
void pack(rg_ctx* ctx, const void* x, int64_t stride, int64_t first, int64_t count, int64_t n, const int32_t* n_dev, int dim, int steps, const int32_t* labels,
          int classes, void* packed, hipStream_t s) {
    const int64_t units = rg_div_up(count, kOwners) * (kOwners / 32) * steps;
    k_pack_rows<T><<<(unsigned)rg_min64(rg_div_up(units, 4), (int64_t)ctx->num_cus * 32), 256, 0, s>>>((const T*)x, stride, first, n, n_dev, dim, steps, labels, classes,
                                                                                                 units, (Words4*)packed);
}

// Splits of the walked rows: as many workgroups as fill the device twice.
int splits_for(rg_ctx* ctx, int64_t workgroups, int64_t walked) {
    return (int)rg_max64(1, rg_min64(rg_div_up(walked, 64), (int64_t)ctx->num_cus * 2 / workgroups));
}

rg_status check_loss(rg_ctx* ctx, const char* who, const void* x, rg_dtype type, int64_t x_stride, int64_t n, int32_t dim, const void* weight,
                     int64_t weight_stride, int32_t classes, const int32_t* labels, const float* lse) {
    RG_REQUIRE(ctx, n >= 0 && n <= kMostRows, "%s: n = %lld out of range", who, (long long)n);
    RG_REQUIRE(ctx, dim >= 1 && dim <= RG_LOSS_MAX_DIM, "%s: dim = %d not in [1,%d]", who, dim, RG_LOSS_MAX_DIM);
    RG_REQUIRE(ctx, classes >= 1, "%s: classes = %d is not positive", who, classes);
    RG_REQUIRE(ctx, rg_type_known(type), "%s: unknown type %d", who, (int)type);
    RG_REQUIRE(ctx, x_stride >= dim && weight_stride >= dim, "%s: bad stride", who);
    RG_REQUIRE(ctx, n == 0 || (x && weight && labels), "%s: null pointer", who);
    const int b = rg_type_bytes(type);
    RG_REQUIRE(ctx, aligned(x, b) && aligned(weight, b) && aligned(labels, 4) && aligned(lse, 4), "%s: pointer not aligned to its numbers", who);
    return RG_OK;
}

// The kernel for a job, and the rows that a workgroup of it owns.
template <typename T, int MODE>
constexpr int owned_blocks() { return Part<T>::P == 1 && MODE == LOSS ? 2 : 1; }

template <typename T, int MODE>
void launch(const Job& job, int64_t slices, hipStream_t s) {
    constexpr bool ONE = Part<T>::P == 1;
    constexpr int OB = owned_blocks<T, MODE>();
    const dim3 grid((unsigned)((int64_t)job.tiles * job.splits), (unsigned)slices);
    switch (job.steps) {
        case 2: k_softmax_rows<T, MODE, OB, 4, 2, ONE><<<grid, kThreads, 0, s>>>(job); break;
        case 4: k_softmax_rows<T, MODE, OB, 4, 4, ONE><<<grid, kThreads, 0, s>>>(job); break;
        case 6: k_softmax_rows<T, MODE, OB, 4, 6, ONE><<<grid, kThreads, 0, s>>>(job); break;
        case 8: k_softmax_rows<T, MODE, OB, 4, 8, ONE><<<grid, kThreads, 0, s>>>(job); break;
        case 12: k_softmax_rows<T, MODE, OB, 8, 12, ONE && MODE == LOSS><<<grid, kThreads, 0, s>>>(job); break;
        case 16: k_softmax_rows<T, MODE, OB, 8, 16, ONE && MODE == LOSS><<<grid, kThreads, 0, s>>>(job); break;
        default: k_softmax_rows<T, MODE, OB, 8, 0, false><<<grid, kThreads, 0, s>>>(job);
    }
}

}  // namespace

extern "C" {

rg_status rg_cross_entropy(rg_ctx* ctx, const void* x, rg_dtype type, int64_t x_stride, int64_t n, const int32_t* n_dev, int32_t dim, const void* weight,
                           int64_t weight_stride, int32_t classes, const int32_t* labels, float* loss, float* lse, void* stream) {
    if (!ctx) return RG_ERR_INVALID_ARG;
    const rg_status bad = check_loss(ctx, "rg_cross_entropy", x, type, x_stride, n, dim, weight, weight_stride, classes, labels, lse);
    if (bad != RG_OK) return bad;
    RG_REQUIRE(ctx, aligned(loss, 4), "rg_cross_entropy: pointer not aligned to its numbers");
    if (n == 0 || (!loss && !lse)) return RG_OK;
    RG_HIP(ctx, hipSetDevice(ctx->device));
    hipStream_t s = (hipStream_t)stream;
    RG_FOR_TYPE(type, {
        constexpr int P = Part<T>::P;
        const int steps = steps_of(dim);
        const int64_t piece = piece_rows(n, steps, P), most = rg_min64(piece, n), tiles = rg_div_up(most, (int64_t)kWaves * 32 * owned_blocks<T, LOSS>());
        const int splits = splits_for(ctx, tiles, classes);
        const size_t packed = (size_t)(rg_div_up(most, kOwners) * kOwners * packed_row(steps, P)), stats = (size_t)splits * most * sizeof(float2);
        const rg_status st = rg_scratch(ctx, ctx->loss_parts, packed + stats + (size_t)most * 4, s, "rg_cross_entropy");
        if (st != RG_OK) return st;
        char* at = (char*)ctx->loss_parts.p;
        Job job = {};
        job.owned = (const Words4*)at;
        job.walked = weight;
        job.stride = weight_stride;
        job.rows = classes;
        job.n = n;
        job.n_dev = n_dev;
        job.dim = dim;
        job.steps = steps;
        job.chunks = (int)rg_div_up(dim, kCols);
        job.classes = classes;
        job.splits = splits;
        job.stats = (float2*)(at + packed);
        job.target = (float*)(at + packed + stats);
        for (int64_t first = 0; first < n; first += piece) {
            const int64_t count = rg_min64(piece, n - first);
            pack<T>(ctx, x, x_stride, first, count, n, n_dev, dim, steps, nullptr, classes, at, s);
            job.owners = count;
            job.first = first;
            job.tiles = (int)rg_div_up(count, (int64_t)kWaves * 32 * owned_blocks<T, LOSS>());
            job.labels = labels + first;
            launch<T, LOSS>(job, 1, s);
            RG_LAUNCH_CHECK(ctx, "k_softmax_rows");
            k_loss_join<<<(unsigned)rg_div_up(count, 16), 256, 0, s>>>(job.stats, splits, first, count, n, n_dev, job.labels, classes, job.target,
                                                                       loss ? loss + first : nullptr, lse ? lse + first : nullptr);
            RG_LAUNCH_CHECK(ctx, "k_loss_join");
        }
    });
    return RG_OK;
}

rg_status rg_cross_entropy_grad(rg_ctx* ctx, const void* x, rg_dtype type, int64_t x_stride, int64_t n, const int32_t* n_dev, int32_t dim, const void* weight,
                                int64_t weight_stride, int32_t classes, const int32_t* labels, const float* lse, const float* dloss, float scale, void* dx,
                                int64_t dx_stride, void* dweight, int64_t dweight_stride, void* stream) {
    if (!ctx) return RG_ERR_INVALID_ARG;
    const rg_status bad = check_loss(ctx, "rg_cross_entropy_grad", x, type, x_stride, n, dim, weight, weight_stride, classes, labels, lse);
    if (bad != RG_OK) return bad;
    RG_REQUIRE(ctx, n == 0 || lse, "rg_cross_entropy_grad: null pointer");
    RG_REQUIRE(ctx, (!dx || dx_stride >= dim) && (!dweight || dweight_stride >= dim), "rg_cross_entropy_grad: bad stride");
    RG_REQUIRE(ctx, scale == scale, "rg_cross_entropy_grad: scale is not a number");
    const int b = rg_type_bytes(type);
    RG_REQUIRE(ctx, aligned(dx, b) && aligned(dweight, b) && aligned(dloss, 4), "rg_cross_entropy_grad: pointer not aligned to its numbers");
    if (!dweight && (!dx || n == 0)) return RG_OK;
    RG_HIP(ctx, hipSetDevice(ctx->device));
    hipStream_t s = (hipStream_t)stream;
    RG_FOR_TYPE(type, {
        constexpr int P = Part<T>::P;
        const int quads = (int)rg_div_up(dim, 4);
        if (n == 0) {
            const int pieces = (int)rg_div_up(dim, 16 / (int)sizeof(T));
            k_zero_rows<T><<<(unsigned)rg_min64(rg_div_up((int64_t)classes * pieces, 256), (int64_t)ctx->num_cus * 32), 256, 0, s>>>((T*)dweight, dweight_stride, classes,
                                                                                                                     dim, pieces);
            RG_LAUNCH_CHECK(ctx, "k_zero_rows");
            return RG_OK;
        }
        const int steps = steps_of(dim), chunks = (int)rg_div_up(dim, kCols);
        const int64_t slices = rg_div_up(chunks, 2);       // (a workgroup's output: up to two chunks of columns)
        struct Side {
            int64_t rows, piece, most, tiles;
            int splits;
            size_t packed, parts;
        };
        const auto side = [&](int64_t rows, int64_t walked) {
            Side v;
            v.rows = rows;
            v.piece = piece_rows(rows, steps, P);
            v.most = rg_min64(v.piece, rows);
            v.tiles = rg_div_up(v.most, kWaves * 32);
            v.splits = splits_for(ctx, v.tiles * slices, walked);
            v.packed = (size_t)(rg_div_up(v.most, kOwners) * kOwners * packed_row(steps, P));
            v.parts = v.splits > 1 ? (size_t)v.splits * v.most * dim * 4 : 0;
            return v;
        };
        const Side for_dx = side(n, classes), for_dw = side(classes, n);
        const size_t dx_bytes = dx ? for_dx.packed + for_dx.parts : 0, dw_bytes = dweight ? for_dw.packed + for_dw.parts : 0;
        const rg_status st = rg_scratch(ctx, ctx->loss_parts, dx_bytes > dw_bytes ? dx_bytes : dw_bytes, s, "rg_cross_entropy_grad");
        if (st != RG_OK) return st;
        char* at = (char*)ctx->loss_parts.p;
        Job job = {};
        job.owned = (const Words4*)at;
        job.n = n;
        job.n_dev = n_dev;
        job.dim = dim;
        job.steps = steps;
        job.chunks = chunks;
        job.classes = classes;
        job.scale = scale;
        const auto take = [&](const Side& v, int64_t first, void* out, int64_t stride) {
            job.owners = rg_min64(v.piece, v.rows - first);
            job.first = first;
            job.tiles = (int)rg_div_up(job.owners, kWaves * 32);
            job.splits = v.splits;
            job.parts = (float*)(at + v.packed);
            job.out = (T*)out + first * stride;
            job.out_stride = stride;
        };
        const auto join = [&](int64_t rows, const int32_t* count) {
            if (job.splits > 1)
                k_grad_join<T><<<(unsigned)rg_min64(rg_div_up(job.owners * quads, 256), (int64_t)ctx->num_cus * 32), 256, 0, s>>>(
                    job.parts, job.splits, job.owners, job.first, rows, count, dim, quads, (T*)job.out, job.out_stride);
        };
        for (int64_t first = 0; dx && first < n; first += for_dx.piece) {
            take(for_dx, first, dx, dx_stride);
            pack<T>(ctx, x, x_stride, first, job.owners, n, n_dev, dim, steps, labels, classes, at, s);
            job.walked = weight;
            job.stride = weight_stride;
            job.rows = classes;
            job.labels = labels + first;
            job.lse = lse + first;
            job.dloss = dloss ? dloss + first : nullptr;
            launch<T, DX>(job, slices, s);
            RG_LAUNCH_CHECK(ctx, "k_softmax_rows");
            join(n, n_dev);
            RG_LAUNCH_CHECK(ctx, "k_grad_join");
        }
        for (int64_t first = 0; dweight && first < classes; first += for_dw.piece) {
            take(for_dw, first, dweight, dweight_stride);
            pack<T>(ctx, weight, weight_stride, first, job.owners, classes, nullptr, dim, steps, nullptr, 0, at, s);
            job.walked = x;
            job.stride = x_stride;
            job.rows = n;
            job.labels = labels;
            job.lse = lse;
            job.dloss = dloss;
            launch<T, DW>(job, slices, s);
            RG_LAUNCH_CHECK(ctx, "k_softmax_rows");
            join(classes, nullptr);
            RG_LAUNCH_CHECK(ctx, "k_grad_join");
        }
    });
    return RG_OK;
}

}  // extern "C"
