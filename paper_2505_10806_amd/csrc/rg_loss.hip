// Softmax cross entropy of rows against the rows of a weight, and its gradients, without the logits in memory.
#include <type_traits>

#include "rg_elements.h"

namespace {

// With z = x . weight^T (n rows, `classes` columns), lse_i = log sum_c exp z_ic:  loss_i = lse_i - z_i,label(i);  with g_ic = exp(z_ic - lse_i) - [c = label(i)]:
// dx_i = share_i sum_c g_ic weight_c,  dweight_c = sum_i share_i g_ic x_i.
// One kernel does all three.  A wavefront owns 32 rows of one operand (of x for the loss and dx, of the weight for dweight) and walks the rows of the other, 64
// at a time through LDS: z of 64 by 32 from the matrix units, with the owned row along the lanes, so that a row's maximum and sum stay in
// its lane; exponentials; then, for a gradient, z's registers are the right operand of the second product as they lie, and the left one is the staged tile
// again, read transposed.  dx and dweight each form z anew: that is one product in four, and nothing of size n by classes is ever stored.
//
// Numbers go through the matrix units as bf16 or f16 as they are; f32 in three parts of bf16 that add up to it, of which the second and third reach 2^-7 and 2^-15 of a
// number: six products of parts (what the other three would add is below 2^-21 + 2^-30 of the product, and has its sign).  Of g, sums are in 32 bits and the second
// product takes g rounded to the rows' type: bf16 off by at most 2^-8 of it, as the result's own rounding is, which takes results of few terms further from
// 64 bits (of many rows over 2 to 100 classes 2.2e-3 of their norm instead of 1.7e-3, dweight of one row, where one g has all of the norm, up to 2^-8; of 1024 rows against 2.4 M
// classes 1.65e-3 and 1.1e-4 either way), where two parts of g would be half as many products again; f32 in three parts as above.
// For f16, g is scaled by 2^14, which keeps g down to 2^-28 in f16's normal range.  dx's g is without the row's share, or with what of it lies in [0.5, 1); dweight's has
// it, as a part of the largest (finite) share of the rows that a workgroup sums, so that of f16 what lies 2^-28 below that one loses bits.
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
constexpr int kWaves = 8, kThreads = 64 * kWaves, kOwners = 32 * kWaves;      // rows that a workgroup owns
constexpr float kLog2e = 1.44269504088896340736f;
// exp(z - a) is formed as exp2(z log2(e) - a log2(e)), one operation beside the exponential; a log2(e) is rounded, which changes the exponent by up to 2^-24 of it: no more
// than a's own rounding does, but beyond 2^31 by more than the exponential's range.  From this size on a is taken from z first.
constexpr float kFar = 1024.0f;
constexpr int kFarLabel = RG_LOSS_MAX_CLASSES;              // a bit above all labels: of a row whose lse is far
__device__ __forceinline__ bool is_far(float a) { return fabsf(a) >= kFar && fabsf(a) < __builtin_inff(); }
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
// Them as parts.  TAIL: they may reach over the row's end.
template <bool TAIL, bool SHORT, typename T>
__device__ __forceinline__ void row_parts(const typename RgPack<T, 8>::type& raw, int col, int dim, Words4 (&w)[Part<T>::P]) {
    if constexpr (Part<T>::P == 1) {
        uint32_t x[4];
        __builtin_memcpy(x, &raw, 16);
        if (TAIL && (!SHORT || dim >= 8)) {                // what was loaded from `over` numbers further left moves down by as many, zeros after it
            const int over = col - min(col, dim - 8);
            if (dim % 8 != 0) {
                const bool four = over & 4, two = over & 2;
                x[0] = four ? x[2] : x[0];
                x[1] = four ? x[3] : x[1];
                x[2] = four ? 0 : x[2];
                x[3] = four ? 0 : x[3];
                x[0] = two ? x[1] : x[0];
                x[1] = two ? x[2] : x[1];
                x[2] = two ? x[3] : x[2];
                x[3] = two ? 0 : x[3];
                const uint32_t odd = 2 * (over & 1);
                x[0] = __builtin_amdgcn_alignbyte(x[1], x[0], odd);
                x[1] = __builtin_amdgcn_alignbyte(x[2], x[1], odd);
                x[2] = __builtin_amdgcn_alignbyte(x[3], x[2], odd);
                x[3] = __builtin_amdgcn_alignbyte(0, x[3], odd);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = over < 8 ? x[j] : 0;
        }
        w[0] = Words4{x[0], x[1], x[2], x[3]};
    } else {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = raw[j];
        if (TAIL && (!SHORT || dim >= 8)) rg_row_end<8>(v, col, dim);
        cut<T>(v, w);
    }
}

__device__ __forceinline__ bool has_label(int label, int classes) { return (uint32_t)label < (uint32_t)classes; }

// |share|, or 0 where it is not finite, and the power of two that brings it below 1.
__device__ __forceinline__ float finite_size(float share) { return fabsf(share) < __builtin_inff() ? fabsf(share) : 0.0f; }
__device__ __forceinline__ int power_of_two(float size) {
    int power = 0;
    if (size > 0.0f) (void)frexpf(size, &power);
    return power;
}

// The owned rows as the matrix units take them: [block of 32 rows][16 columns][part][lane][8 numbers], lane l the row l % 32 and the columns 8 (l / 32) .. + 7.
// Rows that are not there, or (labels given) do not count, are zeros.  For rows that are read again for every tile; bound by memory: 100 k rows of 128 f32, 22 us, 5.8 TB/s.
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
    const void* owned;         // the owned rows (held: as they are, `owned_stride` apart; else packed by k_pack_rows)
    int64_t owned_stride;
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

// Whether owned rows are held in registers: rows of 16-bit numbers, up to 128 of them (256 where there is no sum of as many columns beside them).
template <typename T>
constexpr bool held_rows(int mode, int steps) { return Part<T>::P == 1 && steps > 0 && (steps <= kSteps || (mode == LOSS && steps <= 2 * kSteps)); }

// STEPS: 16 columns each, of rows of up to 256 numbers; 0: any, in chunks of 128 columns.
// Bound by the matrix units, which the loss and dx keep busy 52 to 65 % of the cycles, dweight, whose workgroups walk 1024 rows and then load and store their own, 37 %, at the
// 1.65 to 2.1 GHz that the card's power leaves them (a large library product of
// bf16 reaches 1330 TFLOP/s): loss of 4096 rows of 256 f16 over 233 k classes 470-530 us, 920-1040 TFLOP/s; of 1024 rows of 100 bf16 over 2.4 M, dx 1000-1150 us and
// dweight 1350-1700, 870-1000 and 590-740 TFLOP/s of two products each (of 112 and 128 columns where rows have 100: a fifth more work); of 1024 rows of 128 f32 over
// 200 k, dx 510-575 and dweight 790-880, at six products of parts 1090-1230 and 710-800.  Two wavefronts a SIMD with 256 registers each: with three (32 walked rows) they spill; of two
// blocks of owned rows to a wavefront too.  Two workgroups of 4 wavefronts to a unit took 1342 us where one of 8 takes 1264; one tile between barriers 1260 where two
// take 1200; an order of priorities, deeper reads of fragments, another place of the loads or the first tiles loaded together changed nothing beyond 3 %.
template <typename T, int MODE, int NB, int STEPS>
__global__ void __launch_bounds__(kThreads, 2) k_softmax_rows(const Job job) {
    typedef Part<T> S;
    typedef typename S::type E;
    constexpr int P = S::P, ROWS = MODE == LOSS && STEPS == 0 ? 2 * S::ROWS : S::ROWS, SB = ROWS / 32, GROUPS = ROWS / 16;     // (owned rows are read again for every tile)
    // HOLD: the owned rows stay in registers.  PIPE: the exponentials of a tile are formed between the products of the next one's z, so that the vector and the
    // matrix units work side by side; for that the tile stays in LDS for its second product while two more arrive.
    constexpr bool HOLD = held_rows<T>(MODE, STEPS), PIPE = STEPS > 0 && (STEPS <= kSteps || HOLD);
    // PERIOD: tiles between barriers; LOOK: how far ahead of its second product a tile is staged.
    constexpr int CHUNKS = STEPS > kSteps ? 2 : 1, PERIOD = PIPE && CHUNKS == 1 ? 2 : 1, LOOK = 2 * PERIOD, BUFFERS = PERIOD == 2 ? 6 : PIPE && MODE != LOSS ? 3 : 2;
    constexpr int ITEMS = (STEPS > 0 && STEPS < kSteps ? STEPS / 2 * GROUPS + kWaves - 1 : 4 * GROUPS) / kWaves;
    __shared__ __attribute__((aligned(16))) char staged[BUFFERS][CHUNKS][P][ROWS * kRowBytes];
    __shared__ __attribute__((aligned(16))) float row_lse[BUFFERS][ROWS], row_share[BUFFERS][ROWS], row_both[BUFFERS][ROWS];
    __shared__ __attribute__((aligned(16))) int row_label[BUFFERS][ROWS];
    __shared__ float largest[kWaves];
    const int lane = rg_lane(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5;
    const int order = rg_xcd_block(blockIdx.x, gridDim.x), split = order / job.tiles, tile = order - split * job.tiles;
    const int64_t n_act = rg_rows(job.n, job.n_dev);
    const int64_t rows = MODE == DW ? n_act : job.rows, owners = MODE == DW ? job.owners : rg_least(job.owners, n_act - job.first);
    const int64_t first_owner = (int64_t)tile * kOwners;
    if (first_owner >= owners) return;
    const T* walked = (const T*)job.walked;
    const int dim = job.dim, steps = job.steps, chunks = job.chunks;

    // The walked tiles of this split, and (not PIPE) the stages of a tile: its chunks of 128 columns for z, the last of them one of this workgroup's output columns,
    // which it serves at once; then the other output columns' chunk.
    const int64_t all = (rows + ROWS - 1) / ROWS, per = (all + job.splits - 1) / job.splits, t0 = rg_least(split * per, all);
    const int tiles = (int)rg_least(per, all - t0), here = (int)(rows - t0 * ROWS);        // tiles, and rows from the first of them on
    constexpr int SLICE = NB / 4;
    const int slice = blockIdx.y * SLICE;
    const int more = MODE == LOSS ? 0 : min(SLICE, chunks - slice) - 1;
    const auto chunk_of = [&](int stage) __attribute__((always_inline)) {
        if (MODE == LOSS) return stage;
        if (stage >= chunks) return slice + stage - chunks + 1;
        const int c = slice + 1 + stage;
        return c >= chunks ? c - chunks : c;
    };

    // dweight: shares (finite ones) are scaled by a power of two to at most 1, and the sums back
    int power = 0;
    if (MODE == DW && job.dloss) {
        float top = 0.0f;
        for (int64_t r = t0 * ROWS + threadIdx.x; r < rg_least((t0 + tiles) * ROWS, rows); r += kThreads)
            if (has_label(job.labels[r], job.classes)) top = fmaxf(top, finite_size(job.dloss[r]));
        for (int off = 32; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, RG_WAVE));
        if (lane == 0) largest[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, largest[w]);
        power = power_of_two(top);
    }

    // what a lane's owned row brings
    const int64_t owner = first_owner + wave * 32 + (lane & 31);
    int label = -1;
    float lse2 = 0.0f, m = -__builtin_inff(), s = 0.0f, lost = 0.0f, base = 0.0f;
    bool far = false;                                      // DX: some row's lse is
    if (MODE != DW && owner < owners) {
        label = job.labels[owner];
        if (!has_label(label, job.classes)) label = -1;
        if (MODE == DX && label >= 0) {
            const float lse = job.lse[owner];
            far = is_far(lse);
            lse2 = (far ? 0.0f : lse * kLog2e) - (float)S::BIAS;
        }
    }
    if (MODE == DX) far = __any(far);
    const int told = label - (int)(t0 * ROWS);              // (the label among this split's rows; less than 0 if there is none)
    const Words4* owned = (const Words4*)job.owned + (first_owner / 32 + wave) * steps * (P * 64) + lane;
    Words4 held[HOLD ? STEPS : 1][P];
    if constexpr (HOLD) {                                  // (rows that are not there, or do not count, are zeros)
        const T* row = (const T*)job.owned + rg_least(owner, owners - 1) * job.owned_stride;
        const bool counts = owner < owners && (MODE != DX || label >= 0);
        typename RgPack<T, 8>::type raw[STEPS];
#pragma unroll
        for (int k = 0; k < STEPS; ++k) raw[k] = load_eight<STEPS == 2>(row, k * 16 + half * 8, dim);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            if (k + (STEPS > kSteps ? 4 : 2) >= STEPS) row_parts<true, STEPS == 2, T>(raw[k], k * 16 + half * 8, dim, held[k]);      // (where a row may end)
            else row_parts<false, false, T>(raw[k], k * 16 + half * 8, dim, held[k]);
            if (!counts) held[k][0] = Words4{0, 0, 0, 0};
        }
    }
    // dweight: whether one of the owned numbers is not finite (which times the zeros of a row that does not count is a NaN)
    bool odd = false;
    if constexpr (MODE == DW) {
        const uint32_t top = std::is_same<E, _Float16>::value ? 0x7C00u : 0x7F80u;
        const auto look = [&](const Words4& w) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < 4; ++j) odd |= (w[j] & top) == top || (w[j] >> 16 & top) == top;
        };
        if constexpr (HOLD) {
#pragma unroll
            for (int k = 0; k < STEPS; ++k) look(held[k][0]);
        } else {
#pragma unroll 8
            for (int k = 0; k < steps * P; ++k) look(owned[k * 64]);
        }
        odd = __any(odd);
    }

    // Staging: a wavefront's pieces of 16 rows by 32 columns (four lanes to a row), so that only the last columns' ones look for the rows' end.  Within a row's 16
    // pieces of 16 bytes the place is the column's exclusive or with four bits of the row: both ways of reading the tile (16 rows of one piece, 4 rows of
    // 4) then meet all 64 banks once a cycle, where three bits for 128 bytes took twice as long.
    // (Loads are made without a branch, of the last row where there is no other: registers that are written in some paths only are waited for where paths meet.)
    typename RgPack<T, 8>::type raw[CHUNKS][ITEMS];
    float next_lse = 0.0f, next_share = 0.0f;
    int next_label = -1, to_label = -1;
    const int to_row = wave % GROUPS * 16 + (lane >> 2), group0 = wave / GROUPS;          // (of 32 columns; item u: group0 + u * kWaves / GROUPS)
    const int to_at = to_row * kRowBytes + (((group0 * 4 + (lane & 3)) ^ ((to_row & 3) << 2 | (to_row >> 2 & 3))) << 4);
    const T *ahead = walked + (t0 * ROWS + to_row) * job.stride, *const last = walked + (rows - 1) * job.stride;
    const auto load = [&](int t, int first_chunk, bool first) __attribute__((always_inline)) {
        const T* src = ahead < last ? ahead : last;
        if (MODE == DW) to_label = job.labels[t0 * ROWS + min(t * ROWS + to_row, here - 1)];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int u = 0; u < ITEMS; ++u) {
                if (STEPS > 0 && c * kSteps + u * (kWaves / GROUPS) * 2 >= STEPS) continue;
                raw[c][u] = load_eight<STEPS == 2>(src, (first_chunk + c) * kCols + (group0 + u * (kWaves / GROUPS)) * 32 + (lane & 3) * 8, dim);
            }
        if (MODE == DW && first) {
            const int r = t * ROWS + (threadIdx.x & (ROWS - 1));
            const int64_t from = t0 * ROWS + min(r, here - 1);
            next_label = job.labels[from];
            next_lse = job.lse[from];
            next_share = job.dloss ? job.dloss[from] : 1.0f;
            if (r >= here) next_label = -1;
        }
    };
    const auto next_tile = [&]() __attribute__((always_inline)) { ahead += ROWS * job.stride; };
    const auto store = [&](int t, int first_chunk, int buffer, bool first, int place) __attribute__((always_inline)) {
        int dim = job.dim;
        asm volatile("" : "+s"(dim));                      // (else what depends on it is formed before the loop and takes registers through all of it)
        const bool counts = t * ROWS + to_row < here && (MODE != DW || has_label(to_label, job.classes)), whole = __all(counts);
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int u = 0; u < ITEMS; ++u) {
                if (STEPS > 0 && c * kSteps + u * (kWaves / GROUPS) * 2 >= STEPS) continue;
                const int chunk = first_chunk + c, group = group0 + u * (kWaves / GROUPS), col = chunk * kCols + group * 32 + (lane & 3) * 8;
                // (rows of STEPS steps end in the last two: in the last item's columns, if that)
                const bool may_end = STEPS == 0 || STEPS == 12 || STEPS == 16 || c * kSteps + (u + 1) * (kWaves / GROUPS) * 2 >= STEPS;
                Words4 w[P];
                if (may_end && chunk * kCols + group * 32 + 32 > dim) row_parts<true, STEPS == 2, T>(raw[c][u], col, dim, w);
                else row_parts<false, false, T>(raw[c][u], col, dim, w);
#pragma unroll
                for (int p = 0; p < P; ++p) *(Words4*)(staged[buffer][c][p] + (to_at ^ u * (kWaves / GROUPS) << 6)) = w[p];
            }
        if (!whole && !counts) {                           // (rows that do not count are zeros)
#pragma unroll
            for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
                for (int u = 0; u < ITEMS; ++u)
#pragma unroll
                    for (int p = 0; p < P; ++p) *(Words4*)(staged[buffer][c][p] + (to_at ^ u * (kWaves / GROUPS) << 6)) = Words4{0, 0, 0, 0};
        }
        if (MODE == DW && first && threadIdx.x < ROWS) {
            const bool live = has_label(next_label, job.classes);
            const float lse = live ? next_lse : 0.0f, share = live ? ldexpf(next_share, S::BIAS - power) : 0.0f;
            row_lse[place][threadIdx.x] = lse;
            row_share[place][threadIdx.x] = share;
            row_label[place][threadIdx.x] = live ? next_label | (is_far(lse) ? kFarLabel : 0) : -1;
            // share exp(z - lse) = exp2(z log2(e) - row_both); 0 where the share is
            row_both[place][threadIdx.x] = share > 0.0f ? lse * kLog2e - __builtin_amdgcn_logf(share) : __builtin_inff();
        }
    };

    Acc out[MODE == LOSS ? 1 : NB];
    Words4 g[MODE == LOSS ? 1 : SB][2][P];
    if (MODE != LOSS) {
#pragma unroll
        for (int d = 0; d < NB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) out[d][i] = 0.0f;
    }

    // z += the products of K steps of 16 columns.  Fragments of the walked rows are read RING - 1 products ahead, those of the owned rows, where they are not held,
    // a step or two; the barriers keep the compiler from reading all of them at once, for which there are no registers.  `between` has work for the vector units.
    constexpr int RING = P > 1 ? 2 : 4;
    const int walk_row = lane & 31, walk_at = walk_row * kRowBytes + ((half ^ ((walk_row & 3) << 2 | (walk_row >> 2 & 3))) << 4);
    const bool trim = dim <= (STEPS - 1) * 16;              // the last step has no numbers
    const auto products = [&](auto count, int chunk, int buffer, Acc (&z)[SB], auto between) __attribute__((always_inline)) {
        constexpr int K = decltype(count)::value, UNITS = K * SB, AHEAD = P == 1 ? 3 : 2;
        Words4 left[RING][P], right[AHEAD][P];
        const auto read = [&](int u) __attribute__((always_inline)) {
            const int k = u / SB, q = u % SB;
#pragma unroll
            for (int p = 0; p < P; ++p)
                left[u % RING][p] = *(const Words4*)(staged[buffer][CHUNKS > 1 ? k / kSteps : 0][p] + q * 32 * kRowBytes + (walk_at ^ k % kSteps << 5));
        };
        const auto fetch = [&](int k) __attribute__((always_inline)) {
#pragma unroll
            for (int p = 0; p < P; ++p) right[k % AHEAD][p] = owned[((int64_t)(chunk * kSteps + k) * P + p) * 64];
        };
        if constexpr (!HOLD) {
#pragma unroll
            for (int k = 0; k < AHEAD - 1; ++k)
                if (k < K) fetch(k);
        }
#pragma unroll
        for (int u = 0; u < RING - 1; ++u)
            if (u < UNITS) read(u);
#pragma clang loop unroll(full)                            // (whatever its size: of numbers in parts it is beyond the limit of a plain unroll)
        for (int u = 0; u < UNITS; ++u) {
            const int k = u / SB, q = u % SB;
            if (u + RING - 1 < UNITS) read(u + RING - 1);
            if constexpr (!HOLD) {
                if (q == 0 && k + AHEAD - 1 < K) fetch(k + AHEAD - 1);
            }
            if (STEPS == 0 || k + 1 < K || !trim) {
                if constexpr (HOLD) z[q] = mma_parts<E, P>(left[u % RING], held[HOLD ? k : 0], z[q]);
                else z[q] = mma_parts<E, P>(left[u % RING], right[k % AHEAD], z[q]);
            }
            between(u, UNITS);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    const auto nothing = [](int, int) __attribute__((always_inline)) {};
    const auto clear = [&](Acc (&z)[SB]) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < SB; ++q)
#pragma unroll
            for (int i = 0; i < 16; ++i) z[q][i] = 0.0f;
    };

    // out += g . the staged rows, for D blocks of 32 columns
    const int i16 = lane & 15, low_at = (4 * half + (i16 >> 2)) * kRowBytes + ((((lane >> 4 & 1) * 2 + (i16 >> 1 & 1)) ^ ((i16 >> 2) << 2 | half)) << 4) + (i16 & 1) * 8;
    const auto second = [&](auto base, auto count, int buffer, auto between) __attribute__((always_inline)) {
        constexpr int D0 = decltype(base)::value, D = decltype(count)::value, UNITS = SB * 2 * D;
        Words4 turned[RING][P];
        const auto read = [&](int u) __attribute__((always_inline)) {
            const int q = u / (2 * D), f = u / D % 2, d = u % D;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const char* at = staged[buffer][d / 4][p] + (q * 32 + f * 16) * kRowBytes;
                typedef __attribute__((address_space(3))) Short4 Lds;
                const Words2 low = __builtin_bit_cast(Words2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(at + (low_at ^ d % 4 << 6))));
                const Words2 high = __builtin_bit_cast(Words2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds*)(at + 8 * kRowBytes + (low_at ^ d % 4 << 6 ^ 2 << 4))));
                turned[u % RING][p] = Words4{low[0], low[1], high[0], high[1]};
            }
        };
#pragma unroll
        for (int u = 0; u < RING - 1; ++u)
            if (u < UNITS) read(u);
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            const int q = u / (2 * D), f = u / D % 2, d = u % D;
            if (u + RING - 1 < UNITS) read(u + RING - 1);
            out[D0 + d] = mma_parts<E, P>(turned[u % RING], g[q][f], out[D0 + d]);
            between(u, UNITS);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // z of a whole tile is there, register i of z[q] the walked row q * 32 + row_at(i) + 4 half.  What few tiles need (labels, the ends, a new maximum) stands in blocks
    // of its own that most pass by; side by side with the other path, each with its registers, it made the compiler spill.
    const auto row_at = [](int i) __attribute__((always_inline)) { return 8 * (i >> 2) + (i & 3); };
    const auto open_tile = [&](int t, int place, Acc (&z)[SB]) __attribute__((always_inline)) {
        if (MODE == DW) {
            const int seen = row_label[place][lane & (ROWS - 1)], mine = (int)(job.first + first_owner) + wave * 32;
            const float share = row_share[place][lane & (ROWS - 1)];
            return (bool)__any((seen >= mine && seen - mine < 32) || seen >= kFarLabel || !(share > 0.0f || (share == 0.0f && !odd)));
        }
        if ((t + 1) * ROWS > here) {                       // (behind the last class)
            int end = here - t * ROWS - 4 * half;
            asm volatile("" : "+v"(end));                  // (else the 32 rows that it is compared to are formed before the loop, and kept)
#pragma unroll
            for (int q = 0; q < SB; ++q)
#pragma unroll
                for (int i = 0; i < 16; ++i) z[q][i] = q * 32 + row_at(i) >= end ? -__builtin_inff() : z[q][i];
            __builtin_amdgcn_sched_barrier(0);
        }
        const bool met = told >= t * ROWS && told < (t + 1) * ROWS, hits = __any(met);
        if (MODE == LOSS) {
            if (hits) {
                int at = told - t * ROWS - 4 * half;       // (of this half's, if it equals one of them)
                asm volatile("" : "+v"(at));
                float there = 0.0f;
                bool mine = false;
#pragma unroll
                for (int q = 0; q < SB; ++q)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const bool is = at == q * 32 + row_at(i);
                        there = is ? z[q][i] : there;
                        mine |= is;
                    }
                if (met && mine) job.target[owner] = there;
                __builtin_amdgcn_sched_barrier(0);
            }
            // s is the sum of exp(z - m) with an m that need not be the maximum, but is within e^22 of it
            float top = z[0][0];
#pragma unroll
            for (int q = 0; q < SB; ++q)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, z[q][i]);
            if (__any(!(top - m < 22.0f))) {
                const float higher = fmaxf(m, top);
                if (m != -__builtin_inff()) {
                    const float factor = __builtin_amdgcn_exp2f((m - higher) * kLog2e);
                    s *= factor;
                    lost *= factor;
                }
                m = higher;
                __builtin_amdgcn_sched_barrier(0);
            }
            base = m == -__builtin_inff() || is_far(m) ? 0.0f : m * kLog2e;
        }
        if (MODE == LOSS ? __any(is_far(m)) : far) {
            float a = m;
            if (MODE == DX) a = label >= 0 ? job.lse[owner] : 0.0f;
            a = is_far(a) ? a : 0.0f;
#pragma unroll
            for (int q = 0; q < SB; ++q)
#pragma unroll
                for (int i = 0; i < 16; ++i) z[q][i] -= a;
            __builtin_amdgcn_sched_barrier(0);
        }
        return hits;
    };
    // LOSS: a tile's sum is added to s as a whole, and what s is too coarse for to `lost`: else what many classes have beside one that takes nearly all would be
    // rounded away a bit at a time, always downward (with each number added to s, of 233 k classes that have 0.6 % together, half of it was lost in one walk over all).
    // Rows of 256 f16 against 233 k classes 513 -> 529 us, of 100 bf16 against 2.4 M 714 -> 729, of 128 f32 against 200 k 302 -> 305.
    const auto add_sum = [&](const float (&sum)[4]) __attribute__((always_inline)) {
        const float x = (sum[0] + sum[1]) + (sum[2] + sum[3]), all = s + x, there = all - s;
        lost += (s - (all - there)) + (x - there);
        s = all;
    };
    // exp(z - m), or share g, of row i of z[q] ...
    const auto power_of = [&](float z, float both) __attribute__((always_inline)) {
        return __builtin_amdgcn_exp2f(__builtin_fmaf(z, kLog2e, MODE == LOSS ? -base : MODE == DX ? -lse2 : -both));
    };
    // ... and of the eight rows of z[q]'s half f in a tile that has labels here, or rows that do not count
    const auto mend = [&](int t, int place, const Acc (&z)[SB], int q, int f, float (&v)[8]) __attribute__((always_inline)) {
        if (MODE == DX) {
            int at = told - t * ROWS - 4 * half - q * 32 - f * 16;
            asm volatile("" : "+v"(at));
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] -= at == row_at(j) && told >= 0 ? (float)(1 << S::BIAS) : 0.0f;
        } else {
            const int mine = (int)(job.first + owner);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int row = q * 32 + f * 16 + row_at(j) + 4 * half;
                const float p = __builtin_amdgcn_exp2f((z[q][f * 8 + j] - row_lse[place][row]) * kLog2e), share = row_share[place][row];
                v[j] = share == 0.0f ? 0.0f : share * (p - ((row_label[place][row] & ~kFarLabel) == mine ? 1.0f : 0.0f));       // (nothing of a row that does not count, whatever its p is)
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    // the powers of a whole tile
    const auto powers = [&](int t, int place, Acc (&z)[SB]) __attribute__((always_inline)) {
        const bool rare = open_tile(t, place, z);
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int q = 0; q < SB; ++q)
#pragma unroll
            for (int f = 0; f < 2; ++f) {
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    v[j] = power_of(z[q][f * 8 + j], MODE == DW ? row_both[place][q * 32 + f * 16 + row_at(j) + 4 * half] : 0.0f);
                    if (MODE == LOSS) sum[j & 3] += v[j];
                }
                if (MODE != LOSS) {
                    if (rare) mend(t, place, z, q, f, v);
                    cut<T>(v, g[MODE == LOSS ? 0 : q][f]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        if (MODE == LOSS) add_sum(sum);
    };

#define RG_INT(N) std::integral_constant<int, N>()
    constexpr int FIRST = STEPS == 0 ? 4 : STEPS / 2;      // blocks of output columns
    if constexpr (PIPE) {
        // A tile: its exponentials beside the next one's products, its second product, the tile after the next one to LDS.  (Behind the last tile the products are of
        // what lies there, and are not used.)
        const auto turn = [&](int t, int now, Acc (&z)[SB], Acc (&next)[SB]) __attribute__((always_inline)) {
            const auto behind = [&](int k) __attribute__((always_inline)) { return now + k >= BUFFERS ? now + k - BUFFERS : now + k; };
            const int then = behind(1), free = behind(LOOK % BUFFERS);
            load(t + LOOK, 0, true);
            next_tile();
            const bool rare = open_tile(t, now, z);
            clear(next);
            float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f}, both[2][4], v[8];
            const auto read_both = [&](int e) __attribute__((always_inline)) {
#pragma unroll
                for (int j = 0; j < 4; ++j) both[e / 4 % 2][j] = row_both[now][e / 16 * 32 + row_at(e % 16) + 4 * half + j];
            };
            if (MODE == DW) read_both(0);
            const auto exponentials = [&](int from, int to) __attribute__((always_inline)) {
#pragma unroll
                for (int e = from; e < to; ++e) {
                    const int q = e / 16, i = e % 16;
                    if (MODE == DW && e % 4 == 0 && e + 4 < SB * 16) read_both(e + 4);
                    v[e % 8] = power_of(z[q][i], both[e / 4 % 2][e % 4]);
                    if (MODE == LOSS) sum[i & 3] += v[e % 8];
                    // (held here: the compiler would move them behind all products, where they are used)
                    if (MODE == LOSS) asm volatile("" : "+v"(sum[i & 3]));
                    else asm volatile("" : "+v"(v[e % 8]));
                    if (MODE != LOSS && e % 8 == 7) {
                        if (rare) mend(t, now, z, q, i / 8, v);
                        cut<T>(v, g[MODE == LOSS ? 0 : q][i / 8]);
                    }
                }
            };
            // half of them beside the products of the next z, half beside those of the first half
            constexpr int ALL = SB * 16, BEFORE = MODE == LOSS ? ALL : ALL / 2;
            products(RG_INT(STEPS), 0, then, next, [&](int u, int units) __attribute__((always_inline)) { exponentials(u * BEFORE / units, (u + 1) * BEFORE / units); });
            if (MODE == LOSS) add_sum(sum);
            if constexpr (MODE != LOSS)
                second(RG_INT(0), RG_INT(FIRST), now, [&](int u, int units) __attribute__((always_inline)) {
                    if (u < units / 2) exponentials(BEFORE + u * BEFORE / (units / 2), BEFORE + (u + 1) * BEFORE / (units / 2));
                });
            if (t + LOOK < tiles) store(t + LOOK, 0, free, true, free);
            return then;
        };
        Acc z[2][SB];
        int now = 0;
        if (tiles > 0) {
#pragma unroll 1
            for (int t = 0; t < LOOK; ++t) {
                load(t, 0, true);
                if (t < tiles) store(t, 0, t, true, t);
                next_tile();
            }
            __syncthreads();
            clear(z[0]);
            products(RG_INT(STEPS), 0, 0, z[0], nothing);
            if (BUFFERS == 2) __syncthreads();             // (the first turn's store takes the first tile's place)
        }
#pragma unroll 1
        for (int t = 0; t < tiles; t += 2) {
            now = turn(t, now, z[0], z[1]);
            if (PERIOD == 1) __syncthreads();
            if (t + 1 < tiles) now = turn(t + 1, now, z[1], z[0]);
            __syncthreads();
        }
    } else if constexpr (STEPS > 0) {
        // A tile after the other, the next one's rows on their way: z, powers, second product.  (Sums for 256 output columns leave no registers for a second z.)
        Acc z[SB];
        if (tiles > 0) {
            load(0, 0, true);
            next_tile();
            store(0, 0, 0, true, 0);
            __syncthreads();
        }
#pragma unroll 1
        for (int t = 0; t < tiles; ++t) {
            const int buffer = t & 1;
            clear(z);
            products(RG_INT(STEPS), 0, buffer, z, nothing);
            load(t + 1, 0, true);                          // (behind the products of z, which leave no registers for them)
            next_tile();
            powers(t, buffer, z);
            if constexpr (MODE != LOSS) second(RG_INT(0), RG_INT(FIRST), buffer, nothing);
            if (t + 1 < tiles) store(t + 1, 0, buffer ^ 1, true, buffer ^ 1);
            __syncthreads();
        }
    } else {
        Acc z[SB];
        const auto add_products = [&](int chunk, int buffer) __attribute__((always_inline)) {
            const int here = steps - chunk * kSteps;
            // (of numbers in parts a chunk's sum apart: to a long row's z the products of small parts would add nothing)
            Acc apart[SB];
            Acc(&to)[SB] = P > 1 ? apart : z;
            if (P > 1) clear(apart);
            if (here > 6) products(RG_INT(8), chunk, buffer, to, nothing);
            else if (here > 4) products(RG_INT(6), chunk, buffer, to, nothing);
            else if (here > 2) products(RG_INT(4), chunk, buffer, to, nothing);
            else products(RG_INT(2), chunk, buffer, to, nothing);
            if (P > 1) {
#pragma unroll
                for (int q = 0; q < SB; ++q)
#pragma unroll
                    for (int i = 0; i < 16; ++i) z[q][i] += apart[q][i];
            }
        };
        if (tiles > 0) {
            load(0, chunk_of(0), true);
            store(0, chunk_of(0), 0, true, 0);
            __syncthreads();
        }
        int buffer = 0;
#pragma unroll 1
        for (int t = 0; t < tiles; ++t) {
            const int place = t & 1;
            clear(z);
#pragma unroll 1
            for (int stage = 0; stage < chunks - 1; ++stage) {
                load(t, chunk_of(stage + 1), false);
                add_products(chunk_of(stage), buffer);
                store(t, chunk_of(stage + 1), buffer ^ 1, false, 0);
                __syncthreads();
                buffer ^= 1;
            }
            // (the next rows are asked for behind the products of z, which leave no registers for them)
            const bool rest = NB > 4 && more > 0, go_on = t + 1 < tiles;
            add_products(chunk_of(chunks - 1), buffer);
            powers(t, place, z);
            if (!rest) next_tile();
            load(rest ? t : t + 1, rest ? chunk_of(chunks) : chunk_of(0), !rest);
            if constexpr (MODE != LOSS) second(RG_INT(0), RG_INT(4), buffer, nothing);
            if (rest || go_on) store(rest ? t : t + 1, rest ? chunk_of(chunks) : chunk_of(0), buffer ^ 1, !rest, place ^ 1);
            __syncthreads();
            buffer ^= 1;
            if constexpr (MODE != LOSS && NB > 4) {
                if (rest) {
                    next_tile();
                    load(t + 1, chunk_of(0), true);
                    second(RG_INT(4), RG_INT(4), buffer, nothing);
                    if (go_on) store(t + 1, chunk_of(0), buffer ^ 1, true, place ^ 1);
                    __syncthreads();
                    buffer ^= 1;
                }
            }
        }
    }
#undef RG_INT

    if constexpr (MODE == LOSS) {
        s += lost;
        const float other_m = __shfl_xor(m, 32, RG_WAVE), other_s = __shfl_xor(s, 32, RG_WAVE);
        const float top = fmaxf(m, other_m), from = top == -__builtin_inff() ? 0.0f : top;
        const float sum = s * __builtin_amdgcn_exp2f((m - from) * kLog2e) + other_s * __builtin_amdgcn_exp2f((other_m - from) * kLog2e);
        if (half == 0 && owner < owners) job.stats[split * job.owners + owner] = make_float2(top, sum);
    } else {
        if (owner >= owners) return;
        float factor = job.scale;
        const bool none = MODE == DX && label < 0;
        if (MODE == DX && !none && job.dloss) factor *= job.dloss[owner];
#pragma unroll
        for (int d = 0; d < NB; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int col = (slice * 4 + d) * 32 + i * 8 + half * 4;
                if (col >= dim) continue;
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[j] = out[d][i * 4 + j] * factor;
                    if (MODE == DW || S::BIAS) v[j] = ldexpf(v[j], power - S::BIAS);
                    if (none) v[j] = 0.0f;
                }
                if (job.splits == 1) rg_store_live<4>((T*)job.out + owner * job.out_stride + col, dim - col, v);
                else rg_store_live<4>(job.parts + (split * job.owners + owner) * dim + col, dim - col, v);
            }
    }
}

// Each row's log-sum and loss from its splits, a wavefront to a row.  5 us: a launch and two reads one behind the other.
__global__ void __launch_bounds__(64) k_loss_join(const float2* __restrict__ stats, int splits, int64_t first, int64_t count, int64_t n,
                                                  const int32_t* __restrict__ n_dev, const int32_t* __restrict__ labels, int classes,
                                                  const float* __restrict__ target, float* __restrict__ loss, float* __restrict__ lse) {
    const int64_t row = blockIdx.x;
    if (row >= rg_least(count, rg_rows(n, n_dev) - first)) return;
    float m = -__builtin_inff(), s = 0.0f;
    const auto merge = [&](float other_m, float other_s) {
        const float top = fmaxf(m, other_m), base = top == -__builtin_inff() ? 0.0f : top;
        s = s * __builtin_amdgcn_exp2f((m - base) * kLog2e) + other_s * __builtin_amdgcn_exp2f((other_m - base) * kLog2e);
        m = top;
    };
    constexpr int AHEAD = 4;
    for (int k0 = rg_lane(); k0 < splits; k0 += 64 * AHEAD) {
        float2 part[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) part[u] = stats[(int64_t)min(k0 + 64 * u, splits - 1) * count + row];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (k0 + 64 * u < splits) merge(part[u].x, part[u].y);
    }
    for (int off = 32; off > 0; off >>= 1) merge(__shfl_xor(m, off, RG_WAVE), __shfl_xor(s, off, RG_WAVE));
    if (rg_lane() != 0) return;
    const bool counts = has_label(labels[row], classes);
    const float sum = m + logf(s);
    if (lse) lse[row] = counts ? sum : 0.0f;
    if (loss) loss[row] = counts ? sum - target[row] : 0.0f;
}

// Sums of the splits' parts, in one order: RUNS runs of them side by side, 64 chunks of four columns to a workgroup.  Bound by memory and the reads' latency: 256 parts of
// 47 rows of 256 (12 MB) 8 us, 64 of 1024 rows of 128 (34 MB) 12 us.
template <typename T, int RUNS, bool SHORT>
__global__ void __launch_bounds__(64 * RUNS) k_grad_join(const float* __restrict__ parts, int splits, int64_t rows, int64_t first, int64_t n,
                                                         const int32_t* __restrict__ n_dev, int dim, int chunks, T* __restrict__ out, int64_t stride) {
    constexpr int V = 4;
    __shared__ float sums[RUNS][64][V];
    const int64_t total = rg_least(rows, rg_rows(n, n_dev) - first) * chunks, one = rows * dim;
    const int lane = threadIdx.x & 63, run = threadIdx.x >> 6, each = (splits + RUNS - 1) / RUNS, from = run * each, to = min(from + each, splits);
    for (int64_t i0 = (int64_t)blockIdx.x * 64; i0 < total; i0 += (int64_t)gridDim.x * 64) {
        const int64_t i = i0 + lane, row = rg_least(i, total - 1) / chunks;
        const int col = (int)(rg_least(i, total - 1) - row * chunks) * V;
        const float* part = parts + row * dim;
        float sum[V] = {0.0f, 0.0f, 0.0f, 0.0f};
        constexpr int AHEAD = 8;
        for (int k0 = from; k0 < to; k0 += AHEAD) {
            typename RgPack<float, V>::type v[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) v[u] = SHORT ? rg_load_raw<V>(part + min(k0 + u, to - 1) * one, dim) : rg_load_row<V>(part + min(k0 + u, to - 1) * one, col, dim);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (k0 + u >= to) break;
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] += v[u][j];
            }
        }
        if (!SHORT) rg_row_end<V>(sum, col, dim);
        if constexpr (RUNS > 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) sums[run][lane][j] = sum[j];
            __syncthreads();
            if (run == 0) {
#pragma unroll
                for (int r = 1; r < RUNS; ++r)
#pragma unroll
                    for (int j = 0; j < V; ++j) sum[j] += sums[r][lane][j];
            }
        }
        if (run == 0 && i < total) rg_store_live<V>(out + row * stride + col, dim - col, sum);
        if constexpr (RUNS > 1) __syncthreads();
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

// ---------------------------------------------------------------- few classes
// Up to 64 classes, whose weight rows fit LDS beside a tile of R rows of x: a workgroup walks its rows once, each tile z, g, dx and its share of dweight, so that x is
// read and dx written once and z is formed once.  z is [class][row] (rows along the lanes); g goes through LDS, from where dx's product reads it by rows and
// dweight's transposed.  Outputs go to the wavefronts by blocks of 32 columns; dweight's sums stay in registers until the end, then a second launch joins the workgroups'.
// 1024 rows of 256 f32 over 41 classes 7.2 us (the general kernel and its two companions: 21); gradients of 100 k rows of 256 f32 over 47 classes 92 us, 2.2 TB/s read and
// written: products of three parts, cutting rows into them and the barriers between a tile's steps take turns (four wavefronts instead of eight: 119; the general kernel: 429).
template <int P, int FORMS, int R, int CHUNKS>
struct FewLds {
    static constexpr int ROW = CHUNKS * kRowBytes, G_ROW = 128;
    char weight[P][64 * ROW], x[P][R * ROW], g[FORMS][P][R * G_ROW];
    float top[2][R], sum[2][R], target[R];
    float largest[8], smallest[8];
};
static_assert(sizeof(FewLds<3, 1, 32, 2>) <= 160 * 1024 && sizeof(FewLds<3, 1, 64, 1>) <= 160 * 1024 && sizeof(FewLds<1, 2, 32, 4>) <= 160 * 1024, "LDS of a compute unit");

struct FewJob {
    const void *x, *weight;
    int64_t x_stride, weight_stride, n;
    const int32_t *n_dev, *labels;
    const float *lse, *dloss;
    int dim, classes;
    float scale;
    float *loss, *log_sum;     // LOSS
    void* dx;                  // else; may be NULL
    int64_t dx_stride;
    float* parts;              // [workgroup][class][dim], or NULL
};

constexpr int kClassWaves = 8, kClassThreads = 64 * kClassWaves;

template <typename T, bool GRAD, int R, int CHUNKS>
__global__ void __launch_bounds__(kClassThreads, 2) k_few_classes(const FewJob job) {
    typedef Part<T> S;
    typedef typename S::type E;
    constexpr int FORMS = GRAD && S::BIAS ? 2 : 1;         // of g
    typedef FewLds<S::P, FORMS, R, CHUNKS> Lds;
    constexpr int P = S::P, ROW = Lds::ROW, RB = R / 32, ROWGROUPS = R / 16, ITEMS = ROWGROUPS * CHUNKS * 4 / kClassWaves;
    __shared__ __attribute__((aligned(16))) Lds lds;
    const int lane = rg_lane(), wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5, i16 = lane & 15;
    const int64_t n_act = rg_rows(job.n, job.n_dev);
    const int64_t all = (n_act + R - 1) / R, per = (all + gridDim.x - 1) / gridDim.x, t0 = rg_least(blockIdx.x * per, all);
    const int tiles = (int)rg_least(per, all - t0), here = (int)(n_act - t0 * R), dim = job.dim, classes = job.classes;
    const int steps = 2 * ((dim + 31) / 32), blocks = (dim + 31) / 32;
    if (!GRAD && tiles == 0) return;

    const auto twist = [](int row) __attribute__((always_inline)) { return (row & 3) << 2 | (row >> 2 & 3); };
    const auto g_twist = [](int row) __attribute__((always_inline)) { return (row >> 1 & 1) << 2 | (row >> 2 & 3); };
    // 16 rows by 32 columns of a staged matrix: four lanes to a row
    const auto put = [&](char* const (&plane)[P], const typename RgPack<T, 8>::type& raw, int row, int group, bool counts) __attribute__((always_inline)) {
        Words4 w[P];
        const int col = group * 32 + (lane & 3) * 8;
        if (group * 32 + 32 > dim) row_parts<true, false, T>(raw, col, dim, w);
        else row_parts<false, false, T>(raw, col, dim, w);
        const int piece = group * 4 + (lane & 3);
#pragma unroll
        for (int p = 0; p < P; ++p) *(Words4*)(plane[p] + row * ROW + ((piece ^ twist(row)) << 4)) = counts ? w[p] : Words4{0, 0, 0, 0};
    };
    char *weight_planes[P], *x_planes[P];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        weight_planes[p] = lds.weight[p];
        x_planes[p] = lds.x[p];
    }
    // the next tile's rows, on their way while one is worked on
    typename RgPack<T, 8>::type raw[ITEMS];
    int raw_label = -1;
    const T* x = (const T*)job.x;
    const int to_row = wave % ROWGROUPS * 16 + (lane >> 2), group0 = wave / ROWGROUPS;   // (of 32 columns; item u: group0 + u * kClassWaves / ROWGROUPS)
    const auto load = [&](int t) __attribute__((always_inline)) {
        const int64_t from = t0 * R + min(t * R + to_row, here - 1);
        raw_label = job.labels[from];
        const T* src = x + from * job.x_stride;
#pragma unroll
        for (int u = 0; u < ITEMS; ++u) raw[u] = load_eight<false>(src, (group0 + u * (kClassWaves / ROWGROUPS)) * 32 + (lane & 3) * 8, dim);
    };
    if (tiles > 0) load(0);
    // Shares to at most 1, as above, which dweight's products take with g.  dx's rows go by their own shares: where those of this workgroup's rows are so far apart that
    // g loses bits with the power of two that they have in common (of f16, any), dx gets a g of its own, each row with its own power.  Of f16 both lie in LDS, and wavefronts
    // that would be idle form z and the other g; else there is no room, and dweight's is formed when dx is done.  Powers of two change no bits, so that a row's dx is the
    // same whatever other rows have.  100 k rows of 256 over 47 classes, without shares, with shares of [0, 2), and with some 2^60 below: f32
    // 86, 88 and 109 us, bf16 48, 49 and 62, f16 48, 55 and 55.
    int power = 0;
    bool apart = false;
    if (GRAD && job.dloss) {
        float top = 0.0f, least = __builtin_inff();
        for (int64_t r = t0 * R + threadIdx.x; r < rg_least((t0 + tiles) * R, n_act); r += kClassThreads)
            if (has_label(job.labels[r], classes)) {
                const float size = finite_size(job.dloss[r]);
                top = fmaxf(top, size);
                least = size > 0.0f ? fminf(least, size) : least;
            }
        for (int off = 32; off > 0; off >>= 1) {
            top = fmaxf(top, __shfl_xor(top, off, RG_WAVE));
            least = fminf(least, __shfl_xor(least, off, RG_WAVE));
        }
        if (lane == 0) {
            lds.largest[wave] = top;
            lds.smallest[wave] = least;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kClassWaves; ++w) {
            top = fmaxf(top, lds.largest[w]);
            least = fminf(least, lds.smallest[w]);
        }
        power = power_of_two(top);
        apart = job.dx && (S::BIAS || ldexpf(least, 30 - power) < 1.0f);
    }
    for (int group = wave / 4; group < blocks; group += kClassWaves / 4) {
        const int row = wave % 4 * 16 + (lane >> 2);
        const T* src = (const T*)job.weight + (int64_t)min(row, classes - 1) * job.weight_stride;
        put(weight_planes, load_eight<false>(src, group * 32 + (lane & 3) * 8, dim), row, group, row < classes);
    }

    Acc dw[GRAD ? CHUNKS : 1];                             // unit u = wave + 8 j: columns u / 2 * 32 .., classes u % 2 * 32 ..
    if (GRAD) {
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) dw[j][i] = 0.0f;
    }
    // fragments: rows l % 32 of a block, 16 columns of step k; and, transposed, 16 rows from `first` on of 32 columns
    const int row_at = (lane & 31) * ROW + ((half ^ twist(lane & 31)) << 4);
    const int turned_at = (8 * half + (i16 >> 2)) * ROW + ((((lane >> 4 & 1) * 2 + (i16 >> 1 & 1)) ^ ((i16 >> 2) << 2 | 2 * half)) << 4) + (i16 & 1) * 8;
    typedef __attribute__((address_space(3))) Short4 Lds4;
    const auto turned = [&](const char* plane, int first, int d) __attribute__((always_inline)) {
        const char* at = plane + first * ROW + (d >> 2) * kRowBytes;
        const Words2 low = __builtin_bit_cast(Words2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4*)(at + (turned_at ^ (d & 3) << 6))));
        const Words2 high = __builtin_bit_cast(Words2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4*)(at + 4 * ROW + (turned_at ^ (d & 3) << 6 ^ 1 << 4))));
        return Words4{low[0], low[1], high[0], high[1]};
    };

    for (int t = 0; t < tiles; ++t) {
        __syncthreads();                                   // (the tile before is done with)
        int label[RB], own_power[RB];
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            const int r = t * R + b * 32 + (lane & 31);
            label[b] = job.labels[t0 * R + min(r, here - 1)];
            own_power[b] = apart ? power_of_two(finite_size(job.dloss[t0 * R + min(r, here - 1)])) : power;
            if (r >= here || !has_label(label[b], classes)) label[b] = -1;
        }
        const bool counts = t * R + to_row < here && has_label(raw_label, classes);
#pragma unroll
        for (int u = 0; u < ITEMS; ++u) {
            const int group = group0 + u * (kClassWaves / ROWGROUPS);
            if (group < blocks) put(x_planes, raw[u], to_row, group, counts);
        }
        load(t + 1);                                       // (of the last row, behind the last tile)
        __syncthreads();

        // z: a wavefront's block of 32 classes by 32 rows, of numbers in three parts half of its steps, which the other half's wavefront adds
        const int cb = wave & 1, rb = RB == 2 ? wave >> 1 & 1 : 0, part = wave >> RB, mine = RB == 1 ? label[0] : rb ? label[RB - 1] : label[0];
        const bool second_form = FORMS == 2 && apart && part == 1;
        constexpr int HALVES = P > 1 ? 2 : 1;
        Acc z;
        if (part < HALVES || second_form) {
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = 0.0f;
            const int middle = HALVES == 2 ? steps / 4 * 2 : steps, from = HALVES == 2 ? part * middle : 0, to = part == 0 ? middle : steps;
            for (int k0 = from; k0 < to; k0 += 2) {        // (an even number of them)
                Words4 a[2][P], b[2][P];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int p = 0; p < P; ++p) {
                        const int at = (k0 >> 3) * kRowBytes + (row_at ^ ((k0 & 7) + i) << 5);
                        a[i][p] = *(const Words4*)(lds.weight[p] + cb * 32 * ROW + at);
                        b[i][p] = *(const Words4*)(lds.x[p] + rb * 32 * ROW + at);
                    }
#pragma unroll
                for (int i = 0; i < 2; ++i) z = mma_parts<E, P>(a[i], b[i], z);
            }
        }
        if constexpr (HALVES == 2) {                       // by way of the place of g, which the tile before is done with
            float* const place = (float*)lds.g + (rb * 2 + cb) * 16 * 64 + lane;
            if (part == 1) {
#pragma unroll
                for (int i = 0; i < 16; ++i) place[i * 64] = z[i];
            }
            __syncthreads();
            if (part == 0) {
#pragma unroll
                for (int i = 0; i < 16; ++i) z[i] += place[i * 64];
            }
            __syncthreads();
        }
        const int first = cb * 32 + 4 * half;              // register i: class first + 8 (i >> 2) + (i & 3)
        const auto put_g = [&](int form, int scale_power) __attribute__((always_inline)) {         // share g, to LDS
            const int64_t row = t0 * R + t * R + min(rb * 32 + (lane & 31), here - 1 - t * R);
            const float lse = mine >= 0 ? job.lse[row] : 0.0f, share = mine >= 0 ? ldexpf(job.dloss ? job.dloss[row] : 1.0f, S::BIAS - scale_power) : 0.0f;
            const bool idle = mine < 0 || share == 0.0f;
            float v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int c = first + 8 * (i >> 2) + (i & 3);
                const float p = __builtin_amdgcn_exp2f((z[i] - lse) * kLog2e);
                v[i] = idle || c >= classes ? 0.0f : share * (p - (c == mine ? 1.0f : 0.0f));
            }
            const int at = rb * 32 + (lane & 31);
#pragma unroll
            for (int i = 0; i < 16; i += 8) {
                float eight[8];
                Words4 w[P];
#pragma unroll
                for (int j = 0; j < 8; ++j) eight[j] = v[i + j];
                cut<T>(eight, w);
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        *(Words2*)(lds.g[form][p] + at * Lds::G_ROW + (((cb * 4 + i / 4 + j) ^ g_twist(at)) << 4) + half * 8) = Words2{w[p][2 * j], w[p][2 * j + 1]};
            }
        };
        if (part == 0 || second_form) {
            if constexpr (!GRAD) {
                float top = -__builtin_inff(), there = 0.0f;
                bool met = false;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int c = first + 8 * (i >> 2) + (i & 3);
                    z[i] = c < classes ? z[i] : -__builtin_inff();
                    top = fmaxf(top, z[i]);
                    there = c == mine ? z[i] : there;
                    met |= c == mine;
                }
                top = fmaxf(top, __shfl_xor(top, 32, RG_WAVE));
                const float base = top == -__builtin_inff() ? 0.0f : top;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 16; ++i) sum += __builtin_amdgcn_exp2f((z[i] - base) * kLog2e);
                sum += __shfl_xor(sum, 32, RG_WAVE);
                const int at = rb * 32 + (lane & 31);
                if (half == 0) {
                    lds.top[cb][at] = top;
                    lds.sum[cb][at] = sum;
                }
                if (met) lds.target[at] = there;
            } else put_g(second_form ? 1 : 0, second_form ? power : RB == 1 ? own_power[0] : rb ? own_power[RB - 1] : own_power[0]);
        }
        __syncthreads();
        if constexpr (!GRAD) {
            if (threadIdx.x < R && t * R + (int)threadIdx.x < here) {
                const float m0 = lds.top[0][threadIdx.x], m1 = lds.top[1][threadIdx.x], top = fmaxf(m0, m1), base = top == -__builtin_inff() ? 0.0f : top;
                // (classes whose z are all NaN have a maximum of -infinity, and a NaN as their sum, which stays one; where there are none, the sum is 0)
                const float sum = lds.sum[0][threadIdx.x] * __builtin_amdgcn_exp2f((m0 - base) * kLog2e) + lds.sum[1][threadIdx.x] * __builtin_amdgcn_exp2f((m1 - base) * kLog2e);
                const int64_t row = t0 * R + t * R + threadIdx.x;
                const bool counts = has_label(job.labels[row], classes);
                const float lse = top + logf(sum);
                if (job.log_sum) job.log_sum[row] = counts ? lse : 0.0f;
                if (job.loss) job.loss[row] = counts ? lse - lds.target[threadIdx.x] : 0.0f;
            }
        } else {
            if (job.dx) {
                constexpr int UNITS = RB == 2 ? CHUNKS : (CHUNKS + 1) / 2;
#pragma unroll
                for (int j = 0; j < UNITS; ++j) {
                    const int unit = wave + kClassWaves * j, d = RB == 2 ? unit >> 1 : unit, b = RB == 2 ? unit & 1 : 0, at = b * 32 + (lane & 31);
                    if (d >= blocks) continue;
                    Acc out;
#pragma unroll
                    for (int i = 0; i < 16; ++i) out[i] = 0.0f;
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        Words4 a[P], g[P];
#pragma unroll
                        for (int p = 0; p < P; ++p) {
                            a[p] = turned(lds.weight[p], f * 16, d);
                            g[p] = *(const Words4*)(lds.g[0][p] + at * Lds::G_ROW + (((2 * f + half) ^ g_twist(at)) << 4));
                        }
                        out = mma_parts<E, P>(a, g, out);
                    }
                    const int r = t * R + at, mine = RB == 2 ? (b ? label[RB - 1] : label[0]) : label[0];
                    if (r >= here) continue;
                    T* to = (T*)job.dx + (t0 * R + r) * job.dx_stride;
                    const float factor = mine < 0 ? 0.0f : job.scale;
                    const int back = (RB == 2 ? (b ? own_power[RB - 1] : own_power[0]) : own_power[0]) - S::BIAS;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int col = d * 32 + q * 8 + half * 4;
                        if (col >= dim) continue;
                        float v[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[i] = mine < 0 ? 0.0f : ldexpf(out[q * 4 + i] * factor, back);
                        rg_store_live<4>(to + col, dim - col, v);
                    }
                }
            }
            if (job.parts) {
                const auto& shared = lds.g[FORMS == 2 && apart ? 1 : 0];
                if (FORMS == 1 && apart) {
                    __syncthreads();
                    if (part == 0) put_g(0, power);
                    __syncthreads();
                }
#pragma unroll
                for (int j = 0; j < CHUNKS; ++j) {
                    const int unit = wave + kClassWaves * j, d = unit >> 1, c = unit & 1;
                    if (d >= blocks) continue;
                    Acc here;                              // (of a tile; added to those before in the vector units, see kLongestWalk)
#pragma unroll
                    for (int i = 0; i < 16; ++i) here[i] = 0.0f;
#pragma unroll
                    for (int f = 0; f < R / 16; ++f) {
                        const int row = f * 16 + 8 * half + (i16 >> 2), piece = c * 4 + (lane >> 4 & 1) * 2 + (i16 >> 1 & 1);
                        Words4 a[P], g[P];
#pragma unroll
                        for (int p = 0; p < P; ++p) {
                            a[p] = turned(lds.x[p], f * 16, d);
                            const Words2 low = __builtin_bit_cast(Words2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                (Lds4*)(shared[p] + row * Lds::G_ROW + ((piece ^ g_twist(row)) << 4) + (i16 & 1) * 8)));
                            const Words2 high = __builtin_bit_cast(Words2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                (Lds4*)(shared[p] + (row + 4) * Lds::G_ROW + ((piece ^ g_twist(row + 4)) << 4) + (i16 & 1) * 8)));
                            g[p] = Words4{low[0], low[1], high[0], high[1]};
                        }
                        here = mma_parts<E, P>(a, g, here);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) dw[j][i] += here[i];
                }
            }
        }
    }
    if constexpr (GRAD) {
        if (!job.parts) return;
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            const int unit = wave + kClassWaves * j, own = (unit & 1) * 32 + (lane & 31);
            if (own >= classes) continue;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int col = (unit >> 1) * 32 + q * 8 + half * 4;
                if (col >= dim) continue;
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = ldexpf(dw[j][q * 4 + i] * job.scale, power - S::BIAS);
                rg_store_live<4>(job.parts + ((int64_t)blockIdx.x * classes + own) * dim + col, dim - col, v);
            }
        }
    }
}

// Whether the kernel above takes rows of `dim` numbers, and its launch.  Both sides of the line, 64 and 65 classes, rows of 256: loss of 1024 f32 8 and 21.5 us, of 100 k
// bf16 19 and 52; gradients of 1024 f32 15 and 95, of 100 k f32 90 and 451, of 100 k bf16 50 and 123; rows of 100, 100 k f32 52 and 167.  (f32 rows beyond 128 numbers fill LDS
// with 64 classes.  For the others more classes would fit; the kernel has two blocks of them.)
constexpr int kFewClasses = 64;
template <typename T>
bool few_classes(int classes, int dim) { return classes <= kFewClasses && dim >= 8 && dim <= (Part<T>::P > 1 ? 256 : 512); }
// Rows of a tile: 64, or 32 where LDS or registers do not suffice.
template <typename T>
int few_rows(int dim) { return dim > (Part<T>::P > 1 ? kCols : 2 * kCols) ? 32 : 64; }

template <typename T, bool GRAD>
void launch_few(const FewJob& job, unsigned grid, hipStream_t s) {
    const int chunks = (int)rg_div_up(job.dim, kCols);
    if constexpr (Part<T>::P > 1) {
        if (chunks == 1) k_few_classes<T, GRAD, 64, 1><<<grid, kClassThreads, 0, s>>>(job);
        else k_few_classes<T, GRAD, 32, 2><<<grid, kClassThreads, 0, s>>>(job);
    } else {
        if (chunks == 1) k_few_classes<T, GRAD, 64, 1><<<grid, kClassThreads, 0, s>>>(job);
        else if (chunks == 2) k_few_classes<T, GRAD, 64, 2><<<grid, kClassThreads, 0, s>>>(job);
        else if (chunks == 3) k_few_classes<T, GRAD, 32, 3><<<grid, kClassThreads, 0, s>>>(job);
        else k_few_classes<T, GRAD, 32, 4><<<grid, kClassThreads, 0, s>>>(job);
    }
}

// ---------------------------------------------------------------- few rows
// The loss of up to 32 rows against many classes: the weight is read once, by every wavefront for itself, 32 classes at a time straight into the matrix units' registers
// (x's rows, 16-bit parts of them, stay in LDS).  A lane takes 16 neighbouring columns at a time, two steps' worth: the order of the columns is free as
// long as both operands have the same.  Bound by memory: one row of 100 bf16 against 2.4 M classes 97 us, 5.1 TB/s (the general kernel, which packs rows and stages the weight: 196).
constexpr int kFewWaves = 8;

template <typename T>
__global__ void __launch_bounds__(64 * kFewWaves, 2) k_few_rows(const T* __restrict__ x, int64_t x_stride, int n, const int32_t* __restrict__ n_dev, int dim, int pairs,
                                                                const T* __restrict__ weight, int64_t weight_stride, int classes, const int32_t* __restrict__ labels,
                                                                float2* __restrict__ stats, float* __restrict__ target) {
    typedef typename Part<T>::type E;
    constexpr int P = Part<T>::P, AHEAD = P == 1 ? 4 : 2;
    extern __shared__ __attribute__((aligned(16))) Words4 rows[];          // [pair of steps][step][part][lane]
    __shared__ float tops[kFewWaves][32], sums[kFewWaves][32];
    const int n_act = (int)rg_rows(n, n_dev), lane = rg_lane(), wave = threadIdx.x >> 6, half = lane >> 5, row = lane & 31;
    const auto parts_of = [&](const T* src, int col, bool counts, Words4 (&w)[P]) __attribute__((always_inline)) {
        const typename RgPack<T, 8>::type raw = load_eight<false>(src, col, dim);
        if (col + 8 > dim) row_parts<true, false, T>(raw, col, dim, w);
        else row_parts<false, false, T>(raw, col, dim, w);
        if (!counts) {
#pragma unroll
            for (int p = 0; p < P; ++p) w[p] = Words4{0, 0, 0, 0};
        }
    };
    for (int k = wave; k < 2 * pairs; k += kFewWaves) {
        Words4 w[P];
        parts_of(x + (int64_t)min(row, max(n_act - 1, 0)) * x_stride, (k >> 1) * 32 + half * 16 + (k & 1) * 8, row < n_act, w);
#pragma unroll
        for (int p = 0; p < P; ++p) rows[(k * P + p) * 64 + lane] = w[p];
    }
    const int label = row < n_act && has_label(labels[row], classes) ? labels[row] : -1;
    __syncthreads();
    float m = -__builtin_inff(), s = 0.0f;
    const int blocks = (classes + 31) / 32, step = gridDim.x * kFewWaves;
    for (int block = blockIdx.x * kFewWaves + wave; block < blocks; block += step) {
        const T* src = weight + (int64_t)min(block * 32 + row, classes - 1) * weight_stride;
        Acc z;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0.0f;
        for (int k0 = 0; k0 < pairs; k0 += AHEAD) {
            typename RgPack<T, 8>::type raw[AHEAD][2];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int j = 0; j < 2; ++j) raw[u][j] = load_eight<false>(src, min(k0 + u, pairs - 1) * 32 + half * 16 + j * 8, dim);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (k0 + u >= pairs) break;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    Words4 a[P], b[P];
                    const int col = (k0 + u) * 32 + half * 16 + j * 8;
                    if (k0 + u + 1 == pairs) row_parts<true, false, T>(raw[u][j], col, dim, a);
                    else row_parts<false, false, T>(raw[u][j], col, dim, a);
#pragma unroll
                    for (int p = 0; p < P; ++p) b[p] = rows[(((k0 + u) * 2 + j) * P + p) * 64 + lane];
                    z = mma_parts<E, P>(a, b, z);
                }
            }
        }
        const int first = block * 32 + 4 * half;           // register i: class first + 8 (i >> 2) + (i & 3)
        if (block * 32 + 32 > classes) {
#pragma unroll
            for (int i = 0; i < 16; ++i) z[i] = first + 8 * (i >> 2) + (i & 3) < classes ? z[i] : -__builtin_inff();
        }
        if (__any(label >= block * 32 && label < block * 32 + 32)) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (label == first + 8 * (i >> 2) + (i & 3)) target[row] = z[i];
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, z[i]);
        const float base = top == -__builtin_inff() ? 0.0f : top;
        s *= __builtin_amdgcn_exp2f((m - base) * kLog2e);
#pragma unroll
        for (int i = 0; i < 16; ++i) s += __builtin_amdgcn_exp2f((z[i] - base) * kLog2e);
        m = top;
    }
    const auto merge = [&](float other_m, float other_s) __attribute__((always_inline)) {
        const float top = fmaxf(m, other_m), base = top == -__builtin_inff() ? 0.0f : top;
        s = s * __builtin_amdgcn_exp2f((m - base) * kLog2e) + other_s * __builtin_amdgcn_exp2f((other_m - base) * kLog2e);
        m = top;
    };
    merge(__shfl_xor(m, 32, RG_WAVE), __shfl_xor(s, 32, RG_WAVE));
    if (half == 0) {
        tops[wave][row] = m;
        sums[wave][row] = s;
    }
    __syncthreads();
    if (threadIdx.x >= 32) return;
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) merge(tops[w][row], sums[w][row]);
    if (row < n_act) stats[(int64_t)blockIdx.x * n + row] = make_float2(m, s);
}

// Whether the kernel above takes the call: its rows as parts lie in LDS (16 KB at 256 numbers of 16 bits).  Both sides of the line, 32 and 33 rows of 128 numbers: against
// 200000 classes 31 and 72 us of f32, 17 and 22 of bf16; against 65, 11 and 16 of f32, 10 and 10 of bf16.
constexpr int kFewRows = 32;
template <typename T>
bool few_rows_many_classes(int64_t n, int dim) { return n <= kFewRows && dim >= 8 && rg_div_up(dim, 32) * 2 * Part<T>::P * 1024 <= 60 * 1024; }

bool aligned(const void* p, int bytes) { return (uintptr_t)p % (uintptr_t)bytes == 0; }

constexpr int64_t kMostRows = (1ll << 31) - 1;

// Columns of a row as steps of 16, an even number of them (12 or 16 from 129 columns on, as the kernel holds them).
int steps_of(int dim) {
    const int steps = 2 * (int)rg_div_up(dim, 32);
    return steps <= 8 || steps > 16 ? steps : steps <= 12 ? 12 : 16;
}

// Rows of f32 that a split walks, for a gradient, at most.  To a sum that has grown the matrix units add less and less of the products of small parts, nothing beyond 2^16 steps
// of 16 rows of like size: in walks of 60 k, 200 k and 1 M rows of one sign the sums were off by 3e-5, 1.2e-4 and 1.2e-3 of themselves, in these by 1e-5, 1.7e-5 and 2.5e-5.
// (Sums formed apart, step by step, do not fit the registers.)
constexpr int64_t kLongestWalk = 4096;

int64_t packed_row(int steps, int parts) { return (int64_t)steps * parts * 32; }

// Rows that are owned at a time: their packed form stays in the last level of cache; held ones' sums and targets do (LOSS), or the launch has fewer than 2^32 threads.
int64_t piece_rows(int64_t rows, int steps, int parts, bool held = false) {
    const int64_t most = held ? 1 << 22 : rg_max64(1, (128ll << 20) / packed_row(steps, parts) / kOwners) * kOwners, pieces = rg_div_up(rows, most);
    return rg_div_up(rg_div_up(rows, pieces), kOwners) * kOwners;
}

template <typename T>
void pack(rg_ctx* ctx, const void* x, int64_t stride, int64_t first, int64_t count, int64_t n, const int32_t* n_dev, int dim, int steps, const int32_t* labels,
          int classes, void* packed, hipStream_t s) {
    const int64_t units = rg_div_up(count, kOwners) * (kOwners / 32) * steps;
    k_pack_rows<T><<<(unsigned)rg_min64(rg_div_up(units, 4), (int64_t)ctx->num_cus * 32), 256, 0, s>>>((const T*)x, stride, first, n, n_dev, dim, steps, labels, classes,
                                                                                                 units, (Words4*)packed);
}

template <typename T>
void join_parts(rg_ctx* ctx, const float* parts, int splits, int64_t rows, int64_t first, int64_t n, const int32_t* n_dev, int dim, T* out, int64_t stride, hipStream_t s) {
    const int quads = (int)rg_div_up(dim, 4);
    const unsigned grid = (unsigned)rg_min64(rg_div_up(rows * quads, 64), (int64_t)ctx->num_cus * 32);
    const int runs = splits >= 32 ? 16 : 4;
    const auto kernel = dim < 4 ? k_grad_join<T, 4, true> : runs == 4 ? k_grad_join<T, 4, false> : k_grad_join<T, 16, false>;
    kernel<<<grid, dim < 4 ? 256 : 64 * runs, 0, s>>>(parts, splits, rows, first, n, n_dev, dim, quads, out, stride);
}

// Splits of the walked rows: as many workgroups as there are compute units, one to each (two to each, with half as many owned rows and 4 wavefronts, took 1342 us
// instead of 1264 for dx of 1024 rows of 100 against 2.4 M), or a multiple of that where a split would be longer than `longest` rows (which count in 31 bits).
int splits_for(rg_ctx* ctx, int64_t workgroups, int64_t walked, int64_t longest) {
    const int64_t fit = rg_max64(1, rg_min64(rg_div_up(walked, 64), ctx->num_cus / workgroups)), least = rg_div_up(walked, longest);
    return (int)(rg_div_up(least, fit) * fit);
}

rg_status check_loss(rg_ctx* ctx, const char* who, const void* x, rg_dtype type, int64_t x_stride, int64_t n, int32_t dim, const void* weight,
                     int64_t weight_stride, int32_t classes, const int32_t* labels, const float* lse) {
    RG_REQUIRE(ctx, n >= 0 && n <= kMostRows, "%s: n = %lld out of range", who, (long long)n);
    RG_REQUIRE(ctx, dim >= 1 && dim <= RG_LOSS_MAX_DIM, "%s: dim = %d not in [1,%d]", who, dim, RG_LOSS_MAX_DIM);
    RG_REQUIRE(ctx, classes >= 1 && classes <= RG_LOSS_MAX_CLASSES, "%s: classes = %d not in [1,%d]", who, classes, RG_LOSS_MAX_CLASSES);
    RG_REQUIRE(ctx, rg_type_known(type), "%s: unknown type %d", who, (int)type);
    RG_REQUIRE(ctx, x_stride >= dim && weight_stride >= dim, "%s: bad stride", who);
    RG_REQUIRE(ctx, n == 0 || (x && weight && labels), "%s: null pointer", who);
    const int b = rg_type_bytes(type);
    RG_REQUIRE(ctx, aligned(x, b) && aligned(weight, b) && aligned(labels, 4) && aligned(lse, 4), "%s: pointer not aligned to its numbers", who);
    return RG_OK;
}

// The kernel for a job.
template <typename T, int MODE>
void launch(const Job& job, int64_t slices, hipStream_t s) {
    const dim3 grid((unsigned)((int64_t)job.tiles * job.splits), (unsigned)slices);
    switch (job.steps) {
        case 2: k_softmax_rows<T, MODE, 4, 2><<<grid, kThreads, 0, s>>>(job); break;
        case 4: k_softmax_rows<T, MODE, 4, 4><<<grid, kThreads, 0, s>>>(job); break;
        case 6: k_softmax_rows<T, MODE, 4, 6><<<grid, kThreads, 0, s>>>(job); break;
        case 8: k_softmax_rows<T, MODE, 4, 8><<<grid, kThreads, 0, s>>>(job); break;
        case 12: k_softmax_rows<T, MODE, 8, 12><<<grid, kThreads, 0, s>>>(job); break;
        case 16: k_softmax_rows<T, MODE, 8, 16><<<grid, kThreads, 0, s>>>(job); break;
        default: k_softmax_rows<T, MODE, 8, 0><<<grid, kThreads, 0, s>>>(job);
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
        if (few_classes<T>(classes, dim)) {
            FewJob job = {};
            job.x = x;
            job.weight = weight;
            job.x_stride = x_stride;
            job.weight_stride = weight_stride;
            job.n = n;
            job.n_dev = n_dev;
            job.labels = labels;
            job.dim = dim;
            job.classes = classes;
            job.loss = loss;
            job.log_sum = lse;
            launch_few<T, false>(job, (unsigned)rg_min64(rg_div_up(n, few_rows<T>(dim)), (int64_t)ctx->num_cus * 2), s);
            RG_LAUNCH_CHECK(ctx, "k_few_classes");
            return RG_OK;
        }
        if (few_rows_many_classes<T>(n, dim)) {
            const int pairs = (int)rg_div_up(dim, 32), grid = (int)rg_min64(rg_div_up(classes, 32 * kFewWaves), (int64_t)ctx->num_cus * 2);
            const rg_status st = rg_scratch(ctx, ctx->loss_parts, (size_t)grid * n * sizeof(float2) + kFewRows * 4, s, "rg_cross_entropy");
            if (st != RG_OK) return st;
            float2* stats = (float2*)ctx->loss_parts.p;
            float* target = (float*)(stats + (int64_t)grid * n);
            k_few_rows<T><<<grid, 64 * kFewWaves, pairs * 2 * P * 1024, s>>>((const T*)x, x_stride, (int)n, n_dev, dim, pairs, (const T*)weight, weight_stride, classes,
                                                                             labels, stats, target);
            RG_LAUNCH_CHECK(ctx, "k_few_rows");
            k_loss_join<<<(unsigned)n, 64, 0, s>>>(stats, grid, 0, n, n, n_dev, labels, classes, target, loss, lse);
            RG_LAUNCH_CHECK(ctx, "k_loss_join");
            return RG_OK;
        }
        const int steps = steps_of(dim);
        const bool held = held_rows<T>(LOSS, steps);
        const int64_t piece = piece_rows(n, steps, P, held), most = rg_min64(piece, n), tiles = rg_div_up(most, kOwners);
        const int splits = splits_for(ctx, tiles, classes, 1 << 30);
        const size_t packed = held ? 0 : (size_t)(tiles * kOwners * packed_row(steps, P)), stats = (size_t)splits * most * sizeof(float2);
        const rg_status st = rg_scratch(ctx, ctx->loss_parts, packed + stats + (size_t)most * 4, s, "rg_cross_entropy");
        if (st != RG_OK) return st;
        char* at = (char*)ctx->loss_parts.p;
        Job job = {};
        job.owned_stride = x_stride;
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
            job.owned = held ? (const void*)((const T*)x + first * x_stride) : at;
            if (!held) pack<T>(ctx, x, x_stride, first, count, n, n_dev, dim, steps, nullptr, classes, at, s);
            job.owners = count;
            job.first = first;
            job.tiles = (int)rg_div_up(count, kOwners);
            job.labels = labels + first;
            launch<T, LOSS>(job, 1, s);
            RG_LAUNCH_CHECK(ctx, "k_softmax_rows");
            k_loss_join<<<(unsigned)count, 64, 0, s>>>(job.stats, splits, first, count, n, n_dev, job.labels, classes, job.target,
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
    RG_REQUIRE(ctx, (!dx || (dx != x && dx != weight && dx != dweight)) && (!dweight || (dweight != x && dweight != weight)),
               "rg_cross_entropy_grad: an output is an input, or the other output");
    const int b = rg_type_bytes(type);
    RG_REQUIRE(ctx, aligned(dx, b) && aligned(dweight, b) && aligned(dloss, 4), "rg_cross_entropy_grad: pointer not aligned to its numbers");
    if (!dweight && (!dx || n == 0)) return RG_OK;
    RG_HIP(ctx, hipSetDevice(ctx->device));
    hipStream_t s = (hipStream_t)stream;
    RG_FOR_TYPE(type, {
        constexpr int P = Part<T>::P;
        if (n == 0) {
            const int pieces = (int)rg_div_up(dim, 16 / (int)sizeof(T));
            k_zero_rows<T><<<(unsigned)rg_min64(rg_div_up((int64_t)classes * pieces, 256), (int64_t)ctx->num_cus * 32), 256, 0, s>>>((T*)dweight, dweight_stride, classes,
                                                                                                                     dim, pieces);
            RG_LAUNCH_CHECK(ctx, "k_zero_rows");
            return RG_OK;
        }
        if (few_classes<T>(classes, dim)) {
            const int64_t tiles = rg_div_up(n, few_rows<T>(dim)), grid = rg_min64(tiles, ctx->num_cus);
            if (dweight) {
                const rg_status st = rg_scratch(ctx, ctx->loss_parts, (size_t)grid * classes * dim * 4, s, "rg_cross_entropy_grad");
                if (st != RG_OK) return st;
            }
            FewJob job = {};
            job.x = x;
            job.weight = weight;
            job.x_stride = x_stride;
            job.weight_stride = weight_stride;
            job.n = n;
            job.n_dev = n_dev;
            job.labels = labels;
            job.lse = lse;
            job.dloss = dloss;
            job.dim = dim;
            job.classes = classes;
            job.scale = scale;
            job.dx = dx;
            job.dx_stride = dx_stride;
            job.parts = dweight ? (float*)ctx->loss_parts.p : nullptr;
            launch_few<T, true>(job, (unsigned)grid, s);
            RG_LAUNCH_CHECK(ctx, "k_few_classes");
            if (dweight) {
                join_parts<T>(ctx, job.parts, (int)grid, classes, 0, classes, nullptr, dim, (T*)dweight, dweight_stride, s);
                RG_LAUNCH_CHECK(ctx, "k_grad_join");
            }
            return RG_OK;
        }
        const int steps = steps_of(dim), chunks = (int)rg_div_up(dim, kCols);
        const int64_t slices = rg_div_up(chunks, 2);       // (a workgroup's output: up to two chunks of columns)
        const bool held = held_rows<T>(DX, steps);
        struct Side {
            int64_t rows, piece, most, tiles;
            int splits;
            size_t packed, parts;
        };
        const auto side = [&](int64_t rows, int64_t walked) {
            Side v;
            v.rows = rows;
            v.piece = piece_rows(rows, steps, P, held);
            // (of longer walks: as long as parts of a gigabyte allow, the owned rows in smaller pieces for them)
            const int64_t room = (1ll << 28) / dim, longest = P == 1 ? 1 << 30 : rg_max64(kLongestWalk, rg_div_up(walked, rg_max64(1, room / kOwners)));
            if (walked > longest) v.piece = rg_min64(v.piece, rg_max64(1, room / rg_div_up(walked, longest) / kOwners) * kOwners);
            v.most = rg_min64(v.piece, rows);
            v.tiles = rg_div_up(v.most, kOwners);
            v.splits = splits_for(ctx, v.tiles * slices, walked, longest);
            v.packed = held ? 0 : (size_t)(v.tiles * kOwners * packed_row(steps, P));
            v.parts = v.splits > 1 ? (size_t)v.splits * v.most * dim * 4 : 0;
            return v;
        };
        const Side for_dx = side(n, classes), for_dw = side(classes, n);
        const size_t dx_bytes = dx ? for_dx.packed + for_dx.parts : 0, dw_bytes = dweight ? for_dw.packed + for_dw.parts : 0;
        const rg_status st = rg_scratch(ctx, ctx->loss_parts, dx_bytes > dw_bytes ? dx_bytes : dw_bytes, s, "rg_cross_entropy_grad");
        if (st != RG_OK) return st;
        char* at = (char*)ctx->loss_parts.p;
        Job job = {};
        job.n = n;
        job.n_dev = n_dev;
        job.dim = dim;
        job.steps = steps;
        job.chunks = chunks;
        job.classes = classes;
        job.scale = scale;
        const auto take = [&](const Side& v, int64_t first, const void* owned, int64_t owned_stride, void* out, int64_t stride) {
            job.owned = held ? (const void*)((const T*)owned + first * owned_stride) : at;
            job.owned_stride = owned_stride;
            job.owners = rg_min64(v.piece, v.rows - first);
            job.first = first;
            job.tiles = (int)rg_div_up(job.owners, kOwners);
            job.splits = v.splits;
            job.parts = (float*)(at + v.packed);
            job.out = (T*)out + first * stride;
            job.out_stride = stride;
        };
        const auto join = [&](int64_t rows, const int32_t* count) {
            if (job.splits > 1) join_parts<T>(ctx, job.parts, job.splits, job.owners, job.first, rows, count, dim, (T*)job.out, job.out_stride, s);
        };
        for (int64_t first = 0; dx && first < n; first += for_dx.piece) {
            take(for_dx, first, x, x_stride, dx, dx_stride);
            if (!held) pack<T>(ctx, x, x_stride, first, job.owners, n, n_dev, dim, steps, labels, classes, at, s);
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
            take(for_dw, first, weight, weight_stride, dweight, dweight_stride);
            if (!held) pack<T>(ctx, weight, weight_stride, first, job.owners, classes, nullptr, dim, steps, nullptr, 0, at, s);
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
