// Packed rows of 4-bit numbers with a scale per group of 32 (the layout is the header's): to and from numbers, their product with a
// packed weight, and the gradient of that product to its weight.
#include "rg_elements.h"

#include <type_traits>

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

typedef uint32_t rg_u32x4a __attribute__((ext_vector_type(4)));
constexpr int kGroup = 32;
constexpr uint32_t kScaleNan = 255;

constexpr int kLdsBytes = 160 * 1024;                       // that a workgroup may have

// Between a wavefront's stores to LDS and its other lanes' loads of them (and the other way round): the memory's order is that of the instructions, so that
// nothing is waited for, but only the fences keep the compiler to it.
__device__ __forceinline__ void wave_exchange() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// The scale byte as the float with this exponent: what the conversion instructions read the exponent of (0 stands for 2^-127 and
// 255 for "not a number" to them, as in the format).
__device__ __forceinline__ float scale_bits(uint32_t s) { return __uint_as_float(s << 23); }

// ---------------------------------------------------------------- numbers to packed rows
// s = max(0, E - 2) with E the exponent byte of a group's largest magnitude, codes the numbers times 2^(127 - s), rounded to the nearest of the eight
// magnitudes (halves to the even code, what is beyond 6 to 6).  Bound by memory: 2.4 M rows of 100 floats, 980 MB in and 167 MB out, packed into rows 20
// words apart and unpacked again in turn, take 257 us (4.5 TB/s).  What is stored leaves holes behind rows of less than whole words of 16 bytes, which costs
// more than the bytes: packed again and again 278 us, 213 into rows 17 words apart (of bf16 182 and 171).
// A lane takes 16 bytes of a row (4 numbers of 32 bits, 8 of 16), so that a wavefront's loads and stores are one run of bytes; U pieces a thread
// are on their way together (with one 537 instead of 464 us for these rows and back).  The largest magnitude of a group, as an integer
// (so that NaN and infinities are the largest of all), goes round its 8 or 4 lanes; the numbers times 2^(127 - s), which is exact or far below the smallest magnitude, are rounded by the conversion instruction.
constexpr int kPiecesAhead = 4;

template <int CTRL>
__device__ __forceinline__ uint32_t max_with(uint32_t x) { return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xF, 0xF, false)); }

template <typename T>
__global__ void __launch_bounds__(256) k_mx4_quantize(const T* __restrict__ x, int64_t x_stride, int64_t n, const int32_t* __restrict__ n_dev,
                                                      int dim, uint32_t* __restrict__ packed, int64_t packed_stride, int pieces, uint32_t inv_pieces,
                                                      int rows_per_block) {
    constexpr int V = 16 / sizeof(T), U = kPiecesAhead;
    const int64_t n_act = rg_rows(n, n_dev);
    const int groups = (dim + kGroup - 1) / kGroup;
    for (int64_t row0 = (int64_t)blockIdx.x * rows_per_block; row0 < n_act; row0 += (int64_t)gridDim.x * rows_per_block) {
    const int items = (int)rg_least(rows_per_block, n_act - row0) * pieces;      // a multiple of a group's lanes: groups are in one wavefront
    for (int it0 = threadIdx.x; it0 < items; it0 += 256 * U) {
        float v[U][V];
        int r[U], piece[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int it = it0 + 256 * u;
            r[u] = (int)rg_divide((uint32_t)it, inv_pieces);
            piece[u] = it - r[u] * pieces;
            if (it < items) rg_load_head<V>(x + (row0 + r[u]) * x_stride + piece[u] * V, dim - piece[u] * V, v[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (it0 + 256 * u >= items) break;
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(v[u][i]) & 0x7FFFFFFFu);
            top = max_with<0xB1>(top);                     // lanes 1, 0, 3, 2 of four; 2, 3, 0, 1; of eight the other four
            top = max_with<0x4E>(top);
            if (V == 4) top = max_with<0x141>(top);
            const uint32_t e = top >> 23;
            const bool good = e < 255;
            const uint32_t s = good ? (e > 2 ? e - 2 : 0) : kScaleNan;
            const float f = __uint_as_float((254u - s) << 23);
            uint32_t word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, v[u][0] * f, v[u][1] * f, 1.0f, 0);
            word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[u][2] * f, v[u][3] * f, 1.0f, 1);
            if constexpr (V == 8) {
                word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[u][4] * f, v[u][5] * f, 1.0f, 2);
                word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[u][6] * f, v[u][7] * f, 1.0f, 3);
            }
            if (!good) word = 0;
            uint32_t* row = packed + (row0 + r[u]) * packed_stride;
            if constexpr (V == 8) row[piece[u]] = word;
            else ((uint16_t*)row)[piece[u]] = (uint16_t)word;
            constexpr int LANES = kGroup / V;
            if (piece[u] % LANES == 0) {
                const int group = piece[u] / LANES;
                uint8_t* scales = (uint8_t*)(row + 4 * groups);
                scales[group] = (uint8_t)s;
                if (group == groups - 1)
                    for (int i = groups; i & 3; ++i) scales[i] = 0;
            }
        }
    }
    }
}

// ---------------------------------------------------------------- packed rows to numbers
// A lane makes 16 bytes of a row, from codes and a scale that the conversion instruction multiplies exactly (two neighbouring numbers at a time).
// Bound by what it stores: 2.4 M rows of 100 floats, 167 MB in and 980 MB out, 207 us (5.5 TB/s).
template <typename T, bool ONCE>
__global__ void __launch_bounds__(256) k_mx4_dequantize(const uint32_t* __restrict__ packed, int64_t packed_stride, int64_t n,
                                                        const int32_t* __restrict__ n_dev, int dim, T* __restrict__ x, int64_t x_stride, int pieces,
                                                        uint32_t inv_pieces, int rows_per_block) {
    constexpr int V = 16 / sizeof(T), U = kPiecesAhead;
    typedef float v2f __attribute__((ext_vector_type(2)));
    const int64_t n_act = rg_rows(n, n_dev);
    const int groups = (dim + kGroup - 1) / kGroup;
    for (int64_t row0 = (int64_t)blockIdx.x * rows_per_block; row0 < n_act; row0 += (int64_t)gridDim.x * rows_per_block) {
    const int items = (int)rg_least(rows_per_block, n_act - row0) * pieces;
    for (int it0 = threadIdx.x; it0 < items; it0 += 256 * U) {
        uint32_t code[U], scale[U];
        int r[U], piece[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int it = min(it0 + 256 * u, items - 1);
            r[u] = (int)rg_divide((uint32_t)it, inv_pieces);
            piece[u] = it - r[u] * pieces;
            const uint32_t* row = packed + (row0 + r[u]) * packed_stride;
            code[u] = V == 8 ? row[piece[u]] : ((const uint16_t*)row)[piece[u]];
            scale[u] = ((const uint8_t*)(row + 4 * groups))[piece[u] / (kGroup / V)];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (it0 + 256 * u >= items) break;
            const float s = scale_bits(scale[u]);
            float v[V];
            const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u], s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u], s, 1);
            v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y;
            if constexpr (V == 8) {
                const v2f c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u], s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[u], s, 3);
                v[4] = c.x; v[5] = c.y; v[6] = d.x; v[7] = d.y;
            }
            rg_store_live<V, ONCE>(x + (row0 + r[u]) * x_stride + piece[u] * V, dim - piece[u] * V, v);
        }
    }
    }
}

// Rows to a workgroup of 256 threads when each is `pieces` pieces: kPiecesAhead to a thread where that makes four workgroups or more for every
// compute unit, else one (rows of 100 floats: 2.4 M of them packed and back in 464 us, 537 with one to a thread; 40 k 11.6 and 14.0; 1024 rows of 602
// f16 5.0 and 3.3 to pack).
int rows_per_group(const rg_ctx* ctx, int64_t n, int pieces) {
    const int64_t full = 256 * kPiecesAhead;
    return (int)rg_max64(1, (n * pieces >= (int64_t)ctx->num_cus * 4 * full ? full : 256) / pieces);
}
// Workgroups for n rows, `rows` at a time (a launch has less than 2^32 threads).
unsigned row_groups(int64_t n, int rows) { return (unsigned)rg_min64(rg_div_up(n, rows), 1 << 23); }

// ---------------------------------------------------------------- y = rows . weight^T
// A wavefront makes a tile of 16 R rows by 16 C outputs with the scaled 16 x 16 x 128 matrix instruction: lane 16 q + c holds group
// 4 k + q of row c in step k, 16 bytes of codes and their scale byte, as they lie in the packed row.  The weight is the first operand,
// so that a lane ends up with four neighbouring outputs of one row.  Groups behind the row's last are zeros; rows and outputs beyond
// the last read the last one's and are not stored.
// <1, 1>: few rows, a tile to a wavefront and as many wavefronts as can be; bound by the latency of a launch and two loads (1 row of 602 numbers times 41
// outputs 3.1 us, 1024 rows of 256 times 256 as well).  <2, 4>: rows too long to be kept; bound by the weight's traffic from L2.
template <typename T, int R, int C>
__global__ void __launch_bounds__(256) k_mx4_matmul(const uint32_t* __restrict__ rows, int64_t rows_stride, int64_t n,
                                                    const int32_t* __restrict__ n_dev, const uint32_t* __restrict__ weight,
                                                    int64_t weight_stride, int out_dim, int groups, T* __restrict__ y, int64_t y_stride) {
    const int64_t n_act = rg_rows(n, n_dev);
    const int lane = rg_lane(), c = lane & 15, q = lane >> 4;
    const int steps = (groups + 3) >> 2;
    const int64_t wave = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 6;
    const int64_t waves = ((int64_t)gridDim.x * blockDim.x) >> 6;
    for (int64_t row0 = wave * (16 * R); row0 < n_act; row0 += waves * (16 * R)) {
    const uint32_t* xrow[R];
#pragma unroll
    for (int r = 0; r < R; ++r) xrow[r] = rows + rg_least(row0 + 16 * r + c, n_act - 1) * rows_stride;
    for (int h0 = blockIdx.y * (16 * C); h0 < out_dim; h0 += gridDim.y * (16 * C)) {
        const uint32_t* wrow[C];
#pragma unroll
        for (int t = 0; t < C; ++t) wrow[t] = weight + (int64_t)min(h0 + 16 * t + c, out_dim - 1) * weight_stride;
        v4f acc[R][C];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int t = 0; t < C; ++t) acc[r][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
        for (int k = 0; k < steps; ++k) {
            const int g = 4 * k + q;
            const bool live = g < groups;
            v8i a[C], b[R];
            uint32_t as[C], bs[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                rg_u32x4 w = {0u, 0u, 0u, 0u};
                if (live) w = *(const rg_u32x4*)(xrow[r] + 4 * g);
                bs[r] = live ? (xrow[r][4 * groups + k] >> (8 * q)) & 255u : 127u;
                b[r] = v8i{(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
            }
#pragma unroll
            for (int t = 0; t < C; ++t) {
                rg_u32x4 w = {0u, 0u, 0u, 0u};
                if (live) w = *(const rg_u32x4*)(wrow[t] + 4 * g);
                as[t] = live ? (wrow[t][4 * groups + k] >> (8 * q)) & 255u : 127u;
                a[t] = v8i{(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int t = 0; t < C; ++t)
                    acc[r][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a[t], b[r], acc[r][t], 4, 4, 0, (int)as[t], 0, (int)bs[r]);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = row0 + 16 * r + c;
            if (row >= n_act) continue;
#pragma unroll
            for (int t = 0; t < C; ++t) {
                const int h = h0 + 16 * t + 4 * q;
                const float v[4] = {acc[r][t][0], acc[r][t][1], acc[r][t][2], acc[r][t][3]};
                rg_store_live<4>(y + row * y_stride + h, out_dim - h, v);
            }
        }
    }
    }
}

// The same for many rows: a wavefront keeps the weight of 16 FRAGS outputs (STEPS of 128 numbers) in registers and goes over tiles of 16
// rows, whose codes are loaded a tile ahead; a workgroup's wavefronts share rows (through L1) where there are outputs for them, and take
// different rows where there are not.  Bound by memory: 794 k rows of 256 numbers times 256 outputs of bf16, 515 MB in and out, take 99 us (5.2 TB/s; 104
// GFLOP in that time are a tenth of the matrix unit's peak for 4 bits).  Results go by way of LDS, so that a wavefront's stores cover whole lines: stored as
// the matrix unit leaves them, 64 bytes of a row at a time, they took half as long again (176 us and 126 in an earlier form).  The weight kept in LDS
// instead of registers: 125 us.  Where rows of y follow each other without a gap and end inside 16 bytes (`run_on`), a tile is stored as one run.
constexpr int kKeptThreads = 256, kKeptWaves = kKeptThreads / RG_WAVE;

template <typename T, int STEPS, int FRAGS, bool ONCE>
__global__ void __launch_bounds__(kKeptThreads, STEPS > 5 ? 2 : 1) k_mx4_matmul_kept(
    const uint32_t* __restrict__ rows, int64_t rows_stride, int64_t n, const int32_t* __restrict__ n_dev, const uint32_t* __restrict__ weight,
    int64_t weight_stride, int out_dim, int groups, T* __restrict__ y, int64_t y_stride, int slices, int slice_groups, int run_on,
    uint32_t inv_last) {
    constexpr bool WIDE = sizeof(T) == 4;
    constexpr int OUTS = 16 * FRAGS, E = 16 / sizeof(T), PITCH = OUTS * (int)sizeof(T) + 16;   // numbers in 16 bytes; bytes of a row in LDS
    __shared__ rg_u32x4a stage[kKeptWaves][PITCH];
    const int64_t n_act = rg_rows(n, n_dev);
    const int lane = rg_lane(), c = lane & 15, q = lane >> 4;
    const int wave = threadIdx.x >> 6;
    // `slices` (1, 2 or 4) times OUTS outputs to a workgroup, slice_groups workgroups side by side on the same rows
    const int block = rg_xcd_block(blockIdx.x, gridDim.x);
    const int h0 = ((block % slice_groups) * slices + wave % slices) * OUTS;
    if (h0 >= out_dim) return;
    const int apart = kKeptWaves / slices;                 // row tiles of a workgroup side by side
    const int64_t first = (int64_t)(block / slice_groups) * apart + wave / slices, stride = (int64_t)(gridDim.x / slice_groups) * apart;

    // row r of fragment t: of 32 bits output 16 t + r; of 16 bits, so that two fragments make 16 neighbouring bytes of a lane, output
    // 32 (t / 2) + 8 (r / 4) + 4 (t % 2) + r % 4
    const auto output = [](int t, int r) { return WIDE ? 16 * t + r : 32 * (t >> 1) + 8 * (r >> 2) + 4 * (t & 1) + (r & 3); };
    rg_u32x4 wc[FRAGS][STEPS];
    uint32_t ws[FRAGS][(STEPS + 3) / 4];
#pragma unroll
    for (int t = 0; t < FRAGS; ++t) {
        const uint32_t* w = weight + (int64_t)min(h0 + output(t, c), out_dim - 1) * weight_stride;
#pragma unroll
        for (int k = 0; k < (STEPS + 3) / 4; ++k) ws[t][k] = 0;
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const int g = 4 * k + q;
            const bool live = g < groups;
            wc[t][k] = rg_u32x4{0u, 0u, 0u, 0u};
            if (live) wc[t][k] = *(const rg_u32x4*)(w + 4 * g);
            const uint32_t s = live ? (w[4 * groups + k] >> (8 * q)) & 255u : 127u;
            ws[t][k >> 2] |= s << (8 * (k & 3));
        }
    }

    struct Tile {
        rg_u32x4 code[STEPS];
        uint32_t scale[STEPS];
    };
    const auto load = [&](Tile& x, int64_t tile) {
        const uint32_t* row = rows + rg_least(16 * tile + c, n_act - 1) * rows_stride;
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            x.code[k] = *(const rg_u32x4*)(row + 4 * min(4 * k + q, groups - 1));   // (what is behind the last group meets zeros)
            x.scale[k] = row[4 * groups + min(k, (groups - 1) >> 2)];
        }
    };
    const int64_t tiles = (n_act + 15) >> 4;
    if (first >= tiles) return;
    // how this wavefront's part of a tile lies in LDS and is stored: `width` numbers of a row, in pieces of 16 bytes
    const int width = min(OUTS, out_dim - h0);
    const int pitch = run_on ? width * (int)sizeof(T) : PITCH, lanes = (width + E - 1) / E;
    char* const mine = (char*)stage[wave];
    Tile next;
    load(next, first);
    for (int64_t tile = first; tile < tiles; tile += stride) {
        const Tile x = next;
        load(next, rg_least(tile + stride, tiles - 1));
        v4f acc[FRAGS];
#pragma unroll
        for (int t = 0; t < FRAGS; ++t) acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
            const uint32_t s = 4 * k + q < groups ? x.scale[k] >> (8 * q) : 127u;
            const v8i b = v8i{(int)x.code[k][0], (int)x.code[k][1], (int)x.code[k][2], (int)x.code[k][3], 0, 0, 0, 0};
#pragma unroll
            for (int t = 0; t < FRAGS; ++t) {
                const v8i a = v8i{(int)wc[t][k][0], (int)wc[t][k][1], (int)wc[t][k][2], (int)wc[t][k][3], 0, 0, 0, 0};
                if ((k & 3) == 0) acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[t], 4, 4, 0, (int)ws[t][k >> 2], 0, (int)s);
                if ((k & 3) == 1) acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[t], 4, 4, 1, (int)ws[t][k >> 2], 0, (int)s);
                if ((k & 3) == 2) acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[t], 4, 4, 2, (int)ws[t][k >> 2], 0, (int)s);
                if ((k & 3) == 3) acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc[t], 4, 4, 3, (int)ws[t][k >> 2], 0, (int)s);
            }
        }
        T* const to = (T*)(mine + c * pitch);
        if (run_on) {                                      // number by number: rows start anywhere
#pragma unroll
            for (int t = 0; t < FRAGS; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int at = output(t, 4 * q) + r;
                    if (at < width) to[at] = (T)acc[t][r];
                }
        } else if constexpr (WIDE) {
#pragma unroll
            for (int t = 0; t < FRAGS; ++t) *(v4f*)(to + 16 * t + 4 * q) = acc[t];
        } else {
#pragma unroll
            for (int t = 0; t < FRAGS; t += 2) {
                typename RgPack<T, 8>::type v;
#pragma unroll
                for (int r = 0; r < 8; ++r) v[r] = (T)acc[t + (r >> 2)][r & 3];
                *(rg_u32x4a*)(to + 16 * t + 8 * q) = __builtin_bit_cast(rg_u32x4a, v);
            }
        }
        wave_exchange();
        const int live = (int)rg_least(16, n_act - 16 * tile);
        const int numbers = run_on ? live * width : width, pieces = run_on ? (numbers + E - 1) / E : live * lanes;
        T* const out = y + 16 * tile * y_stride + h0;
#pragma unroll
        for (int p0 = 0; p0 < 16 * OUTS / E; p0 += RG_WAVE) {
            const int p = p0 + lane;
            if (p >= pieces) continue;
            const int r = run_on ? 0 : width == OUTS ? p / (OUTS / E) : (int)rg_divide(p, inv_last);
            const int at = (p - r * lanes) * E, left = numbers - at;
            const rg_u32x4a v = *(const rg_u32x4a*)(mine + r * pitch + at * sizeof(T));
            T* const there = out + r * y_stride + at;
            typedef typename RgPack<T, E>::type Piece;
            if (ONCE) __builtin_nontemporal_store(__builtin_bit_cast(Piece, v), (Piece*)there);
            else if (left >= E) *(Piece*)there = __builtin_bit_cast(Piece, v);
            else {
                const auto e = __builtin_bit_cast(Piece, v);
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if (i < left) there[i] = e[i];
            }
        }
        wave_exchange();
    }
}

// ---------------------------------------------------------------- grad = dy^T . rows
// The contraction runs over the rows, so the matrix unit wants both operands column by column, eight rows of one column side by side.
// Threads turn them on their way into LDS: one loads four neighbouring columns of eight rows of dy, or one word of codes (eight
// columns) of eight rows, and puts pairs of rows together by byte permutations.  4-bit numbers times a scale of up to 2^125 (byte 252, the largest that
// quantisation makes) are bf16 numbers exactly; numbers of dy are cut into bf16 numbers that sum to them exactly (one for bf16, two for f16, three for f32,
// but for what f32 has below 2^-133, the smallest bf16 number; the matrix unit takes subnormal bf16 numbers as they are).

constexpr uint32_t kLowHalves = 0x05040100u, kHighHalves = 0x07060302u;   // of (later, earlier) as {earlier, later}

__device__ __forceinline__ uint32_t bits(v2bf v) { uint32_t u; __builtin_memcpy(&u, &v, 4); return u; }

union Frag {
    uint32_t w[4];
    v8bf v;
};

// Fragments 2 BYTE and 2 BYTE + 1 of eight rows' words of codes: fragment u holds number u of each word's eight.
template <int BYTE>
__device__ __forceinline__ void turn_byte(const uint32_t (&code)[8], const float (&scale)[8], Frag& even, Frag& odd) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        const uint32_t p0 = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[j], scale[j], BYTE));
        const uint32_t p1 = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[j + 1], scale[j + 1], BYTE));
        even.w[j / 2] = __builtin_amdgcn_perm(p1, p0, kLowHalves);
        odd.w[j / 2] = __builtin_amdgcn_perm(p1, p0, kHighHalves);
    }
}

// x less its leading bf16 part (cut off, not rounded): exact, but NaN for infinities.
__device__ __forceinline__ float bf16_rest(float x) { return x - __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }

template <typename T> struct Parts { static constexpr int count = sizeof(T) == 4 ? 3 : 2; };
template <> struct Parts<__bf16> { static constexpr int count = 1; };

// Eight numbers cut into their parts, each as a fragment, handed to put(part, fragment).
template <int P, typename F>
__device__ __forceinline__ void cut(float (&x)[8], F put) {
    float whole[8], most = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        whole[j] = x[j];
        most = fmaxf(most, fabsf(x[j]));
    }
    const bool endless = __any(__builtin_isinf(most));
#pragma unroll
    for (int p = 0; p < P; ++p) {
        Frag f;
#pragma unroll
        for (int j = 0; j < 8; j += 2) f.w[j / 2] = __builtin_amdgcn_perm(__float_as_uint(x[j + 1]), __float_as_uint(x[j]), kHighHalves);
        put(p, f);
        if (p + 1 == P) break;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = bf16_rest(x[j]);
        if (endless) {                                     // infinities have no rest (NaN has, and stays one)
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = __builtin_isinf(whole[j]) ? 0.0f : x[j];
        }
    }
}

// The number in the low or the high half of a word.
template <typename T>
__device__ __forceinline__ float half_number(uint32_t word, int high) {
    const uint16_t h = (uint16_t)(word >> (16 * high));
    T v;
    __builtin_memcpy(&v, &h, 2);
    return (float)v;
}

// Every wavefront's LDS accesses done, and everyone here.  (Loads from memory stay on their way.)
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

constexpr int kGradThreads = 512;

// A workgroup's tile of 64 TH outputs x 128 TF columns, ROWS rows at a time; its eight wavefronts are WH x WF x WK of them, each with
// 64 x 16 FRAGS of the tile and 32 of the rows.
template <typename T, int TF_> struct GradShape {
    static constexpr int TH = 2, TF = TF_, P = Parts<T>::count;
    static constexpr int FRAGS = 4 * TF;
    static constexpr int WH = TH, WF = 8 * TF / FRAGS, WK = 8 / (WH * WF), ROWS = 32 * WK, GROUPS = ROWS / 8;
    static constexpr int kDy = GROUPS * 128 * TF;          // pieces of 16 bytes (eight rows of a column): codes first, then the parts of dy
    static constexpr int kPieces = kDy + P * GROUPS * 64 * TH;
    static constexpr int kSums = 4 * 4 * FRAGS * 64;       // what four wavefronts hand to the others at the end
    static constexpr int kLds = 2 * kPieces > kSums ? 2 * kPieces : kSums;
    static_assert(GROUPS * 16 * TH <= 256 && GROUPS * 16 * TF <= 256, "a thread loads one item of a step");
    static_assert(kLds * 16 <= kLdsBytes, "a workgroup's LDS");
};

// Bound by everything at once.  One pass behind the other, with the join: 794 k rows, 256 x 256, bf16 133 to 137 us; on copies of an earlier form (137) without the
// loads 99, without the products 106, without the turning 120 (62 at the rate of a large library product, 84 for the bytes).  100 k rows, 256 x 602, f32
// (three parts of dy) 100 to 107 us; of 100, 69 without the products (which are 55 at that rate), 89 without the cutting and turning, 93 without the loads.  Smaller
// tiles of 128 x 128 took 165 and 114 us.  (Under a tracer, which runs them one by one: 122 to 125 us and 8.4 for the join, 105 and 6.7.)
// Rows counted on the device: ranges are cut from the room for them, so that workgroups whose range lies behind the count have nothing to do (794 k rows
// counted in room for 4.3 M: 512 us).
// Four wavefronts load dy, the others codes; all of them multiply.  While step s is multiplied from one half of LDS the other half
// is free for step s + 1, whose rows, and those of s + 2, are on their way: one barrier a step.  The WK sums of a piece of the tile are added up in LDS
// at the end, the ranges' of the rows by a second launch in their order.
// Workgroups of one range of rows follow each other on one XCD, whose L2 serves all but the first.
template <typename S, typename T>
__global__ void __launch_bounds__(kGradThreads, 2) k_mx4_grad(const T* __restrict__ dy, int64_t dy_stride, const uint32_t* __restrict__ rows,
                                                             int64_t rows_stride, int64_t n, const int32_t* __restrict__ n_dev, int out_dim,
                                                             int dim, int64_t rows_per_split, float* __restrict__ grad, int64_t grad_stride,
                                                             int64_t split_stride, int tiles_h, int tiles) {
    constexpr int P = S::P, W4 = sizeof(T), FRAGS = S::FRAGS;                    // W4: words of four numbers of dy
    __shared__ Frag lds[S::kLds];
    const int64_t n_act = rg_rows(n, n_dev);
    const int lane = rg_lane(), c = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);      // (the same in every lane, which the compiler may know)
    const int block = rg_xcd_block(blockIdx.x, gridDim.x);
    const int tile = block % tiles;
    const int64_t split = block / tiles;
    const int h0 = (tile % tiles_h) * (64 * S::TH), f0 = (tile / tiles_h) * (128 * S::TF);
    const int groups = (dim + kGroup - 1) / kGroup;
    const int64_t first = split * rows_per_split, last = rg_least(first + rows_per_split, n_act);
    const int64_t steps = last > first ? (last - first) / S::ROWS : 0;
    const int rest = last > first ? (int)((last - first) - steps * S::ROWS) : 0;

    // this wavefront's piece of the tile
    const int wf = wave % S::WF, wh = wave / S::WF % S::WH, wk = wave / (S::WF * S::WH);
    const Frag* from_x = lds + (4 * wk + q) * (128 * S::TF) + 16 * FRAGS * wf + c;
    const Frag* from_dy = lds + S::kDy + (4 * wk + q) * (64 * S::TH) + 64 * wh + c;
    v4f acc[4][FRAGS];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int u = 0; u < FRAGS; ++u) acc[t][u] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    // between(i): what is done behind the products of a fragment, in their shadow
    const auto multiply = [&](int half, auto between) {
        const auto dy_frag = [&](int i) { return from_dy[half * S::kPieces + (i >> 2) * S::GROUPS * 64 * S::TH + 16 * (i & 3)]; };
        Frag b[FRAGS], a[3];
        a[0] = dy_frag(0);
#pragma unroll
        for (int u = 0; u < FRAGS; ++u) b[u] = from_x[half * S::kPieces + 16 * u];
        a[1] = dy_frag(1);
#pragma unroll
        for (int i = 0; i < 4 * P; ++i) {                  // (the next two fragments are on their way from LDS during these products)
            if (i + 2 < 4 * P) a[(i + 2) % 3] = dy_frag(i + 2);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < FRAGS; ++u) acc[i & 3][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[i % 3].v, b[u].v, acc[i & 3][u], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            between(i);
        }
    };

    // ROLE: loads dy (its four columns k) or codes (its word w) of the eight rows of group g.
    const auto run = [&](auto role, int item) {
        constexpr bool DY = decltype(role)::value;
        constexpr int PER = DY ? 16 * S::TH : 16 * S::TF;
        const int g = item / PER, k = item % PER;
        const int h = h0 + 4 * k, h_at = min(h, out_dim - 4), over = h - h_at;
        const bool ragged = h0 + 64 * S::TH > out_dim;
        const int group = min((f0 >> 5) + (k >> 2), groups - 1);
        const T* pd = dy + (first + 8 * g) * dy_stride + h_at;
        const uint32_t* px = rows + (first + 8 * g) * rows_stride + min((f0 >> 3) + k, 4 * groups - 1);
        const uint8_t* ps = (const uint8_t*)(rows + (first + 8 * g) * rows_stride + 4 * groups) + group;
        struct Raw {
            uint32_t w[DY ? 8 * W4 : 16];
        };
        // row `at` (of those from the thread's first on) as the j-th of eight
        const auto load_row = [&](Raw& raw, int j, int64_t at) {
            if constexpr (!DY) {
                raw.w[j] = px[at * rows_stride];
                raw.w[8 + j] = ps[4 * at * rows_stride];
            } else {
                typedef uint32_t Words __attribute__((ext_vector_type(sizeof(T) == 4 ? 4 : 2), aligned(2)));
                const Words v = *(const Words*)(pd + at * dy_stride);
#pragma unroll
                for (int t = 0; t < W4; ++t) raw.w[j * W4 + t] = v[t];
            }
        };
        // step s (behind the last whole one: that one again, which nothing uses)
        const auto load = [&](Raw& raw, int64_t s) {
            if (s >= steps) {
                pd -= S::ROWS * dy_stride;
                px -= S::ROWS * rows_stride;
                ps -= 4 * S::ROWS * rows_stride;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) load_row(raw, j, j);
            pd += S::ROWS * dy_stride;
            px += S::ROWS * rows_stride;
            ps += 4 * S::ROWS * rows_stride;
        };
        // what was loaded as it goes into LDS: of the last, not whole step `live` rows, the others as zeros
        const auto settle = [&](Raw& raw, int live) {
            if constexpr (!DY) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    raw.w[j] = j < live ? raw.w[j] : 0u;
                    raw.w[8 + j] = j < live ? raw.w[8 + j] << 23 : 0u;
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int t = 0; t < W4; ++t) raw.w[j * W4 + t] = j < live ? raw.w[j * W4 + t] : 0u;
                if (ragged) {                              // columns that were loaded from further left
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if constexpr (W4 == 2) {
                            const uint64_t x = (((uint64_t)raw.w[2 * j + 1] << 32) | raw.w[2 * j]) >> ((16 * over) & 63);
                            raw.w[2 * j] = (uint32_t)x;
                            raw.w[2 * j + 1] = (uint32_t)(x >> 32);
                        } else {
                            const uint32_t x0 = raw.w[4 * j], x1 = raw.w[4 * j + 1], x2 = raw.w[4 * j + 2], x3 = raw.w[4 * j + 3];
                            raw.w[4 * j] = over == 0 ? x0 : over == 1 ? x1 : over == 2 ? x2 : x3;
                            raw.w[4 * j + 1] = over == 0 ? x1 : over == 1 ? x2 : x3;
                            raw.w[4 * j + 2] = over == 0 ? x2 : x3;
                        }
                    }
                }
            }
        };
        // a quarter of it (numbers 2 t and 2 t + 1 of the words of codes, column t of dy) into one half of LDS
        const auto turn = [&](const Raw& raw, int half, int t) {
            Frag* to = lds + half * S::kPieces;
            if constexpr (!DY) {
                uint32_t code[8];
                float scale[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    code[j] = raw.w[j];
                    scale[j] = __uint_as_float(raw.w[8 + j]);
                }
                Frag even, odd;
                if (t == 0) turn_byte<0>(code, scale, even, odd);
                else if (t == 1) turn_byte<1>(code, scale, even, odd);
                else if (t == 2) turn_byte<2>(code, scale, even, odd);
                else turn_byte<3>(code, scale, even, odd);
                to[g * (128 * S::TF) + 2 * t * PER + k] = even;
                to[g * (128 * S::TF) + (2 * t + 1) * PER + k] = odd;
            } else {
                Frag* column = to + S::kDy + g * (64 * S::TH) + t * PER + k;
                if constexpr (P == 1) {
                    Frag f;
#pragma unroll
                    for (int j = 0; j < 8; j += 2)
                        f.w[j / 2] = __builtin_amdgcn_perm(raw.w[(j + 1) * W4 + (t >> 1)], raw.w[j * W4 + (t >> 1)], t & 1 ? kHighHalves : kLowHalves);
                    *column = f;
                } else {
                    float x[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if constexpr (W4 == 4) x[j] = __uint_as_float(raw.w[4 * j + t]);
                        else x[j] = half_number<T>(raw.w[2 * j + (t >> 1)], t & 1);
                    }
                    cut<P>(x, [&](int p, const Frag& f) { column[p * S::GROUPS * 64 * S::TH] = f; });
                }
            }
        };
        const auto turn_all = [&](Raw& raw, int half, int live) {
            settle(raw, live);
#pragma unroll
            for (int t = 0; t < 4; ++t) turn(raw, half, t);
        };
        if (steps > 0) {
            if constexpr (P == 1) {
                // Two steps' rows are on their way; the next step's are turned in the shadow of this one's products.  (Turned before them by all
                // wavefronts: 794 k rows, 256 x 256 126 us instead of 122, 1.5 M rows, 256 x 100 166 and 152.)
                const auto step = [&](Raw& raw, int64_t s, int half) {
                    lds_barrier();
                    multiply(half, [&](int i) {
                        if (i == 0) settle(raw, 8);
                        turn(raw, half ^ 1, i);
                        __builtin_amdgcn_sched_barrier(0);
                        if (i == 3) load(raw, s + 3);
                        __builtin_amdgcn_sched_barrier(0);
                    });
                };
                Raw even, odd;
                load(even, 0);
                load(odd, 1);
                turn_all(even, 0, 8);
                load(even, 2);
                int64_t s = 0;
                for (; s + 2 <= steps; s += 2) {
                    step(odd, s, 0);
                    step(even, s + 1, 1);
                }
                if (s < steps) step(odd, s, 0);
            } else {
                // dy's parts take longer to make: of the two wavefronts of a SIMD one does it while the other one multiplies; registers for one step's
                // rows are left.  (In the shadow of the own products, on one set of rows: 300 k rows, 256 x 256 of f16 80 us instead of 77, 128 x 64 32 and 30, f32 the same.)
                Raw raw;
                load(raw, 0);
                turn_all(raw, 0, 8);
                load(raw, 1);
                for (int64_t s = 0; s < steps; ++s) {
                    lds_barrier();
                    if (!DY) multiply((int)(s & 1), [](int) {});
                    if (s + 1 < steps) turn_all(raw, (int)(s + 1) & 1, 8);
                    load(raw, s + 2);
                    __builtin_amdgcn_sched_barrier(0);
                    if (DY) multiply((int)(s & 1), [](int) {});
                }
            }
        }
        if (rest > 0) {
            Raw raw;
#pragma unroll
            for (int j = 0; j < 8; ++j) load_row(raw, j, min(j, rest - 1 - 8 * g));
            turn_all(raw, (int)(steps & 1), rest - 8 * g);
            lds_barrier();
            multiply((int)(steps & 1), [](int) {});
        }
    };
    if (wave < S::GROUPS * S::TH / 4) run(std::true_type(), threadIdx.x);
    else if (wave >= 4 && wave < 4 + S::GROUPS * S::TF / 4) run(std::false_type(), threadIdx.x - 256);
    else                                                   // (nothing left to load)
        for (int64_t s = 0; s < steps + (rest > 0); ++s) {
            lds_barrier();
            multiply((int)(s & 1), [](int) {});
        }

    // the sums over wk, half of the wavefronts giving theirs to the other half (wk is the slowest of a wavefront's coordinates)
    v4f* sums = (v4f*)lds;
    for (int half = 4; half >= S::WH * S::WF; half >>= 1) {
        __syncthreads();
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int u = 0; u < FRAGS; ++u) sums[((wave - half) * (4 * FRAGS) + t * FRAGS + u) * 64 + lane] = acc[t][u];
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int u = 0; u < FRAGS; ++u) acc[t][u] += sums[(wave * (4 * FRAGS) + t * FRAGS + u) * 64 + lane];
        }
    }
    if (wk != 0) return;
    // fragment i of the codes' 8 TF: number i / TF of words 16 (i % TF) + 0 .. 15; of dy's 4 TH: columns 4 (16 (i % TH) + 0 .. 15) + i / TH
    float* out = grad + split * split_stride;
    constexpr int RUN = FRAGS / S::TF;                     // neighbouring numbers of a word
#pragma unroll
    for (int word = 0; word < S::TF; ++word) {
        const int col = f0 + 8 * (16 * word + c) + RUN * wf;
        if (col >= dim) continue;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int piece = 4 * wh + t;
                const int row = h0 + 4 * (16 * (piece % S::TH) + 4 * q + r) + piece / S::TH;
                if (row >= out_dim) continue;
                float v[RUN];
#pragma unroll
                for (int u = 0; u < RUN; ++u) v[u] = acc[t][u * S::TF + word][r];
                rg_store_live<RUN>(out + row * grad_stride + col, dim - col, v);
            }
    }
}

// A wavefront makes a tile of 16 COLS outputs x 128 columns from rows of its own, the eight of a workgroup the same tile from
// neighbouring rows, and adds theirs up in LDS; so the parts that a second launch joins are few.  A row of the tile is 128 bytes of dy,
// 64 of codes and 4 of scales each: a wavefront loads them 16 bytes a lane and turns them round by way of LDS of its own (without a barrier), and
// the next 32 rows are on their way meanwhile.  Bound by the latency of these steps where rows are few, else by memory: 100 k rows, 41 x 602, f32:
// 33 us with the join; 1.5 M rows, 41 x 100, bf16: 59 to 61 us (3.7 TB/s).  (Loaded as the lanes need them, 24 accesses of 4 and 8 bytes to a step instead of 7, a step
// took a compute unit 400 to 540 cycles.)
// Workgroups of one range of rows follow each other on one XCD, whose L2 serves all but the first.
// NARROW: rows of dy are shorter than 16 bytes.
constexpr int kFewWaves = 8;

// (Four columns of three parts each would leave no registers for the rows on their way.)
template <typename T> struct FewTile {
    static constexpr int COLS = sizeof(T) == 4 ? 2 : 4;
    static constexpr int E = 16 / sizeof(T);               // numbers of dy in 16 bytes
    static constexpr int PIECES = COLS * sizeof(T);        // 16 bytes each, of a tile's row of dy
    static constexpr int LOADS = PIECES / 2;               // for 32 rows
};

template <typename T> struct FewLds {
    rg_u32x4 dy[32][FewTile<T>::PIECES];
    rg_u32x4 code[32][4];
    float scale[32][4];
};

template <typename T, bool NARROW>
__global__ void __launch_bounds__(64 * kFewWaves, 2) k_mx4_grad_few(const T* __restrict__ dy, int64_t dy_stride, const uint32_t* __restrict__ rows,
                                                              int64_t rows_stride, int64_t n, const int32_t* __restrict__ n_dev, int out_dim,
                                                              int dim, int64_t rows_per_wave, float* __restrict__ grad, int64_t grad_stride,
                                                              int64_t split_stride, int tiles_h, int tiles) {
    constexpr int COLS = FewTile<T>::COLS, E = FewTile<T>::E, P = Parts<T>::count;
    constexpr int PIECES = FewTile<T>::PIECES, LOADS = FewTile<T>::LOADS, BY = 32 / LOADS;
    __shared__ union {
        FewLds<T> rows[kFewWaves];
        v4f sums[kFewWaves / 2][COLS * 8][64];
    } lds;
    static_assert(sizeof(lds) <= kLdsBytes, "a workgroup's LDS");
    const int64_t n_act = rg_rows(n, n_dev);
    const int lane = rg_lane(), c = lane & 15, q = lane >> 4;
    const int wave = threadIdx.x >> 6;
    const int block = rg_xcd_block(blockIdx.x, gridDim.x);
    const int tile = block % tiles;
    const int64_t split = block / tiles;
    const int h0 = (tile % tiles_h) * (16 * COLS), f0 = (tile / tiles_h) * 128;
    const int groups = (dim + kGroup - 1) / kGroup;
    const int64_t first = (split * kFewWaves + wave) * rows_per_wave, last = rg_least(first + rows_per_wave, n_act);

    // what this lane loads: 16 bytes of dy of every BY-th row (from further left where the row ends before them, and moved behind the
    // load), a group's codes of rows lane / 4 + 0, 16, the scales of row lane % 32
    const int dy_row = lane / PIECES, dy_piece = lane % PIECES;
    const int piece = h0 + dy_piece * E, piece_at = NARROW ? piece : min(piece, out_dim - E), over = piece - piece_at;
    const bool ragged = h0 + 16 * COLS > out_dim;
    const T* pd = dy + (first + dy_row) * dy_stride + piece_at;
    const uint32_t* px = rows + (first + (lane >> 2)) * rows_stride + 4 * min((f0 >> 5) + (lane & 3), groups - 1);
    const uint32_t* ps = rows + (first + (lane & 31)) * rows_stride + 4 * groups + (f0 >> 7);
    FewLds<T>& mine = lds.rows[wave];

    struct Step {
        rg_u32x4 d[LOADS], code[2];
        uint32_t scale;
    };
    // the next 32 rows, of which `left` are there: those behind read the last one
    const auto load = [&](Step& s, int left) {
        const bool whole = left >= 32;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const T* p = pd + (whole ? BY * i : min(BY * i, left - 1 - dy_row)) * dy_stride;
            if constexpr (NARROW) {
                T v[E];
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = piece + e < out_dim ? p[e] : (T)0.0f;
                __builtin_memcpy(&s.d[i], v, 16);
            } else {
                typedef uint32_t Any __attribute__((ext_vector_type(4), aligned(2)));
                s.d[i] = *(const Any*)p;
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) s.code[i] = *(const rg_u32x4*)(px + (whole ? 16 * i : min(16 * i, left - 1 - (lane >> 2))) * rows_stride);
        s.scale = ps[(whole ? 0 : min(0, left - 1 - (lane & 31))) * rows_stride];
        pd += 32 * dy_stride;
        px += 32 * rows_stride;
        ps += 32 * rows_stride;
    };
    // them into LDS, those behind the last as zeros
    const auto place = [&](Step& s, int left) {
        if (left < 32) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i)
                if (BY * i + dy_row >= left) s.d[i] = rg_u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (16 * i + (lane >> 2) >= left) s.code[i] = rg_u32x4{0u, 0u, 0u, 0u};
            if ((lane & 31) >= left) s.scale = 0u;
        }
        if (!NARROW && ragged) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                uint32_t w0 = s.d[i][0], w1 = s.d[i][1], w2 = s.d[i][2], w3 = s.d[i][3];
                const int by = over * (int)sizeof(T);
                if (by & 8) { w0 = w2; w1 = w3; }
                if (by & 4) { w0 = w1; w1 = w2; w2 = w3; }
                if (sizeof(T) == 2 && (by & 2)) {
                    w0 = __builtin_amdgcn_alignbyte(w1, w0, 2);
                    w1 = __builtin_amdgcn_alignbyte(w2, w1, 2);
                    w2 = __builtin_amdgcn_alignbyte(w3, w2, 2);
                    w3 >>= 16;
                }
                s.d[i] = rg_u32x4{w0, w1, w2, w3};
            }
        }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) mine.dy[BY * i + dy_row][dy_piece] = s.d[i];
#pragma unroll
        for (int i = 0; i < 2; ++i) mine.code[16 * i + (lane >> 2)][lane & 3] = s.code[i];
        if (lane < 32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) mine.scale[lane][i] = scale_bits((s.scale >> (8 * i)) & 255u);
        }
    };

    v4f acc[COLS][8];
#pragma unroll
    for (int t = 0; t < COLS; ++t)
#pragma unroll
        for (int u = 0; u < 8; ++u) acc[t][u] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    // lane 16 q + c: rows 4 j + q, columns COLS c .. of dy, word c of the codes
    const auto multiply = [&] {
        wave_exchange();
        uint32_t code[8];
        float scale[8];
        struct alignas(COLS * sizeof(T)) Cols { uint32_t w[COLS * sizeof(T) / 4]; };
        Cols d[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            d[j] = ((const Cols*)mine.dy[4 * j + q])[c];
            code[j] = ((const uint32_t*)mine.code[4 * j + q])[c];
            scale[j] = mine.scale[4 * j + q][c >> 2];
        }
        wave_exchange();
        Frag a[P][COLS];
#pragma unroll
        for (int t = 0; t < COLS; ++t) {
            if constexpr (P == 1) {
#pragma unroll
                for (int j = 0; j < 8; j += 2)
                    a[0][t].w[j / 2] = __builtin_amdgcn_perm(d[j + 1].w[t >> 1], d[j].w[t >> 1], t & 1 ? kHighHalves : kLowHalves);
            } else {
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    if constexpr (sizeof(T) == 4) x[j] = __uint_as_float(d[j].w[t]);
                    else x[j] = half_number<T>(d[j].w[t >> 1], t & 1);
                }
                cut<P>(x, [&](int p, const Frag& f) { a[p][t] = f; });
            }
        }
#define RG_MULTIPLY_BYTE(B)                                                                                                              \
        {                                                                                                                                \
            Frag even, odd;                                                                                                              \
            turn_byte<B>(code, scale, even, odd);                                                                                       \
            _Pragma("unroll") for (int p = 0; p < P; ++p)                                                                                \
                _Pragma("unroll") for (int t = 0; t < COLS; ++t) {                                                                       \
                    acc[t][2 * B] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[p][t].v, even.v, acc[t][2 * B], 0, 0, 0);                  \
                    acc[t][2 * B + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[p][t].v, odd.v, acc[t][2 * B + 1], 0, 0, 0);           \
                }                                                                                                                        \
        }
        RG_MULTIPLY_BYTE(0) RG_MULTIPLY_BYTE(1) RG_MULTIPLY_BYTE(2) RG_MULTIPLY_BYTE(3)
#undef RG_MULTIPLY_BYTE
    };

    const int steps = last > first ? (int)((last - first) >> 5) : 0;
    const int rest = last > first ? (int)(last - first) & 31 : 0;
    Step s;
    if (steps > 0) {
        load(s, 32);
        for (int k = 0; k + 1 < steps; ++k) {
            place(s, 32);
            load(s, 32);
            __builtin_amdgcn_sched_barrier(0);
            multiply();
        }
        place(s, 32);
        multiply();
    }
    if (rest > 0) {
        load(s, rest);
        place(s, rest);
        multiply();
    }

    // half of the wavefronts hand their sums to the other half, until one is left
#pragma unroll
    for (int half = kFewWaves / 2; half > 0; half >>= 1) {
        __syncthreads();
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int t = 0; t < COLS; ++t)
#pragma unroll
                for (int u = 0; u < 8; ++u) lds.sums[wave - half][t * 8 + u][lane] = acc[t][u];
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int t = 0; t < COLS; ++t)
#pragma unroll
                for (int u = 0; u < 8; ++u) acc[t][u] += lds.sums[wave][t * 8 + u][lane];
        }
    }
    const int col = f0 + 8 * c;
    if (wave != 0 || col >= dim) return;
    float* out = grad + split * split_stride;
#pragma unroll
    for (int t = 0; t < COLS; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = h0 + COLS * (4 * q + r) + t;
            if (row >= out_dim) continue;
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = acc[t][u][r];
            rg_store_live<8>(out + row * grad_stride + col, dim - col, v);
        }
}

// grad = the sum of the splits' parts, which it has to read: 128 of 256 x 256 floats 8.4 us (4 TB/s).  A workgroup takes 64 chunks of 4
// numbers, 16 runs of the parts side by side, and adds up in one order.
__global__ void __launch_bounds__(1024) k_mx4_grad_join(const float* __restrict__ parts, int splits, int64_t split_stride, int out_dim, int dim,
                                                        float* __restrict__ grad, int64_t grad_stride) {
    __shared__ float runs[16][256];
    const int lane = rg_lane(), run = threadIdx.x >> 6;
    const int64_t total = (int64_t)out_dim * dim, at = ((int64_t)blockIdx.x * 64 + lane) * 4;
    const int per_run = (splits + 15) >> 4, first = run * per_run, last = min(first + per_run, splits);
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (at < total) {
#pragma unroll 8
        for (int s = first; s < last; ++s) {
            float v[4];
            rg_load_head<4>(parts + s * split_stride + at, (int)rg_least(4, total - at), v);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] += v[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) runs[run][i * 64 + lane] = sum[i];
    __syncthreads();
    if (threadIdx.x >= 256) return;
    const int64_t to = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (to >= total) return;
    float all = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) all += runs[r][(threadIdx.x & 3) * 64 + (threadIdx.x >> 2)];
    grad[to / dim * grad_stride + to % dim] = all;
}

bool aligned(const void* p, int bytes) { return (uintptr_t)p % (uintptr_t)bytes == 0; }

}  // namespace

extern "C" {

int64_t rg_mx4_row_words(int32_t dim) {
    if (dim < 1 || dim > RG_MX4_MAX_DIM) return 0;
    const int64_t groups = rg_div_up(dim, kGroup);
    return 4 * groups + rg_div_up(groups, 4);
}

rg_status rg_mx4_quantize(rg_ctx* ctx, const void* x, rg_dtype x_type, int64_t x_stride, int64_t n, const int32_t* n_dev, int32_t dim,
                          void* packed, int64_t packed_stride, void* stream) {
    if (!ctx) return RG_ERR_INVALID_ARG;
    RG_REQUIRE(ctx, n >= 0 && n <= (1ll << 31) - 1, "rg_mx4_quantize: n = %lld out of range", (long long)n);
    RG_REQUIRE(ctx, dim >= 1 && dim <= RG_MX4_MAX_DIM, "rg_mx4_quantize: dim = %d not in [1,%d]", dim, RG_MX4_MAX_DIM);
    RG_REQUIRE(ctx, rg_type_known(x_type), "rg_mx4_quantize: unknown type %d", (int)x_type);
    RG_REQUIRE(ctx, x_stride >= dim && packed_stride >= rg_mx4_row_words(dim), "rg_mx4_quantize: bad stride");
    if (n == 0) return RG_OK;
    RG_REQUIRE(ctx, x && packed, "rg_mx4_quantize: null pointer");
    RG_REQUIRE(ctx, aligned(x, rg_type_bytes(x_type)) && aligned(packed, 4), "rg_mx4_quantize: pointer not aligned to its numbers");
    RG_HIP(ctx, hipSetDevice(ctx->device));
    hipStream_t s = (hipStream_t)stream;
    const int pieces = (int)rg_div_up(dim, kGroup) * (kGroup * rg_type_bytes(x_type) / 16);
    const int rows = rows_per_group(ctx, n, pieces);
    RG_FOR_TYPE(x_type, k_mx4_quantize<T><<<row_groups(n, rows), 256, 0, s>>>((const T*)x, x_stride, n, n_dev, dim, (uint32_t*)packed,
                                                                                  packed_stride, pieces, rg_inverse(pieces), rows));
    RG_LAUNCH_CHECK(ctx, "k_mx4_quantize");
    return RG_OK;
}

rg_status rg_mx4_dequantize(rg_ctx* ctx, const void* packed, int64_t packed_stride, int64_t n, const int32_t* n_dev, int32_t dim, void* x,
                            rg_dtype x_type, int64_t x_stride, void* stream) {
    if (!ctx) return RG_ERR_INVALID_ARG;
    RG_REQUIRE(ctx, n >= 0 && n <= (1ll << 31) - 1, "rg_mx4_dequantize: n = %lld out of range", (long long)n);
    RG_REQUIRE(ctx, dim >= 1 && dim <= RG_MX4_MAX_DIM, "rg_mx4_dequantize: dim = %d not in [1,%d]", dim, RG_MX4_MAX_DIM);
    RG_REQUIRE(ctx, rg_type_known(x_type), "rg_mx4_dequantize: unknown type %d", (int)x_type);
    RG_REQUIRE(ctx, x_stride >= dim && packed_stride >= rg_mx4_row_words(dim), "rg_mx4_dequantize: bad stride");
    if (n == 0) return RG_OK;
    RG_REQUIRE(ctx, x && packed, "rg_mx4_dequantize: null pointer");
    RG_REQUIRE(ctx, aligned(x, rg_type_bytes(x_type)) && aligned(packed, 4), "rg_mx4_dequantize: pointer not aligned to its numbers");
    RG_HIP(ctx, hipSetDevice(ctx->device));
    hipStream_t s = (hipStream_t)stream;
    const int pieces = (int)rg_div_up((int64_t)dim * rg_type_bytes(x_type), 16);
    const int rows = rows_per_group(ctx, n, pieces);
    RG_FOR_TYPE(x_type, {
        const auto kernel = rg_store_once(x, dim * sizeof(T), x_stride * sizeof(T), n) ? k_mx4_dequantize<T, true> : k_mx4_dequantize<T, false>;
        kernel<<<row_groups(n, rows), 256, 0, s>>>((const uint32_t*)packed, packed_stride, n, n_dev, dim, (T*)x, x_stride, pieces,
                                                           rg_inverse(pieces), rows);
    });
    RG_LAUNCH_CHECK(ctx, "k_mx4_dequantize");
    return RG_OK;
}

rg_status rg_mx4_matmul(rg_ctx* ctx, const void* rows, int64_t rows_stride, int64_t n, const int32_t* n_dev, const void* weight,
                        int64_t weight_stride, int32_t out_dim, int32_t dim, void* y, rg_dtype y_type, int64_t y_stride, void* stream) {
    if (!ctx) return RG_ERR_INVALID_ARG;
    RG_REQUIRE(ctx, n >= 0 && n <= (1ll << 31) - 1, "rg_mx4_matmul: n = %lld out of range", (long long)n);
    RG_REQUIRE(ctx, dim >= 1 && dim <= RG_MX4_MAX_DIM && out_dim >= 1 && out_dim <= RG_MX4_MAX_DIM,
               "rg_mx4_matmul: dim = %d or out_dim = %d not in [1,%d]", dim, out_dim, RG_MX4_MAX_DIM);
    RG_REQUIRE(ctx, rg_type_known(y_type), "rg_mx4_matmul: unknown type %d", (int)y_type);
    const int64_t words = rg_mx4_row_words(dim);
    RG_REQUIRE(ctx, rows_stride >= words && weight_stride >= words && y_stride >= out_dim, "rg_mx4_matmul: bad stride");
    if (n == 0) return RG_OK;
    RG_REQUIRE(ctx, rows && weight && y, "rg_mx4_matmul: null pointer");
    RG_REQUIRE(ctx, aligned(rows, 4) && aligned(weight, 4) && aligned(y, rg_type_bytes(y_type)), "rg_mx4_matmul: pointer not aligned to its numbers");
    RG_HIP(ctx, hipSetDevice(ctx->device));
    hipStream_t s = (hipStream_t)stream;
    const int groups = (dim + kGroup - 1) / kGroup;
    const int steps = (groups + 3) / 4;
    const int64_t tiles = rg_div_up(n, 16) * rg_div_up(out_dim, 16);
    RG_FOR_TYPE(y_type, {
        // Up to 32 matrix products to a compute unit each tile has a wavefront of its own: keeping the weight only pays where it is used often (1 row of
        // 602 numbers times 41 outputs 3.1 us with the weight read by tiles, 4.7 kept; 1024 rows of 256 times 256 3.4 and 6.2; 4096 rows 5.0 and 6.1, 8192
        // rows 7.2 and 6.7; 8192 rows of 602 times 41 5.0 and 6.6, 16384 rows 6.6 and 6.7, 32768 rows 11.0 and 9.1).
        if (tiles * steps <= 32 * (int64_t)ctx->num_cus) {
            const dim3 grid((unsigned)rg_div_up(n, 64), (unsigned)rg_div_up(out_dim, 16));
            k_mx4_matmul<T, 1, 1><<<grid, 256, 0, s>>>((const uint32_t*)rows, rows_stride, n, n_dev, (const uint32_t*)weight, weight_stride, out_dim,
                                                       groups, (T*)y, y_stride);
        } else if (steps <= 8) {
            // Registers hold 128 outputs of up to 256 numbers (794 k rows of 256 times 256 outputs of bf16: 99 us, 155 with 64 to a wavefront), else 64.
            const bool many = steps <= 2 && out_dim > 64;
            const int outs = many ? 128 : 64;
            const int slices = out_dim > 2 * outs ? 4 : out_dim > outs ? 2 : 1;
            const int slice_groups = (int)rg_div_up(out_dim, outs * slices);
            // Two workgroups to a compute unit, four where registers hold up to 64 outputs of up to 384 numbers (1.5 M rows of 100 numbers times 47
            // outputs of f16: 58 / 50 / 59 us with 2 / 4 / 8; 794 k of 256 times 256 of bf16: 102 / 115 / 141), and as many whole turns of
            // the compute units as leave three tiles to a wavefront that has fetched the weight (100 k of 602 times 41: 15 us, 20 with one more).
            const int64_t deep = rg_div_up(rg_div_up(n, 16), kKeptWaves / slices);
            const int64_t turns = rg_min64(out_dim <= 64 && steps <= 3 ? 4 : 2, rg_max64(1, deep / (3 * ctx->num_cus)));
            const unsigned grid = (unsigned)(rg_min64(deep, rg_max64(1, turns * ctx->num_cus / slice_groups)) * slice_groups);
            const int last = out_dim % outs, last_bytes = last * (int)sizeof(T);
            const int run_on = out_dim <= outs && y_stride == out_dim && last_bytes % 16 != 0;
            const auto pick = [&](auto once) {             // (ONCE: rows of whole 16 bytes)
                constexpr bool ONCE = decltype(once)::value;
                if (many) return steps == 1 ? k_mx4_matmul_kept<T, 1, 8, ONCE> : k_mx4_matmul_kept<T, 2, 8, ONCE>;
                return steps == 1   ? k_mx4_matmul_kept<T, 1, 4, ONCE>
                       : steps == 2 ? k_mx4_matmul_kept<T, 2, 4, ONCE>
                       : steps == 3 ? k_mx4_matmul_kept<T, 3, 4, ONCE>
                       : steps == 4 ? k_mx4_matmul_kept<T, 4, 4, ONCE>
                       : steps == 5 ? k_mx4_matmul_kept<T, 5, 4, ONCE>
                                    : k_mx4_matmul_kept<T, 8, 4, ONCE>;
            };
            const bool once = rg_store_once(y, out_dim * sizeof(T), y_stride * sizeof(T), n);
            const auto kernel = once ? pick(std::true_type()) : pick(std::false_type());
            kernel<<<grid, kKeptThreads, 0, s>>>((const uint32_t*)rows, rows_stride, n, n_dev, (const uint32_t*)weight, weight_stride, out_dim, groups,
                                                 (T*)y, y_stride, slices, slice_groups, run_on, rg_inverse((uint32_t)rg_div_up(last_bytes, 16)));
        } else {
            // Longer rows, whose weight registers do not hold: read again (from L2) for every 32 rows.  (100 k rows of 1024 numbers times 256 outputs of bf16
            // this way 131 us, kept 45; of 2048 numbers 280.)  Few rows: workgroups side by side on their outputs (2000 rows of 2048 times 256: 20 us).
            const int64_t across = rg_min64(rg_div_up(n, 128), 1 << 20);
            const dim3 grid((unsigned)across, (unsigned)rg_min64(rg_div_up(out_dim, 64), rg_div_up((int64_t)ctx->num_cus * 4, across)));
            k_mx4_matmul<T, 2, 4><<<grid, 256, 0, s>>>((const uint32_t*)rows, rows_stride, n, n_dev, (const uint32_t*)weight, weight_stride, out_dim,
                                                       groups, (T*)y, y_stride);
        }
    });
    RG_LAUNCH_CHECK(ctx, "k_mx4_matmul");
    return RG_OK;
}

rg_status rg_mx4_matmul_grad(rg_ctx* ctx, const void* dy, rg_dtype dy_type, int64_t dy_stride, const void* rows, int64_t rows_stride, int64_t n,
                             const int32_t* n_dev, int32_t out_dim, int32_t dim, float* grad, int64_t grad_stride, void* stream) {
    if (!ctx) return RG_ERR_INVALID_ARG;
    RG_REQUIRE(ctx, n >= 0 && n <= (1ll << 31) - 1, "rg_mx4_matmul_grad: n = %lld out of range", (long long)n);
    RG_REQUIRE(ctx, dim >= 1 && dim <= RG_MX4_MAX_DIM && out_dim >= 1 && out_dim <= RG_MX4_MAX_DIM,
               "rg_mx4_matmul_grad: dim = %d or out_dim = %d not in [1,%d]", dim, out_dim, RG_MX4_MAX_DIM);
    RG_REQUIRE(ctx, rg_type_known(dy_type), "rg_mx4_matmul_grad: unknown type %d", (int)dy_type);
    RG_REQUIRE(ctx, rows_stride >= rg_mx4_row_words(dim) && dy_stride >= out_dim && grad_stride >= dim, "rg_mx4_matmul_grad: bad stride");
    RG_REQUIRE(ctx, grad && (n == 0 || (dy && rows)), "rg_mx4_matmul_grad: null pointer");
    RG_REQUIRE(ctx, aligned(rows, 4) && aligned(dy, rg_type_bytes(dy_type)) && aligned(grad, 4), "rg_mx4_matmul_grad: pointer not aligned to its numbers");
    RG_HIP(ctx, hipSetDevice(ctx->device));
    hipStream_t s = (hipStream_t)stream;
    // Few outputs: tiles of 64 (32) outputs, which read each row of dy once and need no turning by the whole workgroup.  (With the join, 100 k rows, 41 x 602,
    // f32 33 us, 57 by tiles of 128; 1.5 M rows, 41 x 100, bf16 61 and 92, 64 x 100 67 and 78, 128 x 100 98 and 95; 300 k rows, 128 x 64, f16 33 and 34.)
    // Columns of codes: 256 to a tile, so that dy is turned less often, but 128 where there are no more (1.5 M rows of bf16, 256 x 100 163 us, 213 by 256;
    // 128 x 100 96 and 113; 300 k of f16, 128 x 64 34 and 42).
    const bool few = out_dim <= 64;
    const int tile_h = few ? (dy_type == RG_F32 ? 32 : 64) : 128, tile_f = few || dim <= 128 ? 128 : 256;
    const int waves = few ? kFewWaves : 1, step = few ? 32 : 64;                  // ranges of rows to a workgroup, rows of a step
    const int tiles_h = (int)rg_div_up(out_dim, tile_h);
    const int64_t tiles = (int64_t)tiles_h * rg_div_up(dim, tile_f);
    const int64_t most = rg_max64(1, ctx->num_cus / tiles);
    const int64_t per_range = rg_max64(1, rg_div_up(rg_div_up(n, most * waves), step)) * step;
    const int64_t splits = rg_max64(1, rg_div_up(n, per_range * waves));
    float* parts = grad;
    int64_t parts_stride = grad_stride, split_stride = 0;
    if (splits > 1) {
        parts_stride = dim;
        split_stride = (int64_t)out_dim * dim;
        const rg_status st = rg_scratch(ctx, ctx->mx4_parts, (size_t)(splits * split_stride) * 4, s, "rg_mx4_matmul_grad");
        if (st != RG_OK) return st;
        parts = (float*)ctx->mx4_parts.p;
    }
    const unsigned grid = (unsigned)(tiles * splits);
    RG_FOR_TYPE(dy_type, {
        const auto kernel = !few ? (dim > 128 ? k_mx4_grad<GradShape<T, 2>, T> : k_mx4_grad<GradShape<T, 1>, T>)
                                 : out_dim < FewTile<T>::E ? k_mx4_grad_few<T, true> : k_mx4_grad_few<T, false>;
        kernel<<<grid, 512, 0, s>>>((const T*)dy, dy_stride, (const uint32_t*)rows, rows_stride, n, n_dev, out_dim, dim, per_range, parts, parts_stride,
                                    split_stride, tiles_h, (int)tiles);
    });
    RG_LAUNCH_CHECK(ctx, "k_mx4_grad");
    if (splits > 1) {
        k_mx4_grad_join<<<(unsigned)rg_div_up(split_stride, 256), 1024, 0, s>>>(parts, (int)splits, split_stride, out_dim, dim, grad, grad_stride);
        RG_LAUNCH_CHECK(ctx, "k_mx4_grad_join");
    }
    return RG_OK;
}

}  // extern "C"
