// Packed rows of 4-bit numbers with a scale per group of 32 (the layout is the header's): to and from numbers, their product with a
// packed weight, and the gradient of that product to its weight.
#include "rg_elements.h"

#include <algorithm>

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

constexpr int kGroup = 32;
constexpr uint32_t kScaleNan = 255;

// The scale byte as the float with this exponent: what the conversion instructions read the exponent of (0 stands for 2^-127 and
// 255 for "not a number" to them, as in the format).
__device__ __forceinline__ float scale_bits(uint32_t s) { return __uint_as_float(s << 23); }

// ---------------------------------------------------------------- numbers to packed rows
// 16 lanes take 128 numbers of a row (four groups), 8 each: the largest magnitude of a group, as an integer (so that NaN and
// infinities are the largest of all), goes round its four lanes; the numbers times 2^(127 - s), which is exact or far below the
// smallest magnitude, are rounded by the conversion instruction.
template <typename T>
__global__ void __launch_bounds__(256) k_mx4_quantize(const T* __restrict__ x, int64_t x_stride, int64_t n, const int32_t* __restrict__ n_dev,
                                                      int dim, uint32_t* __restrict__ packed, int64_t packed_stride, int quads, uint32_t inv_quads,
                                                      int rows_per_block) {
    const int64_t n_act = rg_rows(n, n_dev);
    const int64_t row0 = (int64_t)blockIdx.x * rows_per_block;
    if (row0 >= n_act) return;
    const int items = (int)rg_least(rows_per_block, n_act - row0) * quads;
    const int groups = (dim + kGroup - 1) / kGroup;
    const int sub = threadIdx.x & 15;
    for (int it = threadIdx.x >> 4; it < items; it += 16) {
        const int r = (int)rg_divide((uint32_t)it, inv_quads);
        const int quad = it - r * quads;
        const int col = quad * 128 + sub * 8;
        float v[8];
        rg_load_head<8>(x + (row0 + r) * x_stride + col, dim - col, v);
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
        top = max(top, (uint32_t)__shfl_xor((int)top, 1, RG_WAVE));
        top = max(top, (uint32_t)__shfl_xor((int)top, 2, RG_WAVE));
        const uint32_t e = top >> 23;
        const bool good = e < 255;
        const uint32_t s = good ? (e > 2 ? e - 2 : 0) : kScaleNan;
        const float f = __uint_as_float((254u - s) << 23);
        uint32_t word = 0;
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[0] * f, v[1] * f, 1.0f, 0);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[2] * f, v[3] * f, 1.0f, 1);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[4] * f, v[5] * f, 1.0f, 2);
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(word, v[6] * f, v[7] * f, 1.0f, 3);
        if (!good) word = 0;
        uint32_t* row = packed + (row0 + r) * packed_stride;
        const int group = quad * 4 + (sub >> 2);
        if (group < groups) row[quad * 16 + sub] = word;
        if ((sub & 3) == 0) ((uint8_t*)(row + 4 * groups))[group] = group < groups ? (uint8_t)s : 0;
    }
}

// ---------------------------------------------------------------- packed rows to numbers
// A lane takes one word of codes, 8 numbers of one group.
template <typename T>
__global__ void __launch_bounds__(256) k_mx4_dequantize(const uint32_t* __restrict__ packed, int64_t packed_stride, int64_t n,
                                                        const int32_t* __restrict__ n_dev, int dim, T* __restrict__ x, int64_t x_stride, int words,
                                                        uint32_t inv_words, int rows_per_block) {
    const int64_t n_act = rg_rows(n, n_dev);
    const int64_t row0 = (int64_t)blockIdx.x * rows_per_block;
    if (row0 >= n_act) return;
    const int items = (int)rg_least(rows_per_block, n_act - row0) * words;
    const int groups = (dim + kGroup - 1) / kGroup;
    for (int it = threadIdx.x; it < items; it += 256) {
        const int r = (int)rg_divide((uint32_t)it, inv_words);
        const int w = it - r * words;
        const uint32_t* row = packed + (row0 + r) * packed_stride;
        const uint32_t code = row[w];
        const float scale = scale_bits(((const uint8_t*)(row + 4 * groups))[w >> 2]);
        float v[8];
        typedef float v2f __attribute__((ext_vector_type(2)));
        const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 1);
        const v2f c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, scale, 3);
        v[0] = a.x; v[1] = a.y; v[2] = b.x; v[3] = b.y; v[4] = c.x; v[5] = c.y; v[6] = d.x; v[7] = d.y;
        rg_store_live<8>(x + (row0 + r) * x_stride + w * 8, dim - w * 8, v);
    }
}

// Rows that a workgroup takes when each is `per_row` units of work and it does `per_step` units at a time: several steps where
// there are rows enough for all compute units.
int rows_per_group(const rg_ctx* ctx, int64_t n, int per_row, int per_step, int steps) {
    const int64_t total = n * per_row;
    int64_t units = total >= (int64_t)ctx->num_cus * 8 * per_step * steps ? (int64_t)per_step * steps : per_step;
    units = rg_max64(units, total >> 22);                  // (a launch has less than 2^32 threads)
    return (int)rg_max64(1, units / per_row);
}

// ---------------------------------------------------------------- y = rows . weight^T
// A wavefront makes a tile of 16 R rows by 16 C outputs with the scaled 16 x 16 x 128 matrix instruction: lane 16 q + c holds group
// 4 k + q of row c in step k, 16 bytes of codes and their scale byte, as they lie in the packed row.  The weight is the first operand,
// so that a lane ends up with four neighbouring outputs of one row.  Groups behind the row's last are zeros; rows and outputs beyond
// the last read the last one's and are not stored.
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

// ---------------------------------------------------------------- grad = dy^T . rows
// The contraction runs over the rows, so both operands are needed column by column.  They are turned in registers: a lane loads four
// neighbouring columns of eight rows of dy and eight neighbouring columns (one word of codes) of the same rows, and the pairs of rows that
// the 16 x 16 x 32 bf16 matrix instruction wants side by side are put together by byte permutations; which column a lane's row of
// the tile stands for is free.  4-bit numbers times their scale are bf16 numbers exactly.  Numbers of dy are cut into PARTS bf16 numbers
// that sum to them exactly (1 for bf16, 2 for f16, 3 for f32).

constexpr uint32_t kLowHalves = 0x05040100u, kHighHalves = 0x07060302u;   // of (later, earlier) as {earlier, later}

__device__ __forceinline__ uint32_t bits(v2bf v) { uint32_t u; __builtin_memcpy(&u, &v, 4); return u; }

union Frag {
    uint32_t w[4];
    v8bf v;
};

// Fragments u = 0 .. 7 of eight rows' words of codes: fragment u holds number u of each word's eight.
__device__ __forceinline__ void turn_codes(const uint32_t (&code)[8], const uint32_t (&scale)[8], Frag (&f)[8]) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        const float s0 = scale_bits(scale[j]), s1 = scale_bits(scale[j + 1]);
#define RG_TURN_BYTE(B)                                                                                                              \
        {                                                                                                                            \
            const uint32_t p0 = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[j], s0, B));                                     \
            const uint32_t p1 = bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code[j + 1], s1, B));                                 \
            f[2 * B].w[j / 2] = __builtin_amdgcn_perm(p1, p0, kLowHalves);                                                           \
            f[2 * B + 1].w[j / 2] = __builtin_amdgcn_perm(p1, p0, kHighHalves);                                                      \
        }
        RG_TURN_BYTE(0) RG_TURN_BYTE(1) RG_TURN_BYTE(2) RG_TURN_BYTE(3)
#undef RG_TURN_BYTE
    }
}

// x less its leading bf16 part (cut off, not rounded): exact.  Infinities have no rest.
__device__ __forceinline__ float bf16_rest(float x) {
    const float head = __uint_as_float(__float_as_uint(x) & 0xFFFF0000u);
    return x == head ? 0.0f : x - head;
}

template <typename T> struct Parts { static constexpr int count = sizeof(T) == 4 ? 3 : 2; };
template <> struct Parts<__bf16> { static constexpr int count = 1; };

// What a lane holds of 32 rows: COLS neighbouring numbers of dy, the word of codes and the word of scales of its 8 rows.
template <typename T, int COLS> struct GradStep {
    typedef T Vec __attribute__((ext_vector_type(COLS)));
    Vec d[8];
    uint32_t code[8], scale[8];
};

template <typename T, int COLS>
__device__ __forceinline__ typename GradStep<T, COLS>::Vec load_columns(const T* p) {
    typename GradStep<T, COLS>::Vec v;
    if constexpr (COLS == 1) v[0] = *p;
    else {
        const typename RgPack<T, COLS>::type a = *(const typename RgPack<T, COLS>::type*)p;
#pragma unroll
        for (int i = 0; i < COLS; ++i) v[i] = a[i];
    }
    return v;
}

// The columns of a lane that reaches over the end of a row, which were loaded `over` columns further left (0: as they are; what
// comes in from the right is not used).
template <typename T, int COLS>
__device__ __forceinline__ typename GradStep<T, COLS>::Vec move_columns(typename GradStep<T, COLS>::Vec v, int over) {
    if constexpr (COLS == 1) return v;
    else if constexpr (COLS * sizeof(T) == 8 && COLS == 4) {
        uint64_t w;
        __builtin_memcpy(&w, &v, 8);
        w >>= (16 * over) & 63;
        __builtin_memcpy(&v, &w, 8);
        return v;
    } else {
        static_assert(COLS == 2, "two columns, or four of 16 bits");
        v[0] = over ? v[1] : v[0];
        return v;
    }
}

// Part p of one column of eight rows' numbers, as a fragment; the numbers lose that part.
__device__ __forceinline__ void turn_column(float (&x)[8], Frag& f, bool last) {
#pragma unroll
    for (int j = 0; j < 8; j += 2) f.w[j / 2] = __builtin_amdgcn_perm(__float_as_uint(x[j + 1]), __float_as_uint(x[j]), kHighHalves);
    if (!last) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = bf16_rest(x[j]);
    }
}

// A wavefront makes a tile of 16 COLS outputs x 128 columns from rows of its own, WAVES of them (a workgroup) the same tile from
// neighbouring rows, and adds theirs up in LDS; so the parts that a second launch joins are few.  The next 32 rows are on their
// way while the matrix unit works on these.  out_dim >= COLS.  Workgroups of one range of rows follow each other on one XCD: they read the same rows.
constexpr int kGradWaves = 8;

template <typename T, int COLS>
__global__ void __launch_bounds__(64 * kGradWaves, 2) k_mx4_grad(const T* __restrict__ dy, int64_t dy_stride, const uint32_t* __restrict__ rows,
                                                              int64_t rows_stride, int64_t n, const int32_t* __restrict__ n_dev, int out_dim,
                                                              int dim, int64_t rows_per_wave, float* __restrict__ grad, int64_t grad_stride,
                                                              int64_t split_stride, int tiles_h, int tiles) {
    __shared__ v4f sums[kGradWaves / 2][COLS * 8][64];
    const int64_t n_act = rg_rows(n, n_dev);
    const int lane = rg_lane(), c = lane & 15, q = lane >> 4;
    const int wave = threadIdx.x >> 6;
    const int block = rg_xcd_block(blockIdx.x, gridDim.x);
    const int tile = block % tiles;
    const int64_t split = block / tiles;
    const int h0 = (tile % tiles_h) * (16 * COLS), f0 = (tile / tiles_h) * 128;
    const int groups = (dim + kGroup - 1) / kGroup;
    const int h = h0 + COLS * c, col = f0 + 8 * c;
    const int h_at = min(h, out_dim - COLS), over = h - h_at;
    const int shift = 8 * (c >> 2);
    v4f acc[COLS][8];
#pragma unroll
    for (int t = 0; t < COLS; ++t)
#pragma unroll
        for (int u = 0; u < 8; ++u) acc[t][u] = v4f{0.0f, 0.0f, 0.0f, 0.0f};

    const int64_t first = (split * kGradWaves + wave) * rows_per_wave, last = rg_least(first + rows_per_wave, n_act);
    const T* pd = dy + (first + 8 * q) * dy_stride + h_at;
    const uint32_t* px = rows + (first + 8 * q) * rows_stride + min(col >> 3, 4 * groups - 1);
    const uint32_t* ps = rows + (first + 8 * q) * rows_stride + 4 * groups + (f0 >> 7);

    const auto load = [&](GradStep<T, COLS>& s) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            s.d[j] = load_columns<T, COLS>(pd + j * dy_stride);
            s.code[j] = px[j * rows_stride];
            s.scale[j] = ps[j * rows_stride];
        }
        pd += 32 * dy_stride;
        px += 32 * rows_stride;
        ps += 32 * rows_stride;
    };
    const auto multiply = [&](const GradStep<T, COLS>& s) {
        uint32_t scale[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) scale[j] = (s.scale[j] >> shift) & 255u;
        Frag b[8];
        turn_codes(s.code, scale, b);
        typename GradStep<T, COLS>::Vec d[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) d[j] = move_columns<T, COLS>(s.d[j], over);
#pragma unroll
        for (int t = 0; t < COLS; ++t) {
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = (float)d[j][t];
#pragma unroll
            for (int p = 0; p < Parts<T>::count; ++p) {
                Frag a;
                turn_column(x, a, p + 1 == Parts<T>::count);
#pragma unroll
                for (int u = 0; u < 8; ++u) acc[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b[u].v, acc[t][u], 0, 0, 0);
            }
        }
    };

    const int steps = last > first ? (int)((last - first) >> 5) : 0;
    if (steps > 0) {
        GradStep<T, COLS> even, odd;
        load(even);
        for (int k = 0; k + 2 <= steps; k += 2) {
            load(odd);
            __builtin_amdgcn_sched_barrier(0);
            multiply(even);
            // (behind the last whole step the same rows once more, which nothing uses)
            const int64_t back = k + 2 < steps ? 0 : 32;
            pd -= back * dy_stride;
            px -= back * rows_stride;
            ps -= back * rows_stride;
            load(even);
            __builtin_amdgcn_sched_barrier(0);
            multiply(odd);
        }
        if (steps & 1) multiply(even);
    }
    const int64_t i = first + 32ll * steps;
    if (i < last) {                                        // fewer than 32 rows: the others are zeros
        GradStep<T, COLS> s;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const bool live = i + 8 * q + j < last;
            typename GradStep<T, COLS>::Vec none = (typename GradStep<T, COLS>::Vec)(T)0.0f;
            s.d[j] = none;
            s.code[j] = s.scale[j] = 0u;
            if (live) {
                s.d[j] = load_columns<T, COLS>(pd + j * dy_stride);
                s.code[j] = px[j * rows_stride];
                s.scale[j] = ps[j * rows_stride];
            }
        }
        multiply(s);
    }

    // half of the wavefronts hand their sums to the other half, until one is left
#pragma unroll
    for (int half = kGradWaves / 2; half > 0; half >>= 1) {
        __syncthreads();
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int t = 0; t < COLS; ++t)
#pragma unroll
                for (int u = 0; u < 8; ++u) sums[wave - half][t * 8 + u][lane] = acc[t][u];
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int t = 0; t < COLS; ++t)
#pragma unroll
                for (int u = 0; u < 8; ++u) acc[t][u] += sums[wave][t * 8 + u][lane];
        }
    }
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

// grad = the sum of the splits' parts, in their order.
__global__ void __launch_bounds__(256) k_mx4_grad_join(const float* __restrict__ parts, int splits, int64_t split_stride, int out_dim, int dim,
                                                       float* __restrict__ grad, int64_t grad_stride) {
    const int64_t total = (int64_t)out_dim * dim;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        float sum = 0.0f;
        for (int s = 0; s < splits; ++s) sum += parts[s * split_stride + i];
        grad[(i / dim) * grad_stride + i % dim] = sum;
    }
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
    const int quads = (dim + 127) / 128;
    const int rows = rows_per_group(ctx, n, quads, 16, 4);
    RG_FOR_TYPE(x_type, k_mx4_quantize<T><<<(unsigned)rg_div_up(n, rows), 256, 0, s>>>((const T*)x, x_stride, n, n_dev, dim, (uint32_t*)packed,
                                                                                  packed_stride, quads, rg_inverse(quads), rows));
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
    const int words = (dim + 7) / 8;
    const int rows = rows_per_group(ctx, n, words, 256, 4);
    RG_FOR_TYPE(x_type, k_mx4_dequantize<T><<<(unsigned)rg_div_up(n, rows), 256, 0, s>>>((const uint32_t*)packed, packed_stride, n, n_dev, dim,
                                                                                    (T*)x, x_stride, words, rg_inverse(words), rows));
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
    RG_FOR_TYPE(y_type, {
        if (n <= 256) {
            const dim3 grid(1, (unsigned)rg_div_up(out_dim, 16));
            k_mx4_matmul<T, 1, 1><<<dim3((unsigned)rg_div_up(n, 64), grid.y), 256, 0, s>>>((const uint32_t*)rows, rows_stride, n, n_dev, (const uint32_t*)weight,
                                                                               weight_stride, out_dim, groups, (T*)y, y_stride);
        } else {
            k_mx4_matmul<T, 2, 4><<<(unsigned)rg_min64(rg_div_up(n, 128), 1 << 20), 256, 0, s>>>((const uint32_t*)rows, rows_stride, n, n_dev, (const uint32_t*)weight,
                                                                         weight_stride, out_dim, groups, (T*)y, y_stride);
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
    const int cols = out_dim < 4 ? 1 : dy_type == RG_BF16 ? 4 : 2;
    const int tile_h = 16 * cols;
    const int tiles_h = (int)rg_div_up(out_dim, tile_h);
    const int64_t tiles = (int64_t)tiles_h * rg_div_up(dim, 128);
    const int64_t most = rg_max64(1, ctx->num_cus / tiles);
    const int64_t per_wave = rg_max64(1, rg_div_up(rg_div_up(n, most * kGradWaves), 32)) * 32;
    const int64_t splits = rg_max64(1, rg_div_up(n, per_wave * kGradWaves));
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
        constexpr int COLS = Parts<T>::count > 1 ? 2 : 4;
        const auto kernel = cols == 1 ? k_mx4_grad<T, 1> : k_mx4_grad<T, COLS>;
        kernel<<<grid, 64 * kGradWaves, 0, s>>>((const T*)dy, dy_stride, (const uint32_t*)rows, rows_stride, n, n_dev, out_dim, dim, per_wave,
                                                parts, parts_stride, split_stride, tiles_h, (int)tiles);
    });
    RG_LAUNCH_CHECK(ctx, "k_mx4_grad");
    if (splits > 1) {
        const int64_t blocks = rg_min64(rg_div_up(split_stride, 256), (int64_t)ctx->num_cus * 32);
        k_mx4_grad_join<<<(unsigned)blocks, 256, 0, s>>>(parts, (int)splits, split_stride, out_dim, dim, grad, grad_stride);
        RG_LAUNCH_CHECK(ctx, "k_mx4_grad_join");
    }
    return RG_OK;
}

}  // extern "C"
