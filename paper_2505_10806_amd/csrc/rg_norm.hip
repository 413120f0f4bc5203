// Layer norm of rows and its backward pass.
#include "rg_elements.h"

namespace {

// A row lies in the registers of L = 2^log2L lanes: lane l holds chunks l, l + L, ... (NC of them) of V numbers, 16 bytes each.
template <typename T> struct Chunk { static constexpr int V = 16 / (int)sizeof(T); };
// Numbers of each of its rows that a lane holds at most: rows of up to 64 times as many stay in registers, longer ones are read again.  (50 k rows of
// 2048 floats 154 us, 198 if read again, of bf16 84 and 126; the gradient's of 1024 floats 116 and 209, of 1000 bf16 59 and 132.)
constexpr int kHeld = 32, kHeldGrad = 16;

// What another lane of the row of 16 holds.
template <int CTRL>
__device__ __forceinline__ float lane_of(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, false));
}

// Sums over groups of 2^log2L lanes, the same in each of them.  Between vector registers alone: by way of LDS a step of such a sum takes 120 cycles.
// After a step the lanes of half a group hold the same, so that mirrored lanes do for the other half.
template <int N>
__device__ __forceinline__ void group_sums(float (&x)[N], int log2L) {
#define RG_STEP(LOG2, ...) if (log2L >= LOG2) { _Pragma("unroll") for (int i = 0; i < N; ++i) { __VA_ARGS__; } }
    RG_STEP(1, x[i] += lane_of<0xB1>(x[i]))                // lanes 1, 0, 3, 2 of four
    RG_STEP(2, x[i] += lane_of<0x4E>(x[i]))                // 2, 3, 0, 1
    RG_STEP(3, x[i] += lane_of<0x141>(x[i]))               // 7, 6, .. 0 of eight
    RG_STEP(4, x[i] += lane_of<0x140>(x[i]))               // 15, 14, .. 0 of sixteen
    RG_STEP(5, const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[i]), __float_as_uint(x[i]), false, false);
            x[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]))
    RG_STEP(6, const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x[i]), __float_as_uint(x[i]), false, false);
            x[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]))
#undef RG_STEP
}

__device__ __forceinline__ float group_sum(float x, int log2L) {
    float v[1] = {x};
    group_sums(v, log2L);
    return v[0];
}

// Sum over a workgroup of NW wavefronts; smem holds NW floats.  Contains barriers.
template <int NW>
__device__ __forceinline__ float block_sum(float x, float* smem) {
    x = group_sum(x, 6);
    __syncthreads();
    if (rg_lane() == 0) smem[threadIdx.x >> 6] = x;
    __syncthreads();
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) sum += smem[w];
    return sum;
}

template <int V>
__device__ __forceinline__ void load_params(const float* p, int live, float absent, float (&v)[V]) {
    if (p) rg_load_head<V>(p, live, v);
    else {
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = absent;
    }
}

// A chunk of a row in 32 bits (END: one that may reach over the row's end, or not be there, as a lane's last may).
template <typename T, int V, bool END>
__device__ __forceinline__ void chunk_numbers(const typename RgPack<T, V>::type& a, int col, int dim, float (&v)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] = (float)a[j];
    if (END) rg_row_end<V>(v, col, dim);
}

// y = (x - m) s gamma + beta, m the mean, s = 1 / sqrt(mean of (x - m)^2 + eps): two sums, the second of differences that are formed before, so that
// nothing cancels.  A row is read once and stays in registers.  Bound by memory: 270 k rows of 256 floats, 555 MB, 93 us (5.9 TB/s); 1024 rows of 602
// bf16 5.1 us, a launch, a load and two sums.
template <typename T, int NC, bool ONCE>
__global__ void __launch_bounds__(256) k_layer_norm(const T* x, int64_t x_stride, int64_t n, const int32_t* __restrict__ n_dev, int dim,
                                                    const float* __restrict__ gamma, const float* __restrict__ beta, float eps, T* y,
                                                    int64_t y_stride, float* __restrict__ mean, float* __restrict__ rstd, int log2L) {
    constexpr int V = Chunk<T>::V;
    const int64_t n_act = rg_rows(n, n_dev);
    const int lane = rg_lane(), L = 1 << log2L, R = RG_WAVE >> log2L, l = lane & (L - 1);
    const int64_t wave = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 6, waves = ((int64_t)gridDim.x * blockDim.x) >> 6;
    if (wave * R >= n_act) return;
    struct Row {
        typename RgPack<T, V>::type x[NC];
    };
    const auto load = [&](Row& r, int64_t row) {
        const T* src = x + rg_least(row, n_act - 1) * x_stride;
#pragma unroll
        for (int i = 0; i < NC; ++i) r.x[i] = rg_load_row<V>(src, (l + i * L) * V, dim);
    };
    Row next;
    load(next, wave * R + (lane >> log2L));
    float g[NC][V], b[NC][V];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int col = (l + i * L) * V;
        load_params<V>(gamma ? gamma + col : nullptr, dim - col, 1.0f, g[i]);
        load_params<V>(beta ? beta + col : nullptr, dim - col, 0.0f, b[i]);
    }
    for (int64_t row0 = wave * R; row0 < n_act; row0 += waves * R) {
        const int64_t row = row0 + (lane >> log2L);
        const Row r = next;
        load(next, row + waves * R);                       // (on its way while this one is worked on)
        if (row >= n_act) continue;
        float v[NC][V];
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            if (i + 1 < NC && NC <= 4) chunk_numbers<T, V, false>(r.x[i], 0, dim, v[i]);
            else chunk_numbers<T, V, true>(r.x[i], (l + i * L) * V, dim, v[i]);
#pragma unroll
            for (int j = 0; j < V; ++j) sum += v[i][j];
        }
        const float m = group_sum(sum, log2L) / (float)dim;
        float square = 0.0f;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int col = (l + i * L) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                v[i][j] -= m;
                if ((i + 1 < NC && NC <= 4) || col + j < dim) square += v[i][j] * v[i][j];
            }
        }
        const float s = 1.0f / sqrtf(group_sum(square, log2L) / (float)dim + eps);
        T* dst = y + row * y_stride;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int col = (l + i * L) * V;
            if (col >= dim) continue;
#pragma unroll
            for (int j = 0; j < V; ++j) v[i][j] = v[i][j] * s * g[i][j] + b[i][j];
            rg_store_live<V, ONCE>(dst + col, dim - col, v[i]);
        }
        if (l == 0) {
            if (mean) mean[row] = m;
            if (rstd) rstd[row] = s;
        }
    }
}

// Rows too long for a wavefront's registers (and those of less than 16 bytes): a workgroup each, read three times, twice of them from the caches (50 k
// rows of 2056 bf16 165 us).
template <typename T>
__global__ void __launch_bounds__(256) k_layer_norm_long(const T* x, int64_t x_stride, int64_t n, const int32_t* __restrict__ n_dev, int dim,
                                                         const float* __restrict__ gamma, const float* __restrict__ beta, float eps, T* y,
                                                         int64_t y_stride, float* __restrict__ mean, float* __restrict__ rstd) {
    constexpr int V = Chunk<T>::V;
    __shared__ float smem[4];
    const int64_t n_act = rg_rows(n, n_dev);
    for (int64_t row = blockIdx.x; row < n_act; row += gridDim.x) {
        const T* src = x + row * x_stride;
        float sum = 0.0f, square = 0.0f, v[V];
        for (int col = threadIdx.x * V; col < dim; col += 256 * V) {
            rg_load_head<V>(src + col, dim - col, v);
#pragma unroll
            for (int j = 0; j < V; ++j) sum += v[j];
        }
        const float m = block_sum<4>(sum, smem) / (float)dim;
        for (int col = threadIdx.x * V; col < dim; col += 256 * V) {
            rg_load_head<V>(src + col, dim - col, v);
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (col + j < dim) square += (v[j] - m) * (v[j] - m);
        }
        const float s = 1.0f / sqrtf(block_sum<4>(square, smem) / (float)dim + eps);
        for (int col = threadIdx.x * V; col < dim; col += 256 * V) {
            float g[V], b[V];
            rg_load_head<V>(src + col, dim - col, v);
            load_params<V>(gamma ? gamma + col : nullptr, dim - col, 1.0f, g);
            load_params<V>(beta ? beta + col : nullptr, dim - col, 0.0f, b);
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = (v[j] - m) * s * g[j] + b[j];
            rg_store_live<V>(y + row * y_stride + col, dim - col, v);
        }
        if (threadIdx.x == 0) {
            if (mean) mean[row] = m;
            if (rstd) rstd[row] = s;
        }
    }
}

// ---------------------------------------------------------------- backward
// With h = (x - mean) rstd and g = dy gamma: dx = rstd (g - mean(g) - h mean(g h)), dgamma = sum of dy h over the rows, dbeta of dy.
// Every lane adds up dy h and dy of its columns over the rows it meets; a workgroup's sums go to its own part, which a second launch
// joins in the order of the workgroups.  Bound by memory: 794 k rows of 256 bf16, 1.23 GB, 215 us (5.7 TB/s) and 5 for the join.
constexpr int kGradThreads = 512, kGradWaves = kGradThreads / RG_WAVE;

template <typename T, int NC, bool ONCE>
__global__ void __launch_bounds__(kGradThreads) k_layer_norm_grad(const T* dy, int64_t dy_stride, const T* x, int64_t x_stride, int64_t n,
                                                                  const int32_t* __restrict__ n_dev, int dim, const float* __restrict__ gamma,
                                                                  const float* __restrict__ mean, const float* __restrict__ rstd, T* dx,
                                                                  int64_t dx_stride, float* __restrict__ parts, int log2L) {
    constexpr int V = Chunk<T>::V;
    extern __shared__ float wave_sums[];                   // [kGradWaves][dim]
    const int64_t n_act = rg_rows(n, n_dev);
    const int lane = rg_lane(), L = 1 << log2L, R = RG_WAVE >> log2L, l = lane & (L - 1);
    const int64_t wave = (int64_t)blockIdx.x * kGradWaves + (threadIdx.x >> 6), waves = (int64_t)gridDim.x * kGradWaves;
    float g[NC][V], by_gamma[NC][V], by_beta[NC][V];
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int col = (l + i * L) * V;
        load_params<V>(gamma ? gamma + col : nullptr, dim - col, 1.0f, g[i]);
#pragma unroll
        for (int j = 0; j < V; ++j) by_gamma[i][j] = by_beta[i][j] = 0.0f;
    }
    // the next row is on its way while this one is worked on
    struct Row {
        typename RgPack<T, V>::type x[NC], d[NC];
        float mean, rstd;
    };
    const auto load = [&](Row& r, int64_t row) {
        row = rg_least(row, n_act - 1);
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int col = (l + i * L) * V;
            r.x[i] = rg_load_row<V>(x + row * x_stride, col, dim);
            r.d[i] = rg_load_row<V>(dy + row * dy_stride, col, dim);
        }
        r.mean = mean[row];
        r.rstd = rstd[row];
    };
    Row next;
    if (wave * R < n_act) load(next, wave * R + (lane >> log2L));
    for (int64_t row0 = wave * R; row0 < n_act; row0 += waves * R) {
        const int64_t row = row0 + (lane >> log2L);
        const Row r = next;
        load(next, row + waves * R);
        if (row >= n_act) continue;
        float h[NC][V], d[NC][V];
        const float m = r.mean, s = r.rstd;
        float sums[2] = {0.0f, 0.0f};                      // of g h and of g
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            if (i + 1 < NC) {
                chunk_numbers<T, V, false>(r.x[i], 0, dim, h[i]);
                chunk_numbers<T, V, false>(r.d[i], 0, dim, d[i]);
            } else {
                chunk_numbers<T, V, true>(r.x[i], (l + i * L) * V, dim, h[i]);
                chunk_numbers<T, V, true>(r.d[i], (l + i * L) * V, dim, d[i]);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {                  // (behind the row's end dy is 0, and h: m s alone may be infinite where the row's own h are not)
                h[i][j] = i + 1 < NC || (l + i * L) * V + j < dim ? (h[i][j] - m) * s : 0.0f;
                by_gamma[i][j] += d[i][j] * h[i][j];
                by_beta[i][j] += d[i][j];
                d[i][j] *= g[i][j];
                sums[0] += d[i][j] * h[i][j];
                sums[1] += d[i][j];
            }
        }
        if (!dx) continue;
        group_sums(sums, log2L);
        const float along = sums[0] / (float)dim, all = sums[1] / (float)dim;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int col = (l + i * L) * V;
            if (col >= dim) continue;
#pragma unroll
            for (int j = 0; j < V; ++j) d[i][j] = s * (d[i][j] - all - h[i][j] * along);
            rg_store_live<V, ONCE>(dx + row * dx_stride + col, dim - col, d[i]);
        }
    }
    if (!parts) return;                                    // (not wanted; adding them up is no more than the loads leave time for)
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NC; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int col = (l + i * L) * V + j;
                float sum = which ? by_beta[i][j] : by_gamma[i][j];
                for (int off = L; off < RG_WAVE; off <<= 1) sum += __shfl_xor(sum, off, RG_WAVE);
                if (lane < L && col < dim) wave_sums[(threadIdx.x >> 6) * dim + col] = sum;
            }
        __syncthreads();
        for (int col = threadIdx.x; col < dim; col += kGradThreads) {
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kGradWaves; ++w) sum += wave_sums[w * dim + col];
            parts[((int64_t)blockIdx.x * 2 + which) * dim + col] = sum;
        }
    }
}

// Column sums of `count` parts: 64 columns to a workgroup, 16 runs of parts side by side.
__global__ void __launch_bounds__(1024) k_norm_join(const float* __restrict__ parts, int count, int dim, float* __restrict__ dgamma,
                                                    float* __restrict__ dbeta) {
    __shared__ float runs[16][64];
    const int lane = threadIdx.x & 63, run = threadIdx.x >> 6;
    const int col = blockIdx.x * 64 + lane;                // of both rows of a part, one behind the other
    const int per_run = (count + 15) / 16, first = run * per_run, last = min(first + per_run, count);
    float sum = 0.0f;
    if (col < 2 * dim) {
#pragma unroll 8
        for (int b = first; b < last; ++b) sum += parts[(int64_t)b * 2 * dim + col];
    }
    runs[run][lane] = sum;
    __syncthreads();
    if (run != 0 || col >= 2 * dim) return;
    sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) sum += runs[r][lane];
    if (col < dim) {
        if (dgamma) dgamma[col] = sum;
    } else if (dbeta) dbeta[col - dim] = sum;
}

// Longer rows: a workgroup to a row for dx ...
template <typename T>
__global__ void __launch_bounds__(256) k_layer_norm_grad_long(const T* dy, int64_t dy_stride, const T* x, int64_t x_stride, int64_t n,
                                                              const int32_t* __restrict__ n_dev, int dim, const float* __restrict__ gamma,
                                                              const float* __restrict__ mean, const float* __restrict__ rstd, T* dx,
                                                              int64_t dx_stride) {
    constexpr int V = Chunk<T>::V;
    __shared__ float smem[4];
    const int64_t n_act = rg_rows(n, n_dev);
    for (int64_t row = blockIdx.x; row < n_act; row += gridDim.x) {
        const float m = mean[row], s = rstd[row];
        float along = 0.0f, all = 0.0f, h[V], d[V], g[V];
        for (int col = threadIdx.x * V; col < dim; col += 256 * V) {
            rg_load_head<V>(x + row * x_stride + col, dim - col, h);
            rg_load_head<V>(dy + row * dy_stride + col, dim - col, d);
            load_params<V>(gamma ? gamma + col : nullptr, dim - col, 1.0f, g);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                along += col + j < dim ? d[j] * g[j] * ((h[j] - m) * s) : 0.0f;
                all += d[j] * g[j];
            }
        }
        along = block_sum<4>(along, smem) / (float)dim;
        all = block_sum<4>(all, smem) / (float)dim;
        for (int col = threadIdx.x * V; col < dim; col += 256 * V) {
            rg_load_head<V>(x + row * x_stride + col, dim - col, h);
            rg_load_head<V>(dy + row * dy_stride + col, dim - col, d);
            load_params<V>(gamma ? gamma + col : nullptr, dim - col, 1.0f, g);
#pragma unroll
            for (int j = 0; j < V; ++j) d[j] = s * (d[j] * g[j] - all - (h[j] - m) * s * along);
            rg_store_live<V>(dx + row * dx_stride + col, dim - col, d);
        }
    }
}

// ... and, before dx takes their place, a workgroup to 64 chunks of columns and a range of the rows for the sums.  (Both and the join, 50 k rows of 1032 numbers
// of bf16: 144 us; of 1000 numbers, which lanes hold, 59.)
template <typename T>
__global__ void __launch_bounds__(256) k_layer_norm_sums_long(const T* __restrict__ dy, int64_t dy_stride, const T* __restrict__ x, int64_t x_stride,
                                                              int64_t n, const int32_t* __restrict__ n_dev, int dim, const float* __restrict__ mean,
                                                              const float* __restrict__ rstd, float* __restrict__ parts) {
    constexpr int V = Chunk<T>::V;
    __shared__ float runs[2][4][64 * V];
    const int64_t n_act = rg_rows(n, n_dev);
    const int lane = rg_lane(), wave = threadIdx.x >> 6;
    const int col = (blockIdx.x * 64 + lane) * V;
    float by_gamma[V], by_beta[V];
#pragma unroll
    for (int j = 0; j < V; ++j) by_gamma[j] = by_beta[j] = 0.0f;
    for (int64_t row = blockIdx.y * 4 + wave; row < n_act; row += gridDim.y * 4) {
        float h[V], d[V];
        rg_load_head<V>(x + row * x_stride + col, dim - col, h);
        rg_load_head<V>(dy + row * dy_stride + col, dim - col, d);
        const float m = mean[row], s = rstd[row];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            by_gamma[j] += d[j] * ((h[j] - m) * s);
            by_beta[j] += d[j];
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        runs[0][wave][lane * V + j] = by_gamma[j];
        runs[1][wave][lane * V + j] = by_beta[j];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * V; i += 256) {
        const int at = blockIdx.x * 64 * V + i;
        if (at >= dim) continue;
#pragma unroll
        for (int which = 0; which < 2; ++which)
            parts[((int64_t)blockIdx.y * 2 + which) * dim + at] =
                (runs[which][0][i] + runs[which][1][i]) + (runs[which][2][i] + runs[which][3][i]);
    }
}

// Lanes to a row and chunks to a lane: the smallest number of lane slots that holds the row's chunks.
struct Shape {
    int log2L, chunks;         // chunks = 0: too long to be held, or too short for a load of 16 bytes
};

Shape row_shape(int dim, int V, int held) {
    const int total = (int)rg_div_up(dim, V);
    Shape best = {6, 0};
    if (dim < V) return best;                              // (shorter than a load)
    int slots = 1 << 30;
    for (int log2L = 6; log2L >= 0; --log2L) {
        int per = (int)rg_div_up(total, 1 << log2L);
        if (per > 4) per = per <= held / V ? held / V : 0;          // 1, 2, 3, 4 or as many as are held
        if (per == 0 || per * V > held) continue;
        if (per << log2L < slots) { slots = per << log2L; best = {log2L, per}; }
    }
    return best;
}

#define RG_FOR_CHUNKS(shape, most, ...)                                            \
    do {                                                                        \
        if ((shape).chunks == 1) { constexpr int NC = 1; __VA_ARGS__; }         \
        else if ((shape).chunks == 2) { constexpr int NC = 2; __VA_ARGS__; }    \
        else if ((shape).chunks == 3) { constexpr int NC = (most) < 3 ? (most) : 3; __VA_ARGS__; }    \
        else if ((shape).chunks == 4) { constexpr int NC = (most) < 4 ? (most) : 4; __VA_ARGS__; }    \
        else { constexpr int NC = (most); __VA_ARGS__; }                        \
    } while (0)

bool aligned(const void* p, int bytes) { return (uintptr_t)p % (uintptr_t)bytes == 0; }

}  // namespace

extern "C" {

rg_status rg_layer_norm(rg_ctx* ctx, const void* x, rg_dtype type, int64_t x_stride, int64_t n, const int32_t* n_dev, int32_t dim,
                        const float* gamma, const float* beta, float eps, void* y, int64_t y_stride, float* mean, float* rstd, void* stream) {
    if (!ctx) return RG_ERR_INVALID_ARG;
    RG_REQUIRE(ctx, n >= 0 && n <= (1ll << 31) - 1, "rg_layer_norm: n = %lld out of range", (long long)n);
    RG_REQUIRE(ctx, dim >= 1 && dim <= RG_NORM_MAX_DIM, "rg_layer_norm: dim = %d not in [1,%d]", dim, RG_NORM_MAX_DIM);
    RG_REQUIRE(ctx, rg_type_known(type), "rg_layer_norm: unknown type %d", (int)type);
    RG_REQUIRE(ctx, x_stride >= dim && y_stride >= dim, "rg_layer_norm: bad stride");
    RG_REQUIRE(ctx, eps >= 0.0f, "rg_layer_norm: eps is negative or not a number");
    if (n == 0) return RG_OK;
    RG_REQUIRE(ctx, x && y, "rg_layer_norm: null pointer");
    RG_REQUIRE(ctx, x != y || x_stride == y_stride, "rg_layer_norm: y is x with another stride");
    RG_REQUIRE(ctx, aligned(x, rg_type_bytes(type)) && aligned(y, rg_type_bytes(type)) && aligned(gamma, 4) && aligned(beta, 4) &&
               aligned(mean, 4) && aligned(rstd, 4), "rg_layer_norm: pointer not aligned to its numbers");
    RG_HIP(ctx, hipSetDevice(ctx->device));
    hipStream_t s = (hipStream_t)stream;
    RG_FOR_TYPE(type, {
        const Shape shape = row_shape(dim, Chunk<T>::V, kHeld);
        if (shape.chunks == 0) {
            k_layer_norm_long<T><<<(unsigned)rg_min64(n, (int64_t)ctx->num_cus * 32), 256, 0, s>>>((const T*)x, x_stride, n, n_dev, dim, gamma,
                                                                                                  beta, eps, (T*)y, y_stride, mean, rstd);
        } else {
            // (270 k rows of 256 floats 120 / 112 / 104 / 97 / 116 us with 8 / 16 / 32 / 64 / 256 workgroups to a compute unit)
            const unsigned grid = (unsigned)rg_min64(rg_div_up(n, 4 * (RG_WAVE >> shape.log2L)), (int64_t)ctx->num_cus * 64);
            const bool once = rg_store_once(y, dim * sizeof(T), y_stride * sizeof(T), n);
            RG_FOR_CHUNKS(shape, kHeld / Chunk<T>::V, {
                const auto kernel = once ? k_layer_norm<T, NC, true> : k_layer_norm<T, NC, false>;
                kernel<<<grid, 256, 0, s>>>((const T*)x, x_stride, n, n_dev, dim, gamma, beta, eps, (T*)y, y_stride, mean, rstd, shape.log2L);
            });
        }
    });
    RG_LAUNCH_CHECK(ctx, "k_layer_norm");
    return RG_OK;
}

rg_status rg_layer_norm_grad(rg_ctx* ctx, const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, rg_dtype type, int64_t n,
                             const int32_t* n_dev, int32_t dim, const float* gamma, const float* mean, const float* rstd, void* dx,
                             int64_t dx_stride, float* dgamma, float* dbeta, void* stream) {
    if (!ctx) return RG_ERR_INVALID_ARG;
    RG_REQUIRE(ctx, n >= 0 && n <= (1ll << 31) - 1, "rg_layer_norm_grad: n = %lld out of range", (long long)n);
    RG_REQUIRE(ctx, dim >= 1 && dim <= RG_NORM_MAX_DIM, "rg_layer_norm_grad: dim = %d not in [1,%d]", dim, RG_NORM_MAX_DIM);
    RG_REQUIRE(ctx, rg_type_known(type), "rg_layer_norm_grad: unknown type %d", (int)type);
    RG_REQUIRE(ctx, dy_stride >= dim && x_stride >= dim && (!dx || dx_stride >= dim), "rg_layer_norm_grad: bad stride");
    RG_REQUIRE(ctx, n == 0 || (dy && x && mean && rstd), "rg_layer_norm_grad: null pointer");
    RG_REQUIRE(ctx, !dx || ((dx != x || dx_stride == x_stride) && (dx != dy || dx_stride == dy_stride)),
               "rg_layer_norm_grad: dx is an input with another stride");
    const int b = rg_type_bytes(type);
    RG_REQUIRE(ctx, aligned(dy, b) && aligned(x, b) && aligned(dx, b) && aligned(gamma, 4) && aligned(mean, 4) && aligned(rstd, 4) &&
               aligned(dgamma, 4) && aligned(dbeta, 4), "rg_layer_norm_grad: pointer not aligned to its numbers");
    const bool sums = dgamma || dbeta;
    if (!sums && (!dx || n == 0)) return RG_OK;
    RG_HIP(ctx, hipSetDevice(ctx->device));
    hipStream_t s = (hipStream_t)stream;
    int64_t blocks = 0;
    RG_FOR_TYPE(type, {
        constexpr int V = Chunk<T>::V;
        const Shape shape = row_shape(dim, V, kHeldGrad);
        const int64_t stripes = rg_div_up(dim, 64 * V);
        if (shape.chunks == 0) blocks = rg_max64(1, rg_min64(rg_div_up(n, 16), rg_div_up((int64_t)ctx->num_cus * 8, stripes)));
        // Two workgroups to a compute unit (1.5 M rows of 100 numbers of bf16 197 / 182 / 217 / 188 us with 1 / 2 / 3 / 4, 794 k of 256 215 / 217 / 240 /
        // 222), one where lanes hold several chunks of a row, whose sums take longer to join (200 k rows of 602 numbers: of bf16 156 / 160 / 166 / 172, of f32
        // 269 / 278 / 282 / 282).
        else blocks = rg_max64(1, rg_min64(rg_div_up(n, kGradWaves * (RG_WAVE >> shape.log2L)), (int64_t)ctx->num_cus * (shape.chunks > 1 ? 1 : 2)));
        if (sums) {
            const rg_status st = rg_scratch(ctx, ctx->norm_parts, (size_t)blocks * 2 * dim * 4, s, "rg_layer_norm_grad");
            if (st != RG_OK) return st;
        }
        float* parts = sums ? (float*)ctx->norm_parts.p : nullptr;
        if (shape.chunks == 0) {
            if (sums)
                k_layer_norm_sums_long<T><<<dim3((unsigned)stripes, (unsigned)blocks), 256, 0, s>>>((const T*)dy, dy_stride, (const T*)x, x_stride, n,
                                                                                               n_dev, dim, mean, rstd, parts);
            if (dx && n > 0)
                k_layer_norm_grad_long<T><<<(unsigned)rg_min64(n, (int64_t)ctx->num_cus * 32), 256, 0, s>>>(
                    (const T*)dy, dy_stride, (const T*)x, x_stride, n, n_dev, dim, gamma, mean, rstd, (T*)dx, dx_stride);
        } else {
            const size_t lds = sums ? (size_t)kGradWaves * dim * 4 : 0;
            const bool once = rg_store_once(dx, dim * sizeof(T), dx_stride * sizeof(T), n);
            RG_FOR_CHUNKS(shape, kHeldGrad / V, {
                const auto kernel = once ? k_layer_norm_grad<T, NC, true> : k_layer_norm_grad<T, NC, false>;
                kernel<<<(unsigned)blocks, kGradThreads, lds, s>>>((const T*)dy, dy_stride, (const T*)x, x_stride, n, n_dev, dim, gamma, mean, rstd,
                                                                   (T*)dx, dx_stride, parts, shape.log2L);
            });
        }
        RG_LAUNCH_CHECK(ctx, "k_layer_norm_grad");
    });
    if (sums) {
        k_norm_join<<<(unsigned)rg_div_up(2ll * dim, 64), 1024, 0, s>>>((const float*)ctx->norm_parts.p, (int)blocks, dim, dgamma, dbeta);
        RG_LAUNCH_CHECK(ctx, "k_norm_join");
    }
    return RG_OK;
}

}  // extern "C"
