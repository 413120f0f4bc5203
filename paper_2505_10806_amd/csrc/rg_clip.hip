// The norm of all gradients together, and clipping by it.
#include "rg_elements.h"

#include <math.h>

namespace {

constexpr int kThreads = 256;
constexpr int kMostTensors = 64;       // that a launch's arguments describe
constexpr int kChunk = 8192;           // numbers a workgroup takes at a time
constexpr int kMostParts = 2048;       // workgroups of a launch

struct ClipList {
    const void* in[kMostTensors];
    void* out[kMostTensors];
    int64_t size[kMostTensors];
    int64_t first[kMostTensors + 1];   // chunks in front of each tensor
    uint8_t type[kMostTensors];
    int count;
};

// The tensor that chunk `at` belongs to (the last with first <= at: empty ones own none).
__device__ __forceinline__ int tensor_of(const ClipList& list, int64_t at) {
    int lo = 0, hi = list.count;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (list.first[mid] <= at) lo = mid;
        else hi = mid;
    }
    return lo;
}

// f(numbers, place) on every 16 bytes of the chunk, f(number, place) one by one at its end.
template <typename T, typename F>
__device__ __forceinline__ void for_chunk(const T* p, int64_t left, F f) {
    constexpr int V = 16 / (int)sizeof(T);
    const int n = (int)rg_least(left, kChunk);
#pragma unroll
    for (int i = 0; i < kChunk / (kThreads * V); ++i) {
        const int at = (i * kThreads + (int)threadIdx.x) * V;
        float v[V];
        if (at < n) {
            rg_load_head<V>(p + at, n - at, v);
            f(v, at, n - at);
        }
    }
}

__device__ __forceinline__ double block_sum(double x, double* smem) {
#pragma unroll
    for (int off = RG_WAVE / 2; off > 0; off >>= 1) x += __shfl_xor(x, off, RG_WAVE);
    __syncthreads();
    if (rg_lane() == 0) smem[threadIdx.x >> 6] = x;
    __syncthreads();
    return (smem[0] + smem[1]) + (smem[2] + smem[3]);
}

// parts[workgroup] = the sum of the squares of its chunks.
__global__ void __launch_bounds__(kThreads) k_squares(ClipList list, double* __restrict__ parts) {
    __shared__ double smem[kThreads / RG_WAVE];
    double sum = 0.0;
    for (int64_t at = blockIdx.x; at < list.first[list.count]; at += gridDim.x) {
        const int t = tensor_of(list, at);
        const int64_t begin = (at - list.first[t]) * kChunk;
        RG_FOR_TYPE(list.type[t], for_chunk((const T*)list.in[t] + begin, list.size[t] - begin, [&](const auto& v, int, int) {
            for (float x : v) sum += (double)x * (double)x;
        }));
    }
    sum = block_sum(sum, smem);
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

// Every workgroup adds up the parts (in one order) and scales its chunks.
__global__ void __launch_bounds__(kThreads) k_clip(ClipList list, const double* __restrict__ parts, int num_parts, float max_norm,
                                                   float* __restrict__ norm_out) {
    __shared__ double smem[kThreads / RG_WAVE];
    double sum = 0.0;
    for (int i = threadIdx.x; i < num_parts; i += kThreads) sum += parts[i];
    const double norm = sqrt(block_sum(sum, smem));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const bool clipped = norm > (double)max_norm && norm <= 1.7976931348623157e308;
    // in two factors, so that a norm beyond the 32-bit range does not leave a scale of few bits
    const double scale = clipped ? (double)max_norm / norm : 1.0;
    const float coarse = scale < 0x1p-64 ? 0x1p-64f : 1.0f, fine = (float)(scale / (double)coarse);
    for (int64_t at = blockIdx.x; at < list.first[list.count]; at += gridDim.x) {
        const int t = tensor_of(list, at);
        if (!clipped && list.in[t] == list.out[t]) continue;
        const int64_t begin = (at - list.first[t]) * kChunk;
        RG_FOR_TYPE(list.type[t], {
            T* out = (T*)list.out[t] + begin;
            for_chunk((const T*)list.in[t] + begin, list.size[t] - begin, [&](auto& v, int place, int live) {
                for (float& x : v) x = x * coarse * fine;
                rg_store_live<16 / (int)sizeof(T)>(out + place, live, v);
            });
        });
    }
}

}  // namespace

extern "C" rg_status rg_clip_grad_norm(rg_ctx* ctx, const rg_tensor* tensors, int32_t count, float max_norm, float* norm, void* stream) {
    if (!ctx) return RG_ERR_INVALID_ARG;
    RG_REQUIRE(ctx, count >= 0 && (count == 0 || tensors), "rg_clip_grad_norm: count = %d, or no tensors", count);
    RG_REQUIRE(ctx, max_norm >= 0.0f, "rg_clip_grad_norm: max_norm is negative or not a number");
    RG_REQUIRE(ctx, norm && (uintptr_t)norm % 4 == 0, "rg_clip_grad_norm: norm is NULL or not aligned");
    int64_t numbers = 0;
    for (int32_t i = 0; i < count; ++i) {
        const rg_tensor& t = tensors[i];
        RG_REQUIRE(ctx, t.size >= 0 && t.size < (1ll << 40) - numbers, "rg_clip_grad_norm: tensor %d: size = %lld out of range", i, (long long)t.size);
        numbers += t.size;
        RG_REQUIRE(ctx, rg_type_known(t.type), "rg_clip_grad_norm: tensor %d: unknown type %d", i, (int)t.type);
        if (t.size == 0) continue;
        RG_REQUIRE(ctx, t.in && t.out, "rg_clip_grad_norm: tensor %d: null pointer", i);
        const uintptr_t b = (uintptr_t)rg_type_bytes(t.type);
        RG_REQUIRE(ctx, (uintptr_t)t.in % b == 0 && (uintptr_t)t.out % b == 0, "rg_clip_grad_norm: tensor %d: pointer not aligned to its numbers", i);
    }
    RG_HIP(ctx, hipSetDevice(ctx->device));
    hipStream_t s = (hipStream_t)stream;
    const int64_t lists = rg_max64(1, rg_div_up(count, kMostTensors));
    rg_status st = rg_scratch(ctx, ctx->clip_parts, (size_t)(lists * kMostParts) * sizeof(double), s, "rg_clip_grad_norm");
    if (st != RG_OK) return st;
    double* parts = (double*)ctx->clip_parts.p;
    ClipList list;
    const auto fill = [&](int64_t which) {
        list.count = 0;
        list.first[0] = 0;
        for (int64_t i = which * kMostTensors; i < rg_min64(count, (which + 1) * kMostTensors); ++i) {
            const rg_tensor& t = tensors[i];
            if (t.size == 0) continue;
            const int at = list.count++;
            list.in[at] = t.in;
            list.out[at] = t.out;
            list.size[at] = t.size;
            list.type[at] = (uint8_t)t.type;
            list.first[at + 1] = list.first[at] + rg_div_up(t.size, kChunk);
        }
        return (unsigned)rg_max64(1, rg_min64(list.first[list.count], kMostParts));
    };
    int num_parts = 0;
    for (int64_t w = 0; w < lists; ++w) {
        const unsigned grid = fill(w);
        k_squares<<<grid, kThreads, 0, s>>>(list, parts + num_parts);
        RG_LAUNCH_CHECK(ctx, "k_squares");
        num_parts += (int)grid;
    }
    for (int64_t w = 0; w < lists; ++w) {
        const unsigned grid = lists > 1 ? fill(w) : (unsigned)rg_max64(1, rg_min64(list.first[list.count], kMostParts));
        k_clip<<<grid, kThreads, 0, s>>>(list, parts, num_parts, max_norm, w == 0 ? norm : nullptr);
        RG_LAUNCH_CHECK(ctx, "k_clip");
    }
    return RG_OK;
}
