// The norm of all gradients together, and clipping by it: scale = max_norm / norm where the norm is larger.  Squares are added up in 64 bits.  The norm is
// known when all numbers have been read, so they are read twice where they are scaled: three passes over memory.  246 M floats: 158 us for the norm (6.2
// TB/s), 343 for the scaling (5.7 TB/s, reading and writing).  Few numbers: two launches of 3.4 and 4.4 us (462 k); one workgroup in a single launch took 16.
#include "rg_elements.h"

#include <math.h>

namespace {

constexpr int kThreads = 256;
constexpr int kMostTensors = 64;       // that a launch's arguments describe
constexpr int kMostParts = 2048;       // workgroups of a launch (246 M floats' norm 321 / 202 / 158 us with 512 / 1024 / 2048)
// Numbers of a chunk: 8 KB of them, two loads of 16 bytes a thread.  (The last kernel with 4, 8, 16 or 32 KB: 462 k floats 4.7 / 4.6 / 5.3 / 5.9 us,
// 30 M 40.8 / 39.2 / 40.9 / 42.2.)
constexpr int log2_chunk(size_t bytes) { return bytes == 4 ? 11 : 12; }

struct ClipList {
    const void* in[kMostTensors];
    void* out[kMostTensors];
    int64_t size[kMostTensors];
    int32_t first[kMostTensors];       // chunks in front of each tensor (of those that are not there: as many as there can be)
    int32_t type[kMostTensors];        // (words: scalar loads drop the last two bits of each part of an address, and the compiler shares parts)
    int32_t chunks;
};

// The tensor that chunk `at` belongs to: every lane looks at one.
__device__ __forceinline__ int tensor_of(const ClipList& list, int at) {
    static_assert(kMostTensors == RG_WAVE, "a lane for a tensor");
    return __popcll(__ballot(list.first[rg_lane()] <= at)) - 1;
}

// f(numbers, place, how many) on every 16 bytes of the chunk that begins at p.
template <typename T, typename F>
__device__ __forceinline__ void for_chunk(const T* p, int64_t left, F f) {
    constexpr int V = 16 / (int)sizeof(T);
    const int n = (int)rg_least(left, 1 << log2_chunk(sizeof(T)));
#pragma unroll 1
    for (int at = (int)threadIdx.x * V; at < n; at += kThreads * V) {
        float v[V];
        rg_load_head<V>(p + at, n - at, v);
        f(v, at, n - at);
    }
}

// What another lane of the row of 16 holds.
template <int CTRL>
__device__ __forceinline__ double lane_of(double x) {
    const uint64_t u = __double_as_longlong(x);
    const uint32_t low = __builtin_amdgcn_update_dpp(0, (int)u, CTRL, 0xF, 0xF, false);
    const uint32_t high = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xF, 0xF, false);
    return __longlong_as_double((int64_t)((uint64_t)high << 32 | low));
}

// Sum over the workgroup, the same in each thread; smem holds a double for every 16 of them.  Contains a barrier.
__device__ __forceinline__ double block_sum(double x, double* smem) {
    // (between vector registers alone; after a step the lanes of half a group hold the same, so that mirrored lanes do for the other half)
    x += lane_of<0xB1>(x);                                 // lanes 1, 0, 3, 2 of four
    x += lane_of<0x4E>(x);                                 // 2, 3, 0, 1
    x += lane_of<0x141>(x);                                // 7, 6, .. 0 of eight
    x += lane_of<0x140>(x);                                // 15, 14, .. 0 of sixteen
    if (rg_lane() % 16 == 0) smem[threadIdx.x >> 4] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int i = 0; i < kThreads / 16; ++i) x += smem[i];
    return x;
}

// The factor that takes a gradient of this norm to max_norm, in two where it is small: the power of two below it (down to the smallest there is, which is
// enough for factors that leave anything of a 32-bit number) and a rest of at most 1, so that neither has few bits and what is multiplied by the first is no
// smaller than the result.
struct Scale {
    float coarse, fine;
    bool clipped;
};
__device__ __forceinline__ Scale scale_of(double norm, float max_norm) {
    Scale s;
    s.clipped = norm > (double)max_norm && norm <= 1.7976931348623157e308;
    const double scale = s.clipped ? (double)max_norm / norm : 1.0;
    const int power = (int)(__double_as_longlong(scale) >> 52) - 1022;         // scale in [2^(power - 1), 2^power)
    s.coarse = power < -64 && scale > 0.0 ? ldexpf(1.0f, max(power, -149)) : 1.0f;
    s.fine = (float)(scale / (double)s.coarse);
    return s;
}

// parts[workgroup] = the sum of the squares of its chunks.
__global__ void __launch_bounds__(kThreads) k_squares(ClipList list, double* __restrict__ parts) {
    __shared__ double smem[kThreads / 16];
    double sum = 0.0;
    for (int at = blockIdx.x; at < list.chunks; at += gridDim.x) {
        const int t = tensor_of(list, at);
        RG_FOR_TYPE((rg_dtype)list.type[t], {
            const int64_t begin = (int64_t)(at - list.first[t]) << log2_chunk(sizeof(T));
            for_chunk((const T*)list.in[t] + begin, list.size[t] - begin, [&](const auto& v, int, int) {
                for (float x : v) sum += (double)x * (double)x;
            });
        });
    }
    sum = block_sum(sum, smem);
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
}

// Every workgroup adds up the parts (in one order) and scales its chunks, the last ones first: the device's last level of cache still holds what
// was read last.
template <bool ONCE>
__global__ void __launch_bounds__(kThreads) k_clip(ClipList list, const double* __restrict__ parts, int num_parts, float max_norm,
                                                   float* __restrict__ norm_out) {
    __shared__ double smem[kThreads / 16];
    double sum = 0.0;
    constexpr int U = 8;                                   // on their way together
    for (int i0 = threadIdx.x; i0 < num_parts; i0 += kThreads * U) {
        double v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = parts[min(i0 + kThreads * u, num_parts - 1)];
#pragma unroll
        for (int u = 0; u < U; ++u) sum += i0 + kThreads * u < num_parts ? v[u] : 0.0;
    }
    const double norm = sqrt(block_sum(sum, smem));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const Scale scale = scale_of(norm, max_norm);
    for (int at = list.chunks - 1 - (int)blockIdx.x; at >= 0; at -= gridDim.x) {
        const int t = tensor_of(list, at);
        if (!scale.clipped && list.in[t] == list.out[t]) continue;
        RG_FOR_TYPE((rg_dtype)list.type[t], {
            const int64_t begin = (int64_t)(at - list.first[t]) << log2_chunk(sizeof(T));
            T* out = (T*)list.out[t] + begin;
            for_chunk((const T*)list.in[t] + begin, list.size[t] - begin, [&](auto& v, int place, int live) {
                for (float& x : v) x = x * scale.coarse * scale.fine;
                rg_store_live<16 / (int)sizeof(T), ONCE>(out + place, live, v);
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
    // the tensors that hold something, kMostTensors to a launch
    const auto fill = [&](ClipList& list, int32_t& next) {
        int64_t chunks = 0;
        int at = 0;
        for (; next < count && at < kMostTensors; ++next) {
            const rg_tensor& t = tensors[next];
            if (t.size == 0) continue;
            list.in[at] = t.in;
            list.out[at] = t.out;
            list.size[at] = t.size;
            list.type[at] = (int32_t)t.type;
            list.first[at++] = (int32_t)chunks;
            chunks += rg_div_up(t.size, 1ll << log2_chunk(rg_type_bytes(t.type)));
        }
        for (; at < kMostTensors; ++at) list.first[at] = INT32_MAX;
        list.chunks = (int32_t)chunks;
    };
    ClipList list;
    int32_t next = 0;
    const int64_t lists = rg_max64(1, rg_div_up(count, kMostTensors));
    const rg_status st = rg_scratch(ctx, ctx->clip_parts, (size_t)(lists * kMostParts) * sizeof(double), s, "rg_clip_grad_norm");
    if (st != RG_OK) return st;
    double* parts = (double*)ctx->clip_parts.p;
    int num_parts = 0;
    const auto grid_of = [](const ClipList& l) { return (unsigned)rg_max64(1, rg_min64(l.chunks, kMostParts)); };
    do {                                                   // (no tensor at all is a list of none)
        fill(list, next);
        k_squares<<<grid_of(list), kThreads, 0, s>>>(list, parts + num_parts);
        RG_LAUNCH_CHECK(ctx, "k_squares");
        num_parts += (int)grid_of(list);
    } while (next < count);
    const bool single = lists == 1;
    if (!single) next = 0;
    do {
        if (!single) fill(list, next);
        // (where there are more than 16 Mi numbers in all; where each of them lies is not asked: an array has few ends that share 16 bytes with others)
        const auto kernel = rg_store_once(nullptr, 16, 16, numbers / 8) ? k_clip<true> : k_clip<false>;
        kernel<<<grid_of(list), kThreads, 0, s>>>(list, parts, num_parts, max_norm, next == count ? norm : nullptr);
        RG_LAUNCH_CHECK(ctx, "k_clip");
    } while (next < count);
    return RG_OK;
}
