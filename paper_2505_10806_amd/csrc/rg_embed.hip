// Rows of a table by id, and the gradient of the rows that were looked up, summed by id.
#include <type_traits>

#include "rg_elements.h"

namespace {

constexpr int kThreads = 256;

// What lanes of a wavefront exchange through LDS stands between these: they execute together.
__device__ __forceinline__ void wave_exchange() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// V numbers of a row from column `col`, in 32 bits (SHORT: of rows shorter than V).
template <int V, bool SHORT, typename T>
__device__ __forceinline__ typename RgPack<T, V>::type load_chunk(const T* row, int col, int dim) {
    if constexpr (SHORT) return rg_load_raw<V>(row + col, dim - col);
    else return rg_load_row<V>(row, col, dim);
}
template <int V, bool SHORT, typename P>
__device__ __forceinline__ void chunk_numbers(const P& a, int col, int dim, float (&v)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (float)a[i];
    if (!SHORT) rg_row_end<V>(v, col, dim);
}

// ---------------------------------------------------------------- lookup
// y[i] = scale table[ids[i]].  A workgroup takes `group` rows and deals their chunks of V numbers to its threads, kAhead of them on their way at a time: rows
// of any length fill the lanes.  V is what fills 16 bytes of the narrower type.  Bound by memory: 794 k rows of 256 bf16 out of 10 M, 150 us, 5.4 TB/s read and written.
constexpr int kAhead = 4;

template <typename T, typename U, int V, bool SHORT, bool ONCE>
__global__ void __launch_bounds__(kThreads) k_embedding(const T* __restrict__ table, int64_t table_stride, int num_rows, const int32_t* __restrict__ ids,
                                                        int64_t n, const int32_t* __restrict__ n_dev, int dim, int chunks, uint32_t inverse, int group,
                                                        float scale, U* __restrict__ y, int64_t y_stride) {
    const int64_t n_act = rg_rows(n, n_dev);
    for (int64_t first = (int64_t)blockIdx.x * group; first < n_act; first += (int64_t)gridDim.x * group) {
        const int total = (int)rg_least(group, n_act - first) * chunks;
        for (int i0 = threadIdx.x; i0 < total; i0 += kThreads * kAhead) {
            int row[kAhead], col[kAhead], id[kAhead];
            typename RgPack<T, V>::type a[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int i = min(i0 + u * kThreads, total - 1);
                row[u] = (int)rg_divide((uint32_t)i, inverse);
                col[u] = (i - row[u] * chunks) * V;
                id[u] = ids[first + row[u]];
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {             // (padding reads row 0, and is cleared below)
                const int from = (uint32_t)id[u] < (uint32_t)num_rows ? id[u] : 0;
                a[u] = load_chunk<V, SHORT>(table + from * table_stride, col[u], dim);
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (i0 + u * kThreads >= total) break;
                float v[V];
                chunk_numbers<V, SHORT>(a[u], col[u], dim, v);
                const bool there = (uint32_t)id[u] < (uint32_t)num_rows;
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = there ? v[j] * scale : 0.0f;
                rg_store_live<V, ONCE>(y + (first + row[u]) * y_stride + col[u], dim - col[u], v);
            }
        }
    }
}

// ---------------------------------------------------------------- zeros
// Rows of a whole table that no id meets are zeros: all of it is cleared first, by workgroups of their own beside those of the launches that sort the ids (which
// wait for each other more than they work: 65536 ids take 33 us in four launches, with 102 MB of zeros beside them).  pieces `from` .. `to` - 1 of 16 bytes, `chunks` to a row.
struct Zeros {
    void* grad;
    int64_t stride, from, to;
    int dim, chunks, bytes, once;
};

template <typename U, bool ONCE>
__device__ __forceinline__ void clear_as(const Zeros& z, int block, int blocks) {
    constexpr int V = 16 / (int)sizeof(U);
    const float zero[V] = {};
    for (int64_t i = z.from + (int64_t)block * blockDim.x + threadIdx.x; i < z.to; i += (int64_t)blocks * blockDim.x) {
        const int64_t row = i / z.chunks;
        const int col = (int)(i - row * z.chunks) * V;
        rg_store_live<V, ONCE>((U*)z.grad + row * z.stride + col, z.dim - col, zero);
    }
}

__device__ __forceinline__ void clear(const Zeros& z, int block, int blocks) {
    if (z.bytes == 4) z.once ? clear_as<float, true>(z, block, blocks) : clear_as<float, false>(z, block, blocks);
    else z.once ? clear_as<_Float16, true>(z, block, blocks) : clear_as<_Float16, false>(z, block, blocks);
}

__global__ void __launch_bounds__(kThreads) k_clear_rows(const Zeros z) { clear(z, blockIdx.x, gridDim.x); }

// ---------------------------------------------------------------- ids in order
// The gradient's sums run over the entries sorted by id, entries of an id in their own order, so that the same call adds in the same order each time.  Least
// digit first, 8 to 10 bits a pass, as many as leave the fewest passes; padding gets the id behind the last row and comes to lie behind all others.  What bounds a pass of
// few ids is that its launches wait for each other: 794 k ids take 6 + 5 + 11 us a pass of 8 bits (counts, sums, places), 65 k ids 6 + 11 of 9 bits, zeros beside.
struct Entry {
    uint32_t id, at;
};

constexpr int kRounds = 4, kTile = kThreads * kRounds, kSortWaves = kThreads / RG_WAVE;
// Up to this many blocks a pass takes two launches instead of three, the counts added up by every block of the second (a gradient of 16384 / 65536 / 131072 / 524288
// rows of 32 numbers into 200000 takes 35 / 41.5 / 53 / 145 us so, and 36.5 / 42 / 48 / 88 with the launch between).
constexpr int kDirectBlocks = 64;

__device__ __forceinline__ Entry entry_of(const Entry* from, const int32_t* ids, int64_t i, uint32_t num_rows) {
    if (from) return from[i];
    const uint32_t id = (uint32_t)ids[i];
    return {id < num_rows ? id : num_rows, (uint32_t)i};
}

// Lanes that hold the same digit as this one.
template <int BITS>
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, bool live) {
    uint64_t mask = __ballot(live);
#pragma unroll
    for (int b = 0; b < BITS; ++b) {
        const uint64_t set = __ballot(digit >> b & 1);
        mask &= digit >> b & 1 ? set : ~set;
    }
    return mask;
}

// DIRECT: of few blocks; counts lie [block][digit] and the scatter adds them up itself.
template <int BITS, bool DIRECT>
__global__ void __launch_bounds__(kThreads) k_sort_count(const Zeros zeros, int blocks, const Entry* __restrict__ from, const int32_t* __restrict__ ids, int64_t n,
                                                         const int32_t* __restrict__ n_dev, uint32_t num_rows, int shift, int64_t per_block,
                                                         int32_t* __restrict__ counts) {
    constexpr int DIGITS = 1 << BITS;
    __shared__ int32_t bins[DIGITS];
    if ((int)blockIdx.x >= blocks) return clear(zeros, blockIdx.x - blocks, gridDim.x - blocks);
#pragma unroll
    for (int d = threadIdx.x; d < DIGITS; d += kThreads) bins[d] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * per_block, last = rg_least(first + per_block, rg_rows(n, n_dev));
    for (int64_t i = first + threadIdx.x; i < last; i += kThreads) atomicAdd(&bins[entry_of(from, ids, i, num_rows).id >> shift & (DIGITS - 1)], 1);
    __syncthreads();
#pragma unroll
    for (int d = threadIdx.x; d < DIGITS; d += kThreads) counts[DIRECT ? blockIdx.x * DIGITS + d : (int64_t)d * blocks + blockIdx.x] = bins[d];
}

// Each digit's counts become its entries in front of every block; totals[digit] = all of them.  A workgroup to a digit; 5 us of 776 blocks.
__global__ void __launch_bounds__(kThreads) k_sort_scan(const Zeros zeros, int digits, int32_t* __restrict__ counts, int blocks, int32_t* __restrict__ totals) {
    __shared__ int smem[kSortWaves + 1];
    if ((int)blockIdx.x >= digits) return clear(zeros, blockIdx.x - digits, gridDim.x - digits);
    constexpr int EACH = 4;
    int32_t* row = counts + (int64_t)blockIdx.x * blocks;
    int before = 0;
    for (int b0 = 0; b0 < blocks; b0 += kThreads * EACH) {
        const int b = b0 + threadIdx.x * EACH;
        int x[EACH], sum = 0, total;
#pragma unroll
        for (int i = 0; i < EACH; ++i) x[i] = row[min(b + i, blocks - 1)];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            x[i] = b + i < blocks ? x[i] : 0;
            sum += x[i];
        }
        int at = before + rg_block_excl_scan<kSortWaves>(sum, smem, &total);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (b + i < blocks) row[b + i] = at;
            at += x[i];
        }
        before += total;
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = before;
}

// A block's entries to their places, in their order: a wavefront finds the entries before a lane's of the same digit by votes on its bits, wavefronts add up in LDS.
template <int BITS, bool DIRECT>
__global__ void __launch_bounds__(kThreads) k_sort_scatter(const Zeros zeros, int blocks, const Entry* __restrict__ from, const int32_t* __restrict__ ids, int64_t n,
                                                           const int32_t* __restrict__ n_dev, uint32_t num_rows, int shift, int64_t per_block,
                                                           const int32_t* __restrict__ counts, const int32_t* __restrict__ totals, Entry* __restrict__ to) {
    constexpr int DIGITS = 1 << BITS, EACH = DIGITS / kThreads;          // (a thread: EACH neighbouring digits)
    __shared__ int smem[kSortWaves + 1];
    __shared__ int32_t next[DIGITS], met[kSortWaves][DIGITS];
    if ((int)blockIdx.x >= blocks) return clear(zeros, blockIdx.x - blocks, gridDim.x - blocks);
    const int wave = threadIdx.x >> 6, lane = rg_lane();
    int in_front[EACH], mine[EACH], sum = 0, all;          // a digit's entries in blocks in front of this one, and all of the digits' before it in this thread
    if constexpr (DIRECT) {
        constexpr int AHEAD = 16;
        int total[EACH];
#pragma unroll
        for (int d = 0; d < EACH; ++d) in_front[d] = total[d] = 0;
        for (int b0 = 0; b0 < blocks; b0 += AHEAD) {
            int x[AHEAD][EACH];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int d = 0; d < EACH; ++d) x[u][d] = counts[min(b0 + u, blocks - 1) * DIGITS + threadIdx.x * EACH + d];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
#pragma unroll
                for (int d = 0; d < EACH; ++d) {
                    total[d] += b0 + u < blocks ? x[u][d] : 0;
                    in_front[d] += b0 + u < (int)blockIdx.x ? x[u][d] : 0;
                }
        }
#pragma unroll
        for (int d = 0; d < EACH; ++d) {
            mine[d] = sum;
            sum += total[d];
        }
    } else {
#pragma unroll
        for (int d = 0; d < EACH; ++d) {
            mine[d] = sum;
            sum += totals[threadIdx.x * EACH + d];
            in_front[d] = counts[(int64_t)(threadIdx.x * EACH + d) * blocks + blockIdx.x];
        }
    }
    const int base = rg_block_excl_scan<kSortWaves>(sum, smem, &all);
#pragma unroll
    for (int d = 0; d < EACH; ++d) next[threadIdx.x * EACH + d] = base + mine[d] + in_front[d];
    const int64_t first = (int64_t)blockIdx.x * per_block, last = rg_least(first + per_block, rg_rows(n, n_dev));
    for (int64_t tile = first; tile < last; tile += kTile) {
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w)
#pragma unroll
            for (int d = 0; d < EACH; ++d) met[w][threadIdx.x + d * kThreads] = 0;
        __syncthreads();
        Entry e[kRounds];
        int rank[kRounds];
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int64_t i = tile + wave * (kRounds * RG_WAVE) + r * RG_WAVE + lane;
            e[r] = i < last ? entry_of(from, ids, i, num_rows) : Entry{0, 0};
        }
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int64_t i = tile + wave * (kRounds * RG_WAVE) + r * RG_WAVE + lane;
            const uint32_t digit = e[r].id >> shift & (DIGITS - 1);
            const uint64_t same = same_digit<BITS>(digit, i < last);
            const int below = __popcll(same & ((1ull << lane) - 1));
            const int so_far = met[wave][digit];
            wave_exchange();
            if (i < last && below == 0) met[wave][digit] = so_far + __popcll(same);
            wave_exchange();
            rank[r] = so_far + below;
        }
        __syncthreads();
#pragma unroll
        for (int d = 0; d < EACH; ++d) {
            int at = next[threadIdx.x + d * kThreads];
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                const int here = met[w][threadIdx.x + d * kThreads];
                met[w][threadIdx.x + d * kThreads] = at;
                at += here;
            }
            next[threadIdx.x + d * kThreads] = at;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
            const int64_t i = tile + wave * (kRounds * RG_WAVE) + r * RG_WAVE + lane;
            if (i < last) to[met[wave][e[r].id >> shift & (DIGITS - 1)] + rank[r]] = e[r];
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- sums by id
// The sorted entries are cut into pieces of `size`.  An id is met for the first time in a piece where its first entry lies.
__device__ __forceinline__ bool opens(const Entry* sorted, int64_t i) { return i == 0 || sorted[i - 1].id != sorted[i].id; }

// Ids that open in a piece, a wavefront to a piece: where its rows of the list begin.  5 us of 794 k entries.
__global__ void __launch_bounds__(kThreads) k_count_ids(const Entry* __restrict__ sorted, int64_t n, const int32_t* __restrict__ n_dev, uint32_t num_rows,
                                                        int64_t size, int pieces, int32_t* __restrict__ before) {
    const int64_t n_act = rg_rows(n, n_dev);
    const int piece = blockIdx.x * (kThreads / RG_WAVE) + (threadIdx.x >> 6);
    if (piece >= pieces) return;
    const int64_t first = piece * size, last = rg_least(first + size, n_act);
    int count = 0;
    for (int64_t i0 = first; i0 < last; i0 += RG_WAVE) {
        const int64_t i = i0 + rg_lane();
        count += __popcll(__ballot(i < last && sorted[i].id < num_rows && opens(sorted, i)));
    }
    if (rg_lane() == 0) before[piece] = count;
}

// before[piece] = ids met in front of it, before[pieces] and *num_touched = all.  One workgroup, four counts to a thread: 6 us of 8192 pieces (of 16384 10, with 16 counts to a thread 16).
__global__ void __launch_bounds__(1024) k_scan_ids(int32_t* __restrict__ before, int pieces, int32_t* __restrict__ num_touched) {
    __shared__ int smem[17];
    constexpr int EACH = 4;
    int so_far = 0;
    for (int p0 = 0; p0 < pieces; p0 += 1024 * EACH) {
        const int p = p0 + threadIdx.x * EACH;
        int x[EACH], sum = 0, total;
#pragma unroll
        for (int i = 0; i < EACH; ++i) x[i] = before[min(p + i, pieces)];        // (without branches, which the loads would wait for one by one)
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            x[i] = p + i < pieces ? x[i] : 0;
            sum += x[i];
        }
        int at = so_far + rg_block_excl_scan<16>(sum, smem, &total);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (p + i < pieces) before[p + i] = at;
            at += x[i];
        }
        so_far += total;
    }
    if (threadIdx.x == 0) {
        before[pieces] = so_far;
        *num_touched = so_far;
    }
}

// Where sums go: the table's rows (LIST false), or a row for each id met.
template <typename U>
struct Target {
    U* grad;
    int64_t stride;
    int32_t* touched;          // or NULL
    const int32_t* before;
    float scale;
    int add;
};

template <int V, typename U>
__device__ __forceinline__ void put_sum(const Target<U>& t, int64_t row, int col, int dim, float (&v)[V]) {
    U* to = t.grad + row * t.stride + col;
#pragma unroll
    for (int j = 0; j < V; ++j) v[j] *= t.scale;
    if (t.add) {
        float old[V];
        rg_load_head<V>(to, dim - col, old);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] += old[j];
    }
    rg_store_live<V>(to, dim - col, v);
}

// A group of 2^log2L lanes walks a piece, a chunk of V columns to a lane (blockIdx.y: which 2^log2L chunks), kWalk rows on their way at a time, and adds up in 32 bits.
// The sums of an id that opens and ends in the piece are final; what belongs to an id that opened before goes to parts[piece][0], to one that goes on
// behind to parts[piece][1], for k_join_pieces.  V is what fills 16 bytes of the wider type.  Bound by memory: 794 k rows of 256 bf16, all ids different, into f32 rows 264-270 us,
// 4.5 TB/s read and written (5.4 would be the lookup's; with stores past the caches 315 instead of 290); 1.5 M rows of 100 f32 into 47 129 us, 4.65 TB/s of rows that
// begin and end inside lines of 128 bytes, which a neighbour's walk fetches again.
constexpr int kWalk = 8;

template <typename T, typename U, int V, bool SHORT>
__global__ void __launch_bounds__(kThreads) k_sum_pieces(const T* __restrict__ dy, int64_t dy_stride, const Entry* __restrict__ sorted, int64_t n,
                                                         const int32_t* __restrict__ n_dev, uint32_t num_rows, int dim, int64_t size, int pieces, int log2L,
                                                         Target<U> t, float* __restrict__ parts) {
    const int64_t n_act = rg_rows(n, n_dev);
    const int piece = (int)(((int64_t)blockIdx.x * kThreads + threadIdx.x) >> log2L), l = threadIdx.x & ((1 << log2L) - 1);
    const int col = ((blockIdx.y << log2L) + l) * V;
    const int64_t first = piece * size, last = rg_least(first + size, n_act);
    if (piece >= pieces || first >= last || col >= dim) return;
    uint32_t id = sorted[first].id;
    bool open = first > 0 && sorted[first - 1].id == id;   // the first id's sums are not whole
    int64_t row = t.touched ? (int64_t)t.before[piece] - (open ? 1 : 0) : id;
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = 0.0f;
    float* part = parts + (int64_t)piece * 2 * dim + col;
    if (t.touched && !open && id < num_rows && col == 0) t.touched[row] = (int32_t)id;
    Entry e[kWalk], ahead[kWalk];
#pragma unroll
    for (int u = 0; u < kWalk; ++u) ahead[u] = sorted[rg_least(first + u, last - 1)];
    for (int64_t i = first; i < last && id < num_rows; i += kWalk) {
        typename RgPack<T, V>::type a[kWalk];
#pragma unroll
        for (int u = 0; u < kWalk; ++u) {
            e[u] = ahead[u];
            ahead[u] = sorted[rg_least(i + kWalk + u, last - 1)];
        }
#pragma unroll
        for (int u = 0; u < kWalk; ++u) a[u] = load_chunk<V, SHORT>(dy + (int64_t)e[u].at * dy_stride, col, dim);
#pragma unroll
        for (int u = 0; u < kWalk; ++u) {
            if (i + u >= last || id >= num_rows) break;
            if (e[u].id != id) {
                if (open) rg_store_live<V>(part, dim - col, sum);
                else put_sum<V>(t, row, col, dim, sum);
                open = false;
                id = e[u].id;
                if (id >= num_rows) break;
                row = t.touched ? row + 1 : id;
                if (t.touched && col == 0) t.touched[row] = (int32_t)id;
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] = 0.0f;
            }
            float v[V];
            chunk_numbers<V, SHORT>(a[u], col, dim, v);
#pragma unroll
            for (int j = 0; j < V; ++j) sum[j] += v[j];
        }
    }
    if (id >= num_rows) return;
    if (open) rg_store_live<V>(part, dim - col, sum);
    else if (last < n_act && sorted[last].id == id) rg_store_live<V>(part + dim, dim - col, sum);
    else put_sum<V>(t, row, col, dim, sum);
}

// The sums of ids whose entries lie in several pieces: a workgroup for the piece in which one of them opens (nothing to do for most), groups of 2^log2L lanes
// with 4 columns each (blockIdx.y: which 2^log2L) side by side on runs of its pieces.  Most workgroups only look; those that join wait for a few reads one behind the
// other: 8 us of 65 k entries (12 where the last piece was looked for by halving), 5 of 794 k ids met once, 12.5 of 1.5 M entries of 47 ids.  There, ids join hundreds
// of pieces each, and eight lanes a group (32 groups to a workgroup, more workgroups to an id) take 12.5 instead of the 20 of 32 lanes; on the 65 k entries it
// is 21 instead of 8, so that the host takes them where few ids have all entries.  Workgroups of 1024 threads: 42 to 57.
constexpr int kJoinThreads = 256, kJoinPieces = 2;

template <typename U, bool SHORT>
__global__ void __launch_bounds__(kJoinThreads) k_join_pieces(const Entry* __restrict__ sorted, int64_t n, const int32_t* __restrict__ n_dev, uint32_t num_rows, int dim,
                                                              int64_t size, int pieces, int log2L, Target<U> t, const float* __restrict__ parts) {
    constexpr int V = 4;
    __shared__ float sums[kJoinThreads][V];
    const int64_t n_act = rg_rows(n, n_dev);
    const int l = threadIdx.x & ((1 << log2L) - 1), run = threadIdx.x >> log2L, runs = kJoinThreads >> log2L, col = ((blockIdx.y << log2L) + l) * V;
    // (every wavefront looks at the workgroup's kJoinPieces pieces, a lane each)
    const int looked = blockIdx.x * kJoinPieces + (rg_lane() & (kJoinPieces - 1));
    const int64_t begins = looked * size, ends = begins + size, past = n_act > 0 ? n_act - 1 : 0;
    const uint32_t id_behind = sorted[rg_least(ends, past)].id, id_last = sorted[rg_least(ends - 1, past)].id, id_first = sorted[rg_least(begins, past)].id,
                   id_before = sorted[rg_least(begins > 0 ? begins - 1 : 0, past)].id;
    const bool open = looked + 1 < pieces && ends < n_act && id_behind < num_rows && id_last == id_behind && (id_first != id_behind || begins == 0 || id_before != id_first);
    for (uint32_t left = (uint32_t)__ballot(open) & ((1u << kJoinPieces) - 1); left; left &= left - 1) {
        const int piece = blockIdx.x * kJoinPieces + __builtin_ctz(left);
        const int64_t next = (piece + 1) * size;
        const uint32_t id = sorted[next].id;
        // pieces behind this one that begin with the id: those in front of the first entry of a larger one, which is looked for at 64 places at a time
        int64_t lo = next, hi = n_act;                     // (sorted[lo].id == id; larger from hi on)
        while (hi - lo > 1) {
            const int64_t step = (hi - lo + RG_WAVE) / (RG_WAVE + 1), probe = lo + (rg_lane() + 1) * step;
            const int same = __popcll(__ballot(sorted[rg_least(probe, hi - 1)].id == id && probe < hi));
            hi = rg_least(hi, lo + (same + 1) * step);
            lo += same * step;
        }
        const int from = piece + 1, to = (int)(lo / size) + 1, per = (to - from + runs - 1) / runs;
        const int start = from + run * per, stop = min(start + per, to);
        float sum[V] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (col < dim) {
            constexpr int AHEAD = 8;
            for (int p0 = start; p0 < stop; p0 += AHEAD) {
                typename RgPack<float, V>::type a[AHEAD];
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) a[u] = load_chunk<V, SHORT>(parts + (int64_t)min(p0 + u, stop - 1) * 2 * dim, col, dim);
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) {
                    if (p0 + u >= stop) break;
                    float v[V];
                    chunk_numbers<V, SHORT>(a[u], col, dim, v);
#pragma unroll
                    for (int j = 0; j < V; ++j) sum[j] += v[j];
                }
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) sums[threadIdx.x][j] = sum[j];
        __syncthreads();
        if (run == 0 && col < dim) {
            rg_load_head<V>(parts + ((int64_t)piece * 2 + 1) * dim + col, dim - col, sum);
            for (int r = 0; r < min(runs, to - from); ++r)
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] += sums[(r << log2L) + l][j];
            put_sum<V>(t, t.touched ? (int64_t)t.before[piece + 1] - 1 : id, col, dim, sum);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- few entries
// One workgroup sorts them in LDS and lists the ids met: order[] the entries' rows of dy, run r the entries starts[r] .. starts[r + 1] - 1, of id touched[r].
// Up to 2048 entries take two launches so, instead of six or more: 256 of 64 numbers 7.2 + 3.2 us.  Both sides of the line, 2048 and 2049 entries: of 64 numbers into the rows
// met of 1000 11.5 and 29 us, of 128 into 200000 14 and 34.  (More do not fit one workgroup's registers and LDS as they are.)
constexpr int kFew = 2048, kFewThreads = 1024, kFewWaves = kFewThreads / RG_WAVE, kFewRounds = kFew / kFewThreads;

__global__ void __launch_bounds__(kFewThreads) k_sort_few(const Zeros zeros, const int32_t* __restrict__ ids, int n, const int32_t* __restrict__ n_dev, uint32_t num_rows, int bits,
                                                          int32_t* __restrict__ order, int32_t* __restrict__ starts, int32_t* __restrict__ touched,
                                                          int32_t* __restrict__ num_touched, int32_t* __restrict__ count) {
    constexpr int BITS = 8, DIGITS = 1 << BITS;
    __shared__ int smem[kFewWaves + 1];
    __shared__ int32_t met[kFewWaves][DIGITS];
    __shared__ Entry list[kFew];
    if (blockIdx.x) return clear(zeros, blockIdx.x - 1, gridDim.x - 1);
    const int n_act = (int)rg_rows(n, n_dev), wave = threadIdx.x >> 6, lane = rg_lane();
    Entry e[kFewRounds];
#pragma unroll
    for (int r = 0; r < kFewRounds; ++r) {
        const int i = (wave * kFewRounds + r) * RG_WAVE + lane;
        const uint32_t id = i < n_act ? (uint32_t)ids[i] : num_rows;
        e[r] = {id < num_rows ? id : num_rows, (uint32_t)i};
    }
    for (int shift = 0; shift < bits; shift += BITS) {
        int rank[kFewRounds];
        for (int i = threadIdx.x; i < kFewWaves * DIGITS; i += kFewThreads) met[i / DIGITS][i % DIGITS] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kFewRounds; ++r) {             // (places behind the last entry sort as padding and stay behind all others)
            const uint32_t digit = e[r].id >> shift & (DIGITS - 1);
            const uint64_t same = same_digit<BITS>(digit, true);
            const int below = __popcll(same & ((1ull << lane) - 1));
            const int so_far = met[wave][digit];
            wave_exchange();
            if (below == 0) met[wave][digit] = so_far + __popcll(same);
            wave_exchange();
            rank[r] = so_far + below;
        }
        __syncthreads();
        int here[kFewWaves], sum = 0, all;
        if (threadIdx.x < DIGITS) {
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) {
                here[w] = sum;
                sum += met[w][threadIdx.x];
            }
        }
        const int base = rg_block_excl_scan<kFewWaves>(sum, smem, &all);
        if (threadIdx.x < DIGITS) {
#pragma unroll
            for (int w = 0; w < kFewWaves; ++w) met[w][threadIdx.x] = base + here[w];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kFewRounds; ++r) list[met[wave][e[r].id >> shift & (DIGITS - 1)] + rank[r]] = e[r];
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kFewRounds; ++r) e[r] = list[(wave * kFewRounds + r) * RG_WAVE + lane];
    }
    int heads = 0, total;
    bool head[kFewRounds];
#pragma unroll
    for (int r = 0; r < kFewRounds; ++r) {
        const int i = threadIdx.x * kFewRounds + r;
        head[r] = list[i].id < num_rows && (i == 0 || list[i - 1].id != list[i].id);
        heads += head[r];
    }
    int run = rg_block_excl_scan<kFewWaves>(heads, smem, &total);
#pragma unroll
    for (int r = 0; r < kFewRounds; ++r) {
        const int i = threadIdx.x * kFewRounds + r;
        if (list[i].id < num_rows) order[i] = (int32_t)list[i].at;
        else if (i > 0 && list[i - 1].id < num_rows) starts[total] = i;         // the entries' end
        if (head[r]) {
            starts[run] = i;
            touched[run++] = (int32_t)list[i].id;
        }
    }
    if (threadIdx.x == 0) {
        if (list[kFew - 1].id < num_rows) starts[total] = kFew;
        *count = total;
        if (num_touched) *num_touched = total;
    }
}

// A workgroup to a run and 2^log2L chunks of V columns (blockIdx.y), its groups of lanes side by side on the run's entries, added up in their order.
template <typename T, typename U, int V, bool SHORT>
__global__ void __launch_bounds__(kThreads) k_sum_runs(const T* __restrict__ dy, int64_t dy_stride, const int32_t* __restrict__ order, const int32_t* __restrict__ starts,
                                                       const int32_t* __restrict__ touched, const int32_t* __restrict__ count, int dim, int log2L, int rows,
                                                       Target<U> t) {
    __shared__ float sums[kThreads][V];
    const int run = blockIdx.x;
    if (run >= *count) return;
    const int l = threadIdx.x & ((1 << log2L) - 1), group = threadIdx.x >> log2L, groups = kThreads >> log2L, col = ((blockIdx.y << log2L) + l) * V;
    const int first = starts[run], last = starts[run + 1];
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = 0.0f;
    if (col < dim) {
        for (int i = first + group; i < last; i += groups * kWalk) {
            typename RgPack<T, V>::type a[kWalk];
#pragma unroll
            for (int u = 0; u < kWalk; ++u) a[u] = load_chunk<V, SHORT>(dy + (int64_t)order[min(i + u * groups, last - 1)] * dy_stride, col, dim);
#pragma unroll
            for (int u = 0; u < kWalk; ++u) {
                if (i + u * groups >= last) break;
                float v[V];
                chunk_numbers<V, SHORT>(a[u], col, dim, v);
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] += v[j];
            }
        }
    }
    if (last - first > 1) {
#pragma unroll
        for (int j = 0; j < V; ++j) sums[threadIdx.x][j] = sum[j];
        __syncthreads();
        if (group == 0)
            for (int r = 1; r < min(groups, last - first); ++r)
#pragma unroll
                for (int j = 0; j < V; ++j) sum[j] += sums[(r << log2L) + l][j];
    }
    if (group == 0 && col < dim) put_sum<V>(t, rows ? touched[run] : run, col, dim, sum);
}

bool aligned(const void* p, int bytes) { return (uintptr_t)p % (uintptr_t)bytes == 0; }

constexpr int64_t kMostRows = (1ll << 31) - 1;

template <typename U>
Zeros zeros_of(U* grad, int64_t stride, int64_t num_rows, int dim) {
    const int chunks = (int)rg_div_up(dim, 16 / (int)sizeof(U));
    return {grad, stride, 0, num_rows * chunks, dim, chunks, (int)sizeof(U), rg_store_once(grad, (int64_t)dim * sizeof(U), stride * (int64_t)sizeof(U), num_rows)};
}

// Workgroups of `threads` for pieces of zeros.
int clear_blocks(rg_ctx* ctx, int64_t pieces, int threads) { return (int)rg_min64(rg_div_up(pieces, threads * 4), (int64_t)ctx->num_cus * (8192 / threads)); }

// The gradient's two forms: a whole table (touched NULL), or the rows met.
template <typename U>
rg_status sum_by_id(rg_ctx* ctx, const char* who, const void* dy, rg_dtype dy_type, int64_t dy_stride, const int32_t* ids, int64_t n, const int32_t* n_dev,
                    int dim, int64_t num_rows, float scale, U* grad, int64_t grad_stride, int add, int32_t* touched, int32_t* num_touched, hipStream_t s) {
    Zeros zeros = {};
    if (!touched && !add) zeros = zeros_of(grad, grad_stride, num_rows, dim);
    if (!touched && n == 0) {
        k_clear_rows<<<(unsigned)clear_blocks(ctx, zeros.to, kThreads), kThreads, 0, s>>>(zeros);
        RG_LAUNCH_CHECK(ctx, "k_clear_rows");
        return RG_OK;
    }
    int bits = 1;
    while (bits < 31 && num_rows >> bits) ++bits;          // ids 0 .. num_rows, padding the last
    if (n <= kFew) {
        const rg_status st = rg_scratch(ctx, ctx->embed_parts, (3 * kFew + 64) * 4, s, who);
        if (st != RG_OK) return st;
        int32_t* order = (int32_t*)ctx->embed_parts.p;
        int32_t *starts = order + kFew, *named = starts + kFew + 32, *count = named + kFew;
        k_sort_few<<<1 + clear_blocks(ctx, zeros.to, kFewThreads), kFewThreads, 0, s>>>(zeros, ids, (int)n, n_dev, (uint32_t)num_rows, bits, order, starts, touched ? touched : named, num_touched, count);
        RG_LAUNCH_CHECK(ctx, "k_sort_few");
        const Target<U> t = {grad, grad_stride, nullptr, nullptr, scale, add};
        RG_FOR_TYPE(dy_type, {
            constexpr int V = 16 / (int)(sizeof(T) > sizeof(U) ? sizeof(T) : sizeof(U));
            const int chunks = (int)rg_div_up(dim, V);
            int log2L = 0;
            while (log2L < 6 && 1 << log2L < chunks) ++log2L;
            const dim3 grid((unsigned)rg_min64(n, num_rows), (unsigned)rg_div_up(chunks, 1 << log2L));
            const auto kernel = dim < V ? k_sum_runs<T, U, V, true> : k_sum_runs<T, U, V, false>;
            kernel<<<grid, kThreads, 0, s>>>((const T*)dy, dy_stride, order, starts, touched ? touched : named, count, dim, log2L, touched ? 0 : 1, t);
        });
        RG_LAUNCH_CHECK(ctx, "k_sum_runs");
        return RG_OK;
    }
    // pieces of 16 entries or more, and as many of them as fill the device: of 1 M f32 rows of 32 / 128 numbers into the rows met of 100000, 4096 pieces take 146 / 207 us, 8192
    // 124 / 217, 16384 135 / 236.  Where few ids have all entries, each of them is joined from hundreds of pieces, and half as many pieces with narrower groups at the join
    // take less: f32, at 1024 / 16384 / 100 k entries an id, 1.5 M rows of 100 210 / 167 / 163 us so and 206 / 176 / 178 otherwise, 1 M of 256 266 / 231 / 227 and 245 / 230 / 244,
    // 300 k of 100 54 / 47 / 49 and 51 / 50 / 73; bf16, 1.5 M of 100 167 / 129 / 126 and 148 / 122 / 123, 300 k of 100 49 / 43 / 47 and 43 / 44 / 67.  (Of up to 32 columns
    // the groups are narrow anyway: 1 M of 32 91 / 75 / 73 and 70 / 55 / 54.)
    const bool dense = dim > 32 && n / rg_max64(num_rows, 1) >= 16384;
    const int most = (int)rg_max64(1024, rg_min64(dense ? 4096 : 8192, (1ll << 23) / dim));
    const int64_t size = rg_max64(16, rg_div_up(n, most));
    const int pieces = (int)rg_div_up(n, size);
    const int passes = (bits + 9) / 10, digit = (int)rg_max64(8, rg_div_up(bits, passes));
    const int64_t per_block = kTile * rg_max64(1, rg_div_up(n, (int64_t)kTile * 4096));
    const int blocks = (int)rg_div_up(n, per_block);
    // scratch: two lists of entries, counts, totals, ids in front of the pieces, sums of parts
    const size_t list = (size_t)rg_div_up(n * (int64_t)sizeof(Entry), 256) * 256;
    const size_t counts_bytes = (size_t)rg_div_up(((int64_t)(blocks + 1) << digit) * 4, 256) * 256, before_bytes = (size_t)rg_div_up((pieces + 1) * 4ll, 256) * 256;
    const rg_status st = rg_scratch(ctx, ctx->embed_parts, 2 * list + counts_bytes + before_bytes + (size_t)pieces * 2 * dim * 4, s, who);
    if (st != RG_OK) return st;
    char* at = (char*)ctx->embed_parts.p;
    Entry* lists[2] = {(Entry*)at, (Entry*)(at + list)};
    int32_t* counts = (int32_t*)(at + 2 * list);
    int32_t* totals = counts + ((int64_t)blocks << digit);
    int32_t* before = (int32_t*)(at + 2 * list + counts_bytes);
    float* parts = (float*)(at + 2 * list + counts_bytes + before_bytes);
    const int64_t all_zeros = zeros.to;
    const int total_launches = (blocks <= kDirectBlocks ? 2 : 3) * passes;
    int launches = 0;
    const auto part_of_zeros = [&] {                       // a launch's share of the pieces
        zeros.from = all_zeros * launches / total_launches;
        zeros.to = all_zeros * ++launches / total_launches;
        return clear_blocks(ctx, zeros.to - zeros.from, kThreads);
    };
    const Entry* from = nullptr;
    const auto sort = [&](auto width, auto direct) {
        constexpr int BITS = decltype(width)::value;
        constexpr bool DIRECT = decltype(direct)::value;
        for (int pass = 0; pass < passes; ++pass) {
            Entry* to = lists[pass & 1];
            int more = part_of_zeros();
            k_sort_count<BITS, DIRECT><<<blocks + more, kThreads, 0, s>>>(zeros, blocks, from, ids, n, n_dev, (uint32_t)num_rows, pass * BITS, per_block, counts);
            if (!DIRECT) {
                more = part_of_zeros();
                k_sort_scan<<<(1 << BITS) + more, kThreads, 0, s>>>(zeros, 1 << BITS, counts, blocks, totals);
            }
            more = part_of_zeros();
            k_sort_scatter<BITS, DIRECT><<<blocks + more, kThreads, 0, s>>>(zeros, blocks, from, ids, n, n_dev, (uint32_t)num_rows, pass * BITS, per_block, counts, totals,
                                                                            to);
            from = to;
        }
    };
    const auto sort_by = [&](auto width) { blocks <= kDirectBlocks ? sort(width, std::true_type()) : sort(width, std::false_type()); };
    if (digit == 8) sort_by(std::integral_constant<int, 8>());
    else if (digit == 9) sort_by(std::integral_constant<int, 9>());
    else sort_by(std::integral_constant<int, 10>());
    RG_LAUNCH_CHECK(ctx, "k_sort_scatter");
    if (touched) {
        k_count_ids<<<(unsigned)rg_div_up(pieces, kThreads / RG_WAVE), kThreads, 0, s>>>(from, n, n_dev, (uint32_t)num_rows, size, pieces, before);
        k_scan_ids<<<1, 1024, 0, s>>>(before, pieces, num_touched);
        RG_LAUNCH_CHECK(ctx, "k_scan_ids");
    }
    const Target<U> t = {grad, grad_stride, touched, before, scale, add};
    RG_FOR_TYPE(dy_type, {
        constexpr int V = 16 / (int)(sizeof(T) > sizeof(U) ? sizeof(T) : sizeof(U));
        const int chunks = (int)rg_div_up(dim, V);
        int log2L = 0;
        while (log2L < 6 && 1 << log2L < chunks) ++log2L;
        const dim3 grid((unsigned)rg_div_up((int64_t)pieces << log2L, kThreads), (unsigned)rg_div_up(chunks, 1 << log2L));
        const auto kernel = dim < V ? k_sum_pieces<T, U, V, true> : k_sum_pieces<T, U, V, false>;
        kernel<<<grid, kThreads, 0, s>>>((const T*)dy, dy_stride, from, n, n_dev, (uint32_t)num_rows, dim, size, pieces, log2L, t, parts);
    });
    RG_LAUNCH_CHECK(ctx, "k_sum_pieces");
    if (pieces > 1) {
        const int fours = (int)rg_div_up(dim, 4);
        int log2L = 0;
        while (log2L < (dense ? 3 : 6) && 1 << log2L < fours) ++log2L;
        const auto kernel = dim < 4 ? k_join_pieces<U, true> : k_join_pieces<U, false>;
        kernel<<<dim3((unsigned)rg_div_up(pieces, kJoinPieces), (unsigned)rg_div_up(fours, 1 << log2L)), kJoinThreads, 0, s>>>(
            from, n, n_dev, (uint32_t)num_rows, dim, size, pieces, log2L, t, parts);
        RG_LAUNCH_CHECK(ctx, "k_join_pieces");
    }
    return RG_OK;
}

rg_status check_grad(rg_ctx* ctx, const char* who, const void* dy, rg_dtype dy_type, int64_t dy_stride, const int32_t* ids, int64_t n, int32_t dim,
                     int64_t num_rows, float scale) {
    RG_REQUIRE(ctx, n >= 0 && n <= kMostRows, "%s: n = %lld out of range", who, (long long)n);
    RG_REQUIRE(ctx, dim >= 1 && dim <= RG_EMBED_MAX_DIM, "%s: dim = %d not in [1,%d]", who, dim, RG_EMBED_MAX_DIM);
    RG_REQUIRE(ctx, num_rows >= 0 && num_rows <= kMostRows, "%s: num_rows = %lld out of range", who, (long long)num_rows);
    RG_REQUIRE(ctx, rg_type_known(dy_type), "%s: unknown type %d", who, (int)dy_type);
    RG_REQUIRE(ctx, dy_stride >= dim, "%s: bad stride", who);
    RG_REQUIRE(ctx, scale == scale, "%s: scale is not a number", who);
    RG_REQUIRE(ctx, n == 0 || (dy && ids), "%s: null pointer", who);
    RG_REQUIRE(ctx, aligned(dy, rg_type_bytes(dy_type)) && aligned(ids, 4), "%s: pointer not aligned to its numbers", who);
    return RG_OK;
}

__global__ void k_no_ids(int32_t* num_touched) { *num_touched = 0; }

}  // namespace

extern "C" {

rg_status rg_embedding(rg_ctx* ctx, const void* table, rg_dtype table_type, int64_t table_stride, int64_t num_rows, const int32_t* ids, int64_t n,
                       const int32_t* n_dev, int32_t dim, float scale, void* y, rg_dtype y_type, int64_t y_stride, void* stream) {
    if (!ctx) return RG_ERR_INVALID_ARG;
    RG_REQUIRE(ctx, n >= 0 && n <= kMostRows, "rg_embedding: n = %lld out of range", (long long)n);
    RG_REQUIRE(ctx, dim >= 1 && dim <= RG_EMBED_MAX_DIM, "rg_embedding: dim = %d not in [1,%d]", dim, RG_EMBED_MAX_DIM);
    RG_REQUIRE(ctx, num_rows >= 1 && num_rows <= kMostRows, "rg_embedding: num_rows = %lld out of range", (long long)num_rows);
    RG_REQUIRE(ctx, rg_type_known(table_type) && rg_type_known(y_type), "rg_embedding: unknown type");
    RG_REQUIRE(ctx, table_stride >= dim && y_stride >= dim, "rg_embedding: bad stride");
    RG_REQUIRE(ctx, scale == scale, "rg_embedding: scale is not a number");
    if (n == 0) return RG_OK;
    RG_REQUIRE(ctx, table && ids && y, "rg_embedding: null pointer");
    RG_REQUIRE(ctx, y != table && y != (const void*)ids, "rg_embedding: y is an input");
    RG_REQUIRE(ctx, aligned(table, rg_type_bytes(table_type)) && aligned(ids, 4) && aligned(y, rg_type_bytes(y_type)),
               "rg_embedding: pointer not aligned to its numbers");
    RG_HIP(ctx, hipSetDevice(ctx->device));
    hipStream_t s = (hipStream_t)stream;
    const bool once = rg_store_once(y, (int64_t)dim * rg_type_bytes(y_type), y_stride * rg_type_bytes(y_type), n);
    const auto launch = [&](auto t, auto u) {
        typedef decltype(t) T;
        typedef decltype(u) U;
        constexpr int V = 16 / (int)(sizeof(T) < sizeof(U) ? sizeof(T) : sizeof(U));
        const int chunks = (int)rg_div_up(dim, V), group = (int)rg_max64(1, kThreads * kAhead / chunks);
        const auto kernel = dim < V ? k_embedding<T, U, V, true, false> : once ? k_embedding<T, U, V, false, true> : k_embedding<T, U, V, false, false>;
        kernel<<<(unsigned)rg_min64(rg_div_up(n, group), 1 << 22), kThreads, 0, s>>>((const T*)table, table_stride, (int)num_rows, ids, n, n_dev, dim, chunks,
                                                                                     rg_inverse((uint32_t)chunks), group, scale, (U*)y, y_stride);
    };
    RG_FOR_TYPE(table_type, {
        const T t = {};
        if (y_type == RG_F32) launch(t, float());
        else if (y_type == RG_BF16) launch(t, __bf16());
        else launch(t, _Float16());
    });
    RG_LAUNCH_CHECK(ctx, "k_embedding");
    return RG_OK;
}

rg_status rg_embedding_grad(rg_ctx* ctx, const void* dy, rg_dtype dy_type, int64_t dy_stride, const int32_t* ids, int64_t n, const int32_t* n_dev,
                            int32_t dim, int64_t num_rows, float scale, int add, void* grad, rg_dtype grad_type, int64_t grad_stride, void* stream) {
    if (!ctx) return RG_ERR_INVALID_ARG;
    const rg_status bad = check_grad(ctx, "rg_embedding_grad", dy, dy_type, dy_stride, ids, n, dim, num_rows, scale);
    if (bad != RG_OK) return bad;
    RG_REQUIRE(ctx, rg_type_known(grad_type), "rg_embedding_grad: unknown type %d", (int)grad_type);
    RG_REQUIRE(ctx, grad_stride >= dim, "rg_embedding_grad: bad stride");
    if (num_rows == 0 || (add && n == 0)) return RG_OK;
    RG_REQUIRE(ctx, grad, "rg_embedding_grad: null pointer");
    RG_REQUIRE(ctx, n == 0 || (grad != dy && grad != (const void*)ids), "rg_embedding_grad: grad is an input");
    RG_REQUIRE(ctx, aligned(grad, rg_type_bytes(grad_type)), "rg_embedding_grad: pointer not aligned to its numbers");
    RG_HIP(ctx, hipSetDevice(ctx->device));
    hipStream_t s = (hipStream_t)stream;
    const auto sums = [&](auto u) {
        typedef decltype(u) U;
        return sum_by_id<U>(ctx, "rg_embedding_grad", dy, dy_type, dy_stride, ids, n, n_dev, dim, num_rows, scale, (U*)grad, grad_stride, add, nullptr, nullptr, s);
    };
    const rg_status st = grad_type == RG_F32 ? sums(float()) : grad_type == RG_BF16 ? sums(__bf16()) : sums(_Float16());
    return st;
}

rg_status rg_embedding_grad_rows(rg_ctx* ctx, const void* dy, rg_dtype dy_type, int64_t dy_stride, const int32_t* ids, int64_t n, const int32_t* n_dev,
                                 int32_t dim, int64_t num_rows, float scale, float* grad, int64_t grad_stride, int32_t* touched, int32_t* num_touched,
                                 void* stream) {
    if (!ctx) return RG_ERR_INVALID_ARG;
    const rg_status bad = check_grad(ctx, "rg_embedding_grad_rows", dy, dy_type, dy_stride, ids, n, dim, num_rows, scale);
    if (bad != RG_OK) return bad;
    RG_REQUIRE(ctx, grad_stride >= dim, "rg_embedding_grad_rows: bad stride");
    RG_REQUIRE(ctx, num_touched && (n == 0 || num_rows == 0 || (grad && touched)), "rg_embedding_grad_rows: null pointer");
    RG_REQUIRE(ctx, aligned(grad, 4) && aligned(touched, 4) && aligned(num_touched, 4), "rg_embedding_grad_rows: pointer not aligned to its numbers");
    RG_REQUIRE(ctx, n == 0 || num_rows == 0 || ((const void*)grad != dy && touched != ids && num_touched != touched && num_touched != ids),
               "rg_embedding_grad_rows: an output is an input, or another output");
    RG_HIP(ctx, hipSetDevice(ctx->device));
    hipStream_t s = (hipStream_t)stream;
    if (n == 0 || num_rows == 0) {
        k_no_ids<<<1, 1, 0, s>>>(num_touched);
        RG_LAUNCH_CHECK(ctx, "k_no_ids");
        return RG_OK;
    }
    return sum_by_id<float>(ctx, "rg_embedding_grad_rows", dy, dy_type, dy_stride, ids, n, n_dev, dim, num_rows, scale, grad, grad_stride, 0, touched, num_touched, s);
}

}  // extern "C"
