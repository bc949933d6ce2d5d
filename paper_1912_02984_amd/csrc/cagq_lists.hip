// The groups turned round: for each point the centers whose groups hold it,
// ascending (cagq_point_lists).
//
// A counting sort by point: count the slots of each point (integer atomics,
// whose order does not matter), scan the counts, hand every slot a place in
// its point's list, and sort each list, so that the result does not depend on
// the order in which the slots arrived.
#include "cagq_features.h"

namespace cagq {

namespace {

constexpr int kPlThreads = 256;
constexpr int kPlItems = 8;                         // points per thread of the scan
constexpr int kPlTile = kPlThreads * kPlItems;      // points per scan tile
constexpr int kPlShort = kWave;                     // longest list that one wave sorts in registers
constexpr int kPlLongThreads = 1024;
constexpr int kPlChunk = 8192;                      // entries a workgroup sorts in LDS
constexpr int kPlLongBlocks = 512;                  // workgroups for the lists above kPlShort

struct PlLayout {
    int64_t points, tiles, most_long;
    size_t count, tile, nlong, longs, total;
};

PlLayout pl_layout(const Groups& g, int32_t B) {
    PlLayout L;
    L.points = (int64_t)B * g.N;
    L.tiles = (L.points + kPlTile - 1) / kPlTile;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at = (at + bytes + 255) & ~(size_t)255;
        return here;
    };
    L.count = take((size_t)L.points * 8);
    L.tile = take((size_t)L.tiles * 8);
    L.nlong = take(4);
    // a list above kPlShort has that many slots: at most slots / (kPlShort + 1) of them
    L.most_long = g.idx_len / (kPlShort + 1);
    if (L.most_long > L.points) L.most_long = L.points;
    L.longs = take((size_t)(L.most_long + 1) * 4);
    L.total = at;
    return L;
}

__global__ __launch_bounds__(kPlThreads) void k_pl_clear(uint64_t* __restrict__ count, int64_t points,
                                                         uint32_t* __restrict__ nlong, int32_t* __restrict__ center,
                                                         int64_t capacity) {
    const int64_t step = (int64_t)gridDim.x * kPlThreads;
    const int64_t t = (int64_t)blockIdx.x * kPlThreads + threadIdx.x;
    for (int64_t i = t; i < points; i += step) count[i] = 0;
    for (int64_t i = t; i < capacity; i += step) center[i] = -1;
    if (t == 0) *nlong = 0;
}

// Calls f(point over the batch, center) for every slot that counts: a wave per
// group, its lanes over the slots.
template <typename F>
__device__ __forceinline__ void each_slot(const Groups& g, F f) {
    const int lane = lane_id();
    const int64_t waves = (int64_t)gridDim.x * (kPlThreads / kWave);
    for (int64_t row = (int64_t)blockIdx.x * (kPlThreads / kWave) + threadIdx.x / kWave; row < g.rows; row += waves) {
        int64_t beg, end;
        g.range((int32_t)row, beg, end);
        const uint32_t b = udiv((uint32_t)row, g.mm);
        const int32_t j = (int32_t)((uint32_t)row - b * (uint32_t)g.M);
        for (int64_t s = beg + lane; s < end; s += kWave) {
            const int32_t i = g.idx[s];
            if ((uint32_t)i < (uint32_t)g.N) f((int64_t)b * g.N + i, j);
        }
    }
}

__global__ __launch_bounds__(kPlThreads) void k_pl_count(Groups g, uint64_t* __restrict__ count) {
    each_slot(g, [&](int64_t i, int32_t) { atomicAdd((unsigned long long*)&count[i], 1ull); });
}

__global__ __launch_bounds__(kPlThreads) void k_pl_tiles(const uint64_t* __restrict__ count, int64_t points,
                                                         uint64_t* __restrict__ tile) {
    __shared__ uint64_t s_wave[kPlThreads / kWave];
    const int64_t i0 = (int64_t)blockIdx.x * kPlTile + (int64_t)threadIdx.x * kPlItems;
    uint64_t sum = 0;
    for (int k = 0; k < kPlItems; ++k)
        if (i0 + k < points) sum += count[i0 + k];
    uint64_t total;
    block_excl_scan(sum, s_wave, &total);
    if (threadIdx.x == 0) tile[blockIdx.x] = total;
}

// Exclusive prefix of the tiles' totals, by one workgroup.
__global__ __launch_bounds__(kPlThreads) void k_pl_scan(uint64_t* __restrict__ tile, int64_t tiles) {
    __shared__ uint64_t s_wave[kPlThreads / kWave];
    uint64_t run = 0;
    for (int64_t t0 = 0; t0 < tiles; t0 += kPlThreads) {
        const int64_t t = t0 + threadIdx.x;
        const uint64_t v = t < tiles ? tile[t] : 0;
        uint64_t total;
        const uint64_t excl = block_excl_scan(v, s_wave, &total);
        if (t < tiles) tile[t] = run + excl;
        run += total;
        __syncthreads();
    }
}

// Offsets, and each point's first free place in `count`.
__global__ __launch_bounds__(kPlThreads) void k_pl_offsets(uint64_t* __restrict__ count, int64_t points,
                                                           const uint64_t* __restrict__ tile,
                                                           int64_t* __restrict__ off, uint32_t* __restrict__ nlong,
                                                           uint32_t* __restrict__ longs, int64_t most_long) {
    __shared__ uint64_t s_wave[kPlThreads / kWave];
    const int64_t i0 = (int64_t)blockIdx.x * kPlTile + (int64_t)threadIdx.x * kPlItems;
    uint64_t c[kPlItems], sum = 0;
#pragma unroll
    for (int k = 0; k < kPlItems; ++k) {
        c[k] = i0 + k < points ? count[i0 + k] : 0;
        sum += c[k];
    }
    uint64_t total;
    uint64_t run = tile[blockIdx.x] + block_excl_scan(sum, s_wave, &total);
#pragma unroll
    for (int k = 0; k < kPlItems; ++k) {
        if (i0 + k >= points) break;
        off[i0 + k] = (int64_t)run;
        count[i0 + k] = run;
        if (c[k] > kPlShort) {
            const uint32_t l = atomicAdd(nlong, 1u);
            if (l < most_long) longs[l] = (uint32_t)(i0 + k);
        }
        run += c[k];
        if (i0 + k == points - 1) off[points] = (int64_t)run;
    }
}

__global__ __launch_bounds__(kPlThreads) void k_pl_fill(Groups g, uint64_t* __restrict__ count,
                                                        int32_t* __restrict__ center, int64_t capacity) {
    each_slot(g, [&](int64_t i, int32_t j) {
        const int64_t at = (int64_t)atomicAdd((unsigned long long*)&count[i], 1ull);
        if (at < capacity) center[at] = j;
    });
}

// Lists of at most a wave's entries: each entry's place is the number of
// smaller ones (equal ones keep their order).
__global__ __launch_bounds__(kPlThreads) void k_pl_short(const int64_t* __restrict__ off, int64_t points,
                                                         int32_t* __restrict__ center, int64_t capacity) {
    const int lane = lane_id();
    const int64_t waves = (int64_t)gridDim.x * (kPlThreads / kWave);
    for (int64_t i = (int64_t)blockIdx.x * (kPlThreads / kWave) + threadIdx.x / kWave; i < points; i += waves) {
        const int64_t beg = off[i];
        const int64_t n = off[i + 1] - beg;
        if (n < 2 || n > kPlShort || beg + n > capacity) continue;
        const int32_t v = lane < n ? center[beg + lane] : 0;
        int rank = 0;
        for (int k = 0; k < (int)n; ++k) {
            const int32_t o = __builtin_amdgcn_readlane(v, k);
            rank += o < v || (o == v && k < lane);
        }
        if (lane < n) center[beg + rank] = v;
    }
}

// Longer lists, a workgroup each: a bitonic sort whose comparisons all put the
// smaller entry first (the first step of a merge mirrors its second half), so
// that entries past the end count as largest and need not exist. Distances
// within a chunk run in LDS, longer ones in global memory.
__global__ __launch_bounds__(kPlLongThreads) void k_pl_long(const int64_t* __restrict__ off,
                                                            const uint32_t* __restrict__ nlong,
                                                            const uint32_t* __restrict__ longs, int64_t most_long,
                                                            int32_t* __restrict__ center, int64_t capacity) {
    __shared__ int32_t s[kPlChunk];
    const uint32_t lists = *nlong < most_long ? *nlong : (uint32_t)most_long;
    for (uint32_t l = blockIdx.x; l < lists; l += gridDim.x) {
        const int64_t beg = off[longs[l]];
        const int64_t n = off[(int64_t)longs[l] + 1] - beg;
        if (beg + n > capacity) continue;
        int32_t* a = center + beg;
        // steps of a merge of 2 * k sorted pairs, from distance j down, within the chunk at c0
        auto clean = [&](int64_t c0, int64_t j) {
            for (; j > 0; j >>= 1) {
                __syncthreads();
                for (int t = threadIdx.x; t < kPlChunk / 2; t += kPlLongThreads) {
                    const int x = (int)((t / j) * 2 * j + t % j), y = x + (int)j;
                    if (c0 + y < n && s[y] < s[x]) {
                        const int32_t v = s[x];
                        s[x] = s[y];
                        s[y] = v;
                    }
                }
            }
        };
        auto load = [&](int64_t c0) {
            __syncthreads();
            for (int t = threadIdx.x; t < kPlChunk && c0 + t < n; t += kPlLongThreads) s[t] = a[c0 + t];
        };
        auto store = [&](int64_t c0) {
            __syncthreads();
            for (int t = threadIdx.x; t < kPlChunk && c0 + t < n; t += kPlLongThreads) a[c0 + t] = s[t];
        };
        for (int64_t c0 = 0; c0 < n; c0 += kPlChunk) {
            load(c0);
            for (int k = 2; k <= kPlChunk; k <<= 1) {
                if (k / 2 >= n - c0) break;  // one sorted run already
                __syncthreads();
                for (int t = threadIdx.x; t < kPlChunk / 2; t += kPlLongThreads) {
                    const int h = k / 2;
                    const int x = (t / h) * k + t % h, y = (t / h) * k + k - 1 - t % h;
                    if (c0 + y < n && s[y] < s[x]) {
                        const int32_t v = s[x];
                        s[x] = s[y];
                        s[y] = v;
                    }
                }
                clean(c0, k / 4);
            }
            store(c0);
        }
        for (int64_t k = 2 * (int64_t)kPlChunk; k / 2 < n; k <<= 1) {
            const int64_t half = k / 2;
            __threadfence_block();
            __syncthreads();
            for (int64_t t = threadIdx.x; t < n; t += kPlLongThreads) {  // t: pair number
                const int64_t x = (t / half) * k + t % half, y = (t / half) * k + k - 1 - t % half;
                if (x >= n) break;
                if (y < n && a[y] < a[x]) {
                    const int32_t v = a[x];
                    a[x] = a[y];
                    a[y] = v;
                }
            }
            for (int64_t j = half / 2; j >= kPlChunk; j >>= 1) {
                __threadfence_block();
                __syncthreads();
                for (int64_t t = threadIdx.x; t < n; t += kPlLongThreads) {
                    const int64_t x = (t / j) * 2 * j + t % j, y = x + j;
                    if (x >= n) break;
                    if (y < n && a[y] < a[x]) {
                        const int32_t v = a[x];
                        a[x] = a[y];
                        a[y] = v;
                    }
                }
            }
            __threadfence_block();
            for (int64_t c0 = 0; c0 < n; c0 += kPlChunk) {
                load(c0);
                clean(c0, kPlChunk / 2);
                store(c0);
            }
        }
        __syncthreads();
    }
}

int blocks_for(int64_t items, int64_t per_block, int most) {
    const int64_t n = (items + per_block - 1) / per_block;
    return (int)(n < 1 ? 1 : n > most ? most : n);
}

}  // namespace

size_t point_lists_bytes(const Groups& g, int32_t B) { return pl_layout(g, B).total; }

hipError_t launch_point_lists(const Groups& g, int32_t B, int64_t* pt_off, int32_t* pt_center, int64_t capacity,
                              void* ws, hipStream_t s) {
    const PlLayout L = pl_layout(g, B);
    uint64_t* count = at<uint64_t>(ws, L.count);
    uint64_t* tile = at<uint64_t>(ws, L.tile);
    uint32_t* nlong = at<uint32_t>(ws, L.nlong);
    uint32_t* longs = at<uint32_t>(ws, L.longs);
    const int64_t most = L.points > capacity ? L.points : capacity;
    k_pl_clear<<<blocks_for(most, kPlThreads * 4, 4096), kPlThreads, 0, s>>>(count, L.points, nlong, pt_center,
                                                                             capacity);
    const int rb = blocks_for(g.rows, kPlThreads / kWave, 1 << 16);
    k_pl_count<<<rb, kPlThreads, 0, s>>>(g, count);
    k_pl_tiles<<<(uint32_t)L.tiles, kPlThreads, 0, s>>>(count, L.points, tile);
    k_pl_scan<<<1, kPlThreads, 0, s>>>(tile, L.tiles);
    k_pl_offsets<<<(uint32_t)L.tiles, kPlThreads, 0, s>>>(count, L.points, tile, pt_off, nlong, longs,
                                                           L.most_long);
    k_pl_fill<<<rb, kPlThreads, 0, s>>>(g, count, pt_center, capacity);
    k_pl_short<<<blocks_for(L.points, kPlThreads / kWave, 1 << 16), kPlThreads, 0, s>>>(pt_off, L.points, pt_center,
                                                                                           capacity);
    k_pl_long<<<kPlLongBlocks, kPlLongThreads, 0, s>>>(pt_off, nlong, longs, L.most_long, pt_center, capacity);
    return hipGetLastError();
}

}  // namespace cagq
