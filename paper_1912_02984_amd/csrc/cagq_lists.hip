// The groups turned round: for each point the centers whose groups hold it,
// ascending (cagq_point_lists).
//
// A stable sort of the slots by point, in two steps, so that every list comes
// out in the order of the slots, that is of the centers, and nothing is sorted
// afterwards: the points of the batch are cut into bins of 2^shift in a row;
//   k_pl_hist     counts each tile's slots per bin,
//   k_pl_scan     turns the counts, bin by bin and tile by tile, into places,
//   k_pl_scatter  writes each slot's (point, center) to its bin, in slot order,
//   k_pl_build    does the same within a bin, point by point, and writes the
//                 offsets.
// Within a workgroup each wave takes consecutive entries and keeps counters of
// its own; equal keys of a wave's 64 entries are found by ballots of the keys'
// bits. Counting and placing slots by atomics on the points' counters instead,
// and sorting each list, took 155 us for the indoor scenes (779000 of 2^20
// slots that count, 327680 points): the atomics cross the XCDs' L2s. The four
// launches here take 36 us (hist 6, scan 6, scatter 11, build 14; 9 MB at the
// card's copy rate would take 2): latency, each of them two or three dependent
// loads and a few barriers. Objects (16 x 1024 points, 512 centers of 32) take
// 22 us, of which the launches' host time is 18.
#include "cagq_features.h"

namespace cagq {

namespace {

constexpr int kPlThreads = 512;
constexpr int kPlWaves = kPlThreads / kWave;
constexpr int kPlTile = 1024;       // slots per tile, while that makes at most kPlTiles tiles
constexpr int kPlTiles = 512;
constexpr int kPlRows = 1024;       // ragged: rows of a tile whose starts a workgroup keeps in LDS
constexpr int kPlBins = 2048;       // most bins
constexpr int kPlRange = 2048;      // most points of a bin whose counters fit a workgroup's LDS at once
constexpr int kPlBinSlots = 4096;   // slots a bin should hold (at most 2^shift = kPlRange points for that)
constexpr int kPlKeep = 4;          // slots or entries whose loads a lane has on their way at once
constexpr int kPlScanItems = 8;
constexpr int kPlScanTile = kScanThreads * kPlScanItems;

struct PlLayout {
    int64_t points;
    int32_t shift, bins, tiles, tile_slots, scan_tiles;
    size_t hist, desc, rec, total;
};

PlLayout pl_layout(const Groups& g, int32_t B) {
    PlLayout L;
    L.points = (int64_t)B * g.N;
    int64_t ts = (g.idx_len + kPlTiles - 1) / kPlTiles;
    ts = ts < kPlTile ? kPlTile : (ts + kPlThreads - 1) / kPlThreads * kPlThreads;
    L.tile_slots = (int32_t)ts;
    L.tiles = (int32_t)((g.idx_len + ts - 1) / ts);
    if (L.tiles < 1) L.tiles = 1;
    // points to a bin: a power of two
    const int64_t per = g.idx_len > 0 ? kPlBinSlots * L.points / g.idx_len : kPlRange;
    L.shift = 2;
    while ((2ll << L.shift) <= per && (2 << L.shift) <= kPlRange) ++L.shift;
    while ((L.points + (1ll << L.shift) - 1) >> L.shift > kPlBins) ++L.shift;
    L.bins = (int32_t)((L.points + (1ll << L.shift) - 1) >> L.shift);
    L.scan_tiles = (int32_t)(((int64_t)L.bins * L.tiles + kPlScanTile - 1) / kPlScanTile);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at = (at + bytes + 255) & ~(size_t)255;
        return here;
    };
    L.hist = take(((size_t)L.bins * L.tiles + 1) * 4);
    L.desc = take(((size_t)L.scan_tiles + 1) * 8);  // look-back descriptors, then the ticket
    L.rec = take((size_t)g.idx_len * 8);
    L.total = at;
    return L;
}

// The slots [s0, s1) of a tile: their groups' rows.
struct Tile {
    int64_t s0;
    int32_t row0, rows;   // ragged: rows the tile may touch after row0
    const int32_t* start; // LDS: where each of them starts, from s0
    Magic by_k;

    // The last row whose list starts at or before s, or row 0: a wave's lanes probe 64 rows at once.
    static __device__ __forceinline__ int32_t row_of(const Groups& g, int64_t s) {
        int32_t lo = 0, n = g.rows;
        while (n > 1) {
            const int32_t step = (n + kWave - 1) / kWave;
            const int64_t at = (int64_t)lane_id() * step;
            const int c = __popcll(__ballot(at < n && g.off[lo + (at < n ? at : 0)] <= s));
            const int32_t skip = c > 0 ? (c - 1) * step : 0;
            lo += skip;
            n = n - skip < step ? n - skip : step;
        }
        return lo;
    }
    // Every thread of the block; ends with a barrier.
    __device__ __forceinline__ Tile(const Groups& g, int64_t s0_, int64_t s1, Magic by_k_, int32_t* lds)
        : s0(s0_), rows(0), start(lds), by_k(by_k_) {
        if (g.K > 0) {
            row0 = (int32_t)(s0 / g.K);
        } else {
            row0 = row_of(g, s0);
            rows = row_of(g, s1 - 1) - row0;
            for (int r = threadIdx.x; r <= rows && r < kPlRows; r += kPlThreads) {
                const int64_t d = g.off[row0 + r] - s0;
                lds[r] = (int32_t)(d < -1 ? -1 : d > 0x7FFFFFFF ? 0x7FFFFFFF : d);
            }
        }
        __syncthreads();
    }
    // Whether slot s counts; its point over the batch and its center.
    __device__ __forceinline__ bool slot(const Groups& g, int64_t s, uint32_t& gp, int32_t& j) const {
        int32_t row;
        const int32_t i = g.idx[s];
        bool ok = (uint32_t)i < (uint32_t)g.N;
        if (g.K > 0) {
            const uint32_t d = (uint32_t)(s - (int64_t)row0 * g.K), r = udiv(d, by_k);
            row = row0 + (int32_t)r;
            if (g.n_valid) ok = ok && (int32_t)(d - r * (uint32_t)g.K) < g.n_valid[row];
        } else {
            int32_t lo = 0, hi = rows;
            while (lo < hi) {
                const int32_t mid = lo + (hi - lo + 1) / 2;
                const bool before = rows < kPlRows ? start[mid] <= (int32_t)(s - s0) : g.off[row0 + mid] <= s;
                if (before) lo = mid;
                else hi = mid - 1;
            }
            row = row0 + lo;
            ok = ok && g.off[row] <= s && s < g.off[row + 1];
        }
        const uint32_t b = udiv((uint32_t)row, g.mm);
        gp = b * (uint32_t)g.N + (uint32_t)i;
        j = row - (int32_t)(b * (uint32_t)g.M);
        return ok;
    }
};

__global__ __launch_bounds__(kPlThreads) void k_pl_hist(Groups g, PlLayout L, Magic by_k, uint32_t* __restrict__ hist,
                                                        uint64_t* __restrict__ desc) {
    extern __shared__ uint32_t s_cnt[];
    __shared__ int32_t s_start[kPlRows];
    for (int i = threadIdx.x; i < L.bins; i += kPlThreads) s_cnt[i] = 0;
    for (int64_t i = (int64_t)blockIdx.x * kPlThreads + threadIdx.x; i <= L.scan_tiles;
         i += (int64_t)gridDim.x * kPlThreads)
        desc[i] = 0;
    __syncthreads();
    const int64_t s0 = (int64_t)blockIdx.x * L.tile_slots;
    const int64_t s1 = s0 + L.tile_slots < g.idx_len ? s0 + L.tile_slots : g.idx_len;
    if (s0 < s1) {
        const Tile t(g, s0, s1, by_k, s_start);
        for (int64_t s = s0 + threadIdx.x; s < s1; s += kPlKeep * kPlThreads) {
            uint32_t gp[kPlKeep];
            int32_t j;
            bool on[kPlKeep];
#pragma unroll
            for (int i = 0; i < kPlKeep; ++i)
                on[i] = s + i * kPlThreads < s1 && t.slot(g, s + i * kPlThreads, gp[i], j);
#pragma unroll
            for (int i = 0; i < kPlKeep; ++i)
                if (on[i]) atomicAdd(&s_cnt[gp[i] >> L.shift], 1u);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < L.bins; i += kPlThreads) hist[(int64_t)i * L.tiles + blockIdx.x] = s_cnt[i];
}

// Exclusive prefix of the counts in place, the total behind them.
__global__ __launch_bounds__(kScanThreads) void k_pl_scan(int64_t n, uint32_t* __restrict__ hist,
                                                          uint64_t* __restrict__ desc, unsigned* __restrict__ ticket) {
    __shared__ uint64_t s_wave[kScanThreads / kWave];
    __shared__ uint64_t s_prefix;
    __shared__ uint32_t s_ticket;
    if (threadIdx.x == 0) s_ticket = atomicAdd(ticket, 1u);
    __syncthreads();
    const int64_t tile = s_ticket;
    const int64_t i0 = tile * kPlScanTile + (int64_t)threadIdx.x * kPlScanItems;
    uint32_t v[kPlScanItems], sum = 0;
#pragma unroll
    for (int k = 0; k < kPlScanItems; ++k) {
        v[k] = i0 + k < n ? hist[i0 + k] : 0;
        sum += v[k];
    }
    uint64_t agg;
    const uint64_t excl = block_excl_scan(sum, s_wave, &agg);
    uint32_t run = (uint32_t)(tile_lookback(desc, tile, agg, &s_prefix) + excl);
#pragma unroll
    for (int k = 0; k < kPlScanItems; ++k) {
        if (i0 + k < n) hist[i0 + k] = run;
        run += v[k];
        if (i0 + k == n - 1) hist[n] = run;
    }
}

// Lanes of the wave with the same key (of `bits` bits) as this one, among
// those that are `on`.
__device__ __forceinline__ uint64_t same_key(uint32_t key, int bits, bool on) {
    uint64_t m = __ballot(on);
    for (int b = 0; b < bits; ++b) {
        const bool one = key >> b & 1;
        const uint64_t o = __ballot(one);
        m &= one ? o : ~o;
    }
    return m;
}

// The entry's place among its wave's entries of that key: the counter (a
// wave's own) before it, moved on by the last lane of the key.
__device__ __forceinline__ uint32_t next_place(uint32_t* cnt, uint32_t key, int bits, bool on) {
    const int lane = lane_id();
    const uint64_t m = same_key(key, bits, on);
    const uint32_t before = (uint32_t)__popcll(m & ((1ull << lane) - 1));
    uint32_t at = 0;
    if (on) {
        at = cnt[key] + before;
        if ((m >> lane) == 1) cnt[key] = at + 1;
    }
    __builtin_amdgcn_wave_barrier();
    return at;
}

__global__ __launch_bounds__(kPlThreads) void k_pl_scatter(Groups g, PlLayout L, Magic by_k, int bits,
                                                           const uint32_t* __restrict__ hist,
                                                           uint2* __restrict__ rec) {
    extern __shared__ uint32_t s_cnt[];  // [wave][bin]
    __shared__ int32_t s_start[kPlRows];
    const int wave = threadIdx.x / kWave, lane = lane_id();
    const int64_t s0 = (int64_t)blockIdx.x * L.tile_slots;
    const int64_t s1 = s0 + L.tile_slots < g.idx_len ? s0 + L.tile_slots : g.idx_len;
    if (s0 >= s1) return;
    for (int i = threadIdx.x; i < kPlWaves * L.bins; i += kPlThreads) s_cnt[i] = 0;
    const Tile t(g, s0, s1, by_k, s_start);
    const int64_t per = L.tile_slots / kPlWaves;
    const int64_t a = s0 + wave * per, b = a + per < s1 ? a + per : s1;
    uint32_t* cnt = s_cnt + wave * L.bins;
    // the wave's first 64 * kPlKeep slots stay in registers
    uint32_t gp[kPlKeep];
    int32_t j[kPlKeep];
    bool on[kPlKeep];
    auto load = [&](int64_t s) {
#pragma unroll
        for (int i = 0; i < kPlKeep; ++i) {
            gp[i] = 0;
            j[i] = 0;
            on[i] = s + i * kWave + lane < b && t.slot(g, s + i * kWave + lane, gp[i], j[i]);
        }
    };
    for (int64_t s = a + kPlKeep * kWave; s < b; s += kPlKeep * kWave) {
        load(s);
#pragma unroll
        for (int i = 0; i < kPlKeep; ++i)
            if (on[i]) atomicAdd(&cnt[gp[i] >> L.shift], 1u);
    }
    load(a);
#pragma unroll
    for (int i = 0; i < kPlKeep; ++i)
        if (on[i]) atomicAdd(&cnt[gp[i] >> L.shift], 1u);
    __syncthreads();
    for (int i = threadIdx.x; i < L.bins; i += kPlThreads) {
        uint32_t run = hist[(int64_t)i * L.tiles + blockIdx.x];
        for (int w = 0; w < kPlWaves; ++w) {
            const uint32_t c = s_cnt[w * L.bins + i];
            s_cnt[w * L.bins + i] = run;
            run += c;
        }
    }
    __syncthreads();
    for (int64_t s = a; s < b; s += kPlKeep * kWave) {
        if (s > a) load(s);
#pragma unroll
        for (int i = 0; i < kPlKeep; ++i) {
            const uint32_t at = next_place(cnt, on[i] ? gp[i] >> L.shift : 0u, bits, on[i]);
            if (on[i]) rec[at] = make_uint2(gp[i], (uint32_t)j[i]);
        }
    }
}

__global__ __launch_bounds__(kPlThreads) void k_pl_build(PlLayout L, const uint32_t* __restrict__ hist,
                                                         const uint2* __restrict__ rec, int64_t* __restrict__ off,
                                                         int32_t* __restrict__ center, int64_t capacity) {
    extern __shared__ uint32_t s_cnt[];  // [wave][point]
    __shared__ uint32_t s_sum[kPlWaves];
    const int wave = threadIdx.x / kWave, lane = lane_id();
    const int64_t n = (int64_t)L.bins * L.tiles;
    const uint32_t total = hist[n];
    const uint32_t e0 = hist[(int64_t)blockIdx.x * L.tiles];
    const uint32_t e1 = (int)blockIdx.x + 1 < L.bins ? hist[((int64_t)blockIdx.x + 1) * L.tiles] : total;
    const int64_t first = (int64_t)blockIdx.x << L.shift;
    const int64_t last = first + (1ll << L.shift) < L.points ? first + (1ll << L.shift) : L.points;
    // a quarter of the entries (by waves) each, in order
    const uint32_t per = ((e1 - e0 + kPlWaves - 1) / kPlWaves + kWave - 1) & ~(uint32_t)(kWave - 1);
    const uint32_t a = e0 + wave * per < e1 ? e0 + wave * per : e1, b = a + per < e1 ? a + per : e1;
    uint32_t done = e0;
    // bins of more than kPlRange points: that many at a time
    for (int64_t p0 = first; p0 < last; p0 += kPlRange) {
        const int np = last - p0 < kPlRange ? (int)(last - p0) : kPlRange;
        int bits = 0;
        while ((1 << bits) < np) ++bits;
        uint32_t* cnt = s_cnt + wave * np;
        for (int i = threadIdx.x; i < kPlWaves * np; i += kPlThreads) s_cnt[i] = 0;
        __syncthreads();
        for (uint32_t e = a + lane; e < b; e += kPlKeep * kWave) {
            uint32_t k[kPlKeep];
#pragma unroll
            for (int i = 0; i < kPlKeep; ++i)
                k[i] = e + i * kWave < b ? rec[e + i * kWave].x - (uint32_t)p0 : 0xFFFFFFFFu;
#pragma unroll
            for (int i = 0; i < kPlKeep; ++i)
                if (k[i] < (uint32_t)np) atomicAdd(&cnt[k[i]], 1u);
        }
        __syncthreads();
        // each thread's points in a row: their totals, then the prefix over all
        const int each = (np + kPlThreads - 1) / kPlThreads;
        const int i0 = threadIdx.x * each, i1 = i0 + each < np ? i0 + each : np;
        uint32_t sum = 0;
        for (int i = i0; i < i1; ++i)
            for (int w = 0; w < kPlWaves; ++w) sum += s_cnt[w * np + i];
        const uint32_t incl = wave_incl_sum_u32(sum);
        if (lane == kWave - 1) s_sum[wave] = incl;
        __syncthreads();
        uint32_t run = done + incl - sum, all = 0;
        for (int w = 0; w < kPlWaves; ++w) {
            if (w < wave) run += s_sum[w];
            all += s_sum[w];
        }
        for (int i = i0; i < i1; ++i) {
            off[p0 + i] = run;
            for (int w = 0; w < kPlWaves; ++w) {
                const uint32_t c = s_cnt[w * np + i];
                s_cnt[w * np + i] = run;
                run += c;
            }
        }
        done += all;
        __syncthreads();
        for (uint32_t e = a; e < b; e += kPlKeep * kWave) {
            uint2 r[kPlKeep];
#pragma unroll
            for (int i = 0; i < kPlKeep; ++i) {
                r[i] = make_uint2(0, 0);
                if (e + i * kWave + lane < b) r[i] = rec[e + i * kWave + lane];
            }
#pragma unroll
            for (int i = 0; i < kPlKeep; ++i) {
                const uint32_t k = r[i].x - (uint32_t)p0;
                const bool on = e + i * kWave + lane < b && k < (uint32_t)np;
                const uint32_t at = next_place(cnt, on ? k : 0u, bits, on);
                if (on && at < capacity) center[at] = (int32_t)r[i].y;
            }
        }
        __syncthreads();
    }
    if (last == L.points && threadIdx.x == 0) off[L.points] = total;
    for (int64_t i = total + (int64_t)blockIdx.x * kPlThreads + threadIdx.x; i < capacity;
         i += (int64_t)gridDim.x * kPlThreads)
        center[i] = -1;
}

int bits_of(int64_t n) {  // of numbers below n
    int b = 0;
    while ((1ll << b) < n) ++b;
    return b;
}

template <typename K>
hipError_t allow_lds(K kern, size_t bytes) {
    if (bytes <= (48 << 10)) return hipSuccess;
    return hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

}  // namespace

size_t point_lists_bytes(const Groups& g, int32_t B) { return pl_layout(g, B).total; }

hipError_t launch_point_lists(const Groups& g, int32_t B, int64_t* pt_off, int32_t* pt_center, int64_t capacity,
                              void* ws, hipStream_t s) {
    const PlLayout L = pl_layout(g, B);
    uint32_t* hist = at<uint32_t>(ws, L.hist);
    uint64_t* desc = at<uint64_t>(ws, L.desc);
    uint2* rec = at<uint2>(ws, L.rec);
    const Magic by_k = make_magic(g.K > 0 ? (uint32_t)g.K : 1u);
    const int64_t range = (1ll << L.shift) < kPlRange ? (1ll << L.shift) : kPlRange;
    const size_t bins_lds = (size_t)L.bins * 4, waves_lds = bins_lds * kPlWaves;
    const size_t range_lds = (size_t)range * 4 * kPlWaves;
    hipError_t e;
    if ((e = allow_lds(k_pl_scatter, waves_lds)) != hipSuccess) return e;
    if ((e = allow_lds(k_pl_build, range_lds)) != hipSuccess) return e;
    k_pl_hist<<<L.tiles, kPlThreads, bins_lds, s>>>(g, L, by_k, hist, desc);
    k_pl_scan<<<L.scan_tiles, kScanThreads, 0, s>>>((int64_t)L.bins * L.tiles, hist, desc,
                                                    (unsigned*)(desc + L.scan_tiles));
    k_pl_scatter<<<L.tiles, kPlThreads, waves_lds, s>>>(g, L, by_k, bits_of(L.bins), hist, rec);
    k_pl_build<<<L.bins, kPlThreads, range_lds, s>>>(L, hist, rec, pt_off, pt_center, capacity);
    return hipGetLastError();
}

}  // namespace cagq
