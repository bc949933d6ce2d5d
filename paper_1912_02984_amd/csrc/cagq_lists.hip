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
// loads and a few barriers.
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

// Small clouds in one or two launches instead of four: k_pl_cloud takes a range
// of a cloud's points, reads all of the cloud's slots, keeps those of its
// points in LDS in slot order, and places them as k_pl_build does. What comes
// before its range it counts on the way, what the clouds before hold k_pl_total
// has counted. For clouds whose slots fit its LDS, and batches whose workgroups
// all run at once. Against the four launches, in a row on a stream: one object
// (1024 points, 512 centers of 32) 18.9 -> 12.9 us, 16 of them 22.6 -> 16.8, 256
// of them 80 -> 43; four of 8192 points 23.6 -> 16.8; 64 of 1024 points with 128
// centers 25 -> 11.
constexpr int kPcThreads = 1024;
constexpr int kPcWaves = kPcThreads / kWave;
constexpr int kPcSlots = 16384;     // most slots of a cloud
constexpr int kPcWaveSlots = kPcSlots / kPcWaves;
constexpr int kPcRange = 1024;      // most points of a workgroup
constexpr int kPcBits = 10;         // of a point within it
constexpr int kPcAim = 1024;        // slots that its points should have
constexpr int kPcBlocks = 256;      // most workgroups (their LDS leaves one on a CU)
constexpr int kPcTotals = 4;        // most parts in which a cloud's slots are counted

struct PlLayout {
    int64_t points;
    int32_t shift, bins, tiles, tile_slots, scan_tiles;
    int32_t parts, range, totals;  // small clouds: workgroups of a cloud, points of each, counts; otherwise 0
    size_t hist, desc, rec, total;
};

void small_clouds(const Groups& g, int32_t B, PlLayout& L) {
    L.parts = L.range = L.totals = 0;
    const int64_t slots = g.K > 0 ? (int64_t)g.M * g.K : g.idx_len;  // a ragged cloud may have them all
    if (B < 1 || B > kPcBlocks || g.rows < 1 || g.N < 1 || slots < 1 || slots > kPcSlots || g.M >> (32 - kPcBits))
        return;
    int64_t parts = (slots + kPcAim - 1) / kPcAim;
    if (parts > kPcBlocks / B) parts = kPcBlocks / B;
    if (parts < (g.N + kPcRange - 1) / kPcRange) parts = (g.N + kPcRange - 1) / kPcRange;
    const int64_t range = (g.N + parts - 1) / parts;
    parts = (g.N + range - 1) / range;
    if (B * parts > kPcBlocks) return;
    L.parts = (int32_t)parts;
    L.range = (int32_t)range;
    L.totals = kPcBlocks / B < kPcTotals ? kPcBlocks / B : kPcTotals;
}

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
    small_clouds(g, B, L);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at = (at + bytes + 255) & ~(size_t)255;
        return here;
    };
    if (L.parts) {
        L.hist = take((size_t)B * L.totals * 4);  // slots that count, of each cloud's parts
        L.total = at;
        return L;
    }
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
    const int32_t* start; // LDS: where each of them starts, and the last ends, from s0
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
            for (int r = threadIdx.x; r <= rows + 1 && r <= kPlRows; r += blockDim.x) {
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
            const auto search = [&](const auto* from, auto at) {
                int32_t lo = 0, hi = rows;
                while (lo < hi) {
                    const int32_t mid = lo + (hi - lo + 1) / 2;
                    if (from[mid] <= at) lo = mid;
                    else hi = mid - 1;
                }
                row = row0 + lo;
                ok = ok && from[lo] <= at && at < from[lo + 1];
            };
            if (rows < kPlRows) search(start, (int32_t)(s - s0));
            else search(g.off + row0, s);
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
    __shared__ int32_t s_start[kPlRows + 1];
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
    __shared__ int32_t s_start[kPlRows + 1];
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

// The slots of a cloud, and of one of its waves' part of them.
__device__ __forceinline__ void cloud_slots(const Groups& g, int32_t b, int64_t& beg, int64_t& end) {
    int64_t x;
    g.range(b * g.M, beg, x);
    g.range(b * g.M + g.M - 1, x, end);
}

__global__ __launch_bounds__(kPcThreads) void k_pl_total(Groups g, int32_t totals, Magic by_k,
                                                         uint32_t* __restrict__ total) {
    __shared__ int32_t s_start[kPlRows + 1];
    __shared__ uint32_t s_sum[kPcWaves];
    int64_t beg, end;
    const int32_t b = (int32_t)blockIdx.x / totals, t0 = (int32_t)blockIdx.x - b * totals;
    cloud_slots(g, b, beg, end);
    const int64_t n = end - beg;
    end = beg + n * (t0 + 1) / totals;
    beg += n * t0 / totals;
    uint32_t c = 0;
    if (beg < end) {
        const Tile t(g, beg, end, by_k, s_start);
        for (int64_t s = beg + threadIdx.x; s < end; s += kPlKeep * kPcThreads) {
#pragma unroll
            for (int i = 0; i < kPlKeep; ++i) {
                uint32_t gp;
                int32_t j;
                if (s + i * kPcThreads < end) c += t.slot(g, s + i * kPcThreads, gp, j);
            }
        }
    }
    c = wave_incl_sum_u32(c);
    if (lane_id() == kWave - 1) s_sum[threadIdx.x / kWave] = c;
    __syncthreads();
    if (threadIdx.x == 0) {
        uint32_t all = 0;
        for (int w = 0; w < kPcWaves; ++w) all += s_sum[w];
        total[blockIdx.x] = all;
    }
}

// total: of the clouds' parts; null: there is one, and its workgroups count all of it.
__global__ __launch_bounds__(kPcThreads) void k_pl_cloud(Groups g, int32_t B, int32_t parts, int32_t range, Magic by_k,
                                                         int32_t totals, const uint32_t* __restrict__ total,
                                                         int64_t* __restrict__ off, int32_t* __restrict__ center,
                                                         int64_t capacity) {
    extern __shared__ uint32_t s_dyn[];  // [wave][point] counters, [wave][kPcWaveSlots] (center, point)
    __shared__ int32_t s_start[kPlRows + 1];
    __shared__ uint32_t s_sum[kPcWaves], s_base[kPcWaves], s_all[kPcWaves];
    const int wave = threadIdx.x / kWave, lane = lane_id();
    const int32_t b = (int32_t)blockIdx.x / parts, p0 = ((int32_t)blockIdx.x - b * parts) * range;
    const int np = g.N - p0 < range ? g.N - p0 : range;
    uint32_t* cnt = s_dyn + wave * np;
    uint32_t* mine = s_dyn + kPcWaves * range + wave * kPcWaveSlots;
    for (int i = threadIdx.x; i < kPcWaves * np; i += kPcThreads) s_dyn[i] = 0;
    uint32_t base = 0, all = 0;  // slots before this range; all of the batch
    if (total)
        for (int i = threadIdx.x; i < B * totals; i += kPcThreads) {
            const uint32_t c = total[i];
            all += c;
            base += i < b * totals ? c : 0;
        }
    int64_t beg, end;
    cloud_slots(g, b, beg, end);
    int kept = 0;
    if (beg < end) {
        const Tile t(g, beg, end, by_k, s_start);  // with a barrier
        const int64_t per = ((end - beg + kPcWaves - 1) / kPcWaves + kWave - 1) & ~(int64_t)(kWave - 1);
        const int64_t a = beg + wave * per, z = a + per < end ? a + per : end;
        for (int64_t s = a + lane; s - lane < z; s += kPlKeep * kWave) {
            uint32_t gp[kPlKeep];
            int32_t j[kPlKeep];
            bool on[kPlKeep];
#pragma unroll
            for (int i = 0; i < kPlKeep; ++i) on[i] = s + i * kWave < z && t.slot(g, s + i * kWave, gp[i], j[i]);
#pragma unroll
            for (int i = 0; i < kPlKeep; ++i) {
                const uint32_t k = gp[i] - ((uint32_t)b * (uint32_t)g.N + (uint32_t)p0);
                const bool in = on[i] && k < (uint32_t)np;
                base += on[i] && (int32_t)k < 0;
                all += !total && on[i];
                const uint64_t m = __ballot(in);
                if (in) {
                    mine[kept + __popcll(m & ((1ull << lane) - 1))] = (uint32_t)j[i] << kPcBits | k;
                    atomicAdd(&cnt[k], 1u);
                }
                kept += __popcll(m);
            }
        }
    }
    base = wave_incl_sum_u32(base);
    all = wave_incl_sum_u32(all);
    if (lane == kWave - 1) {
        s_base[wave] = base;
        s_all[wave] = all;
    }
    __syncthreads();
    // a thread's point (at most kPcRange = kPcThreads): its entries, then the prefix over all
    uint32_t sum = 0;
    if ((int)threadIdx.x < np)
        for (int w = 0; w < kPcWaves; ++w) sum += s_dyn[w * np + threadIdx.x];
    const uint32_t incl = wave_incl_sum_u32(sum);
    if (lane == kWave - 1) s_sum[wave] = incl;
    __syncthreads();
    uint32_t run = incl - sum;
    all = 0;
    for (int w = 0; w < kPcWaves; ++w) {
        run += s_base[w] + (w < wave ? s_sum[w] : 0u);
        all += s_all[w];
    }
    if ((int)threadIdx.x < np) {
        off[(int64_t)b * g.N + p0 + threadIdx.x] = run;
        for (int w = 0; w < kPcWaves; ++w) {
            const uint32_t c = s_dyn[w * np + threadIdx.x];
            s_dyn[w * np + threadIdx.x] = run;
            run += c;
        }
    }
    __syncthreads();
    int bits = 0;
    while ((1 << bits) < np) ++bits;
    for (int e = 0; e < kept; e += kWave) {
        const bool on = e + lane < kept;
        const uint32_t x = on ? mine[e + lane] : 0u;
        const uint32_t at = next_place(cnt, x & ((1u << kPcBits) - 1u), bits, on);
        if (on && at < capacity) center[at] = (int32_t)(x >> kPcBits);
    }
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) off[(int64_t)B * g.N] = all;
    for (int64_t i = all + (int64_t)blockIdx.x * kPcThreads + threadIdx.x; i < capacity;
         i += (int64_t)gridDim.x * kPcThreads)
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
    if (L.parts) {
        const size_t lds = ((size_t)kPcWaves * L.range + kPcSlots) * 4;
        if ((e = allow_lds(k_pl_cloud, lds)) != hipSuccess) return e;
        if (B > 1) k_pl_total<<<B * L.totals, kPcThreads, 0, s>>>(g, L.totals, by_k, hist);
        k_pl_cloud<<<B * L.parts, kPcThreads, lds, s>>>(g, B, L.parts, L.range, by_k, L.totals,
                                                        B > 1 ? hist : nullptr, pt_off, pt_center, capacity);
        return hipGetLastError();
    }
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
