// Attention of each center over the features of its group, and its gradients
// (cagq_group_attention, cagq_group_attention_backward; the formulas are in
// include/cagq.h).
//
// A query here meets a list of its own, so there is no tile of queries that
// share keys and no matrix product to make of it: a pair costs 4 D flops and
// reads 2 D features. The work is gathering rows, and the kernels are built to
// keep many gathered rows in flight:
//   - G lanes to a head of a row (16 bytes of features each), the row's heads
//     side by side, and as many rows at once as the wave has lanes for (slots);
//   - a list's entries are made ready a chunk at a time, one per lane (index,
//     place, the bias of every head), and left in LDS for the rows' lanes;
//   - two to four rows of each slot are loaded before the first is used. Loads go
//     through a bounds-checked buffer, in which an entry that is not there has
//     an offset past the end and reads as zeros, without a branch;
//   - three ways to share the work: EACH, a list per slot (many short lists: no
//     slot waits for another list's end, nothing is joined); one list for all of
//     a wave's slots, joined by permutes at its end; BLOCK, in the forward pass
//     alone, one list for all of a workgroup's waves, joined in LDS, in parts
//     where lists are few.
// Scores stay in natural units (times log2 e, a bias of the type's lowest
// value would become -infinity), and only differences of them are taken to
// base 2.
//
// The gradients take two passes: at the centers (dq, and delta = sum p dp) and
// at the points (dk, dv and the bias's), each recomputing the scores: that
// reads two rows a pair, as storing and fetching weights for every pair and
// head would need memory for them all. An entry that is not there, and a pair
// that the bias masks, add zeros to every sum whatever k, v, q and dout hold: a
// value that is not finite is selected away, not multiplied by 0.
//
// Measured on indoor scenes (4 x 81920 points, 8192 centers of 32, 8 heads of
// 32 channels in bfloat16: 779000 pairs, of which each reads two rows of 512
// bytes): forward 100 us, gradients 113 us at the centers and 257 us at the
// points. The caches' misses bound all three: 0.58, 0.60 and 1.32 GB at 5.1 to
// 5.8 TB/s (rows are as much as a cloud's 84 MB apart in time of use, an L2
// holds 4 MB), against 0.35 GB that the forward cannot do without; its loads
// without any arithmetic take 97 us. Short rows are bound by issue instead:
// whole contexts (2 x 3001 centers, 1.28 M pairs, 6 heads of 16) 90 us, of
// which 45 are vector instructions, the rest of it the longest lists' ends and
// the L1's 64 lanes' gathers. A few short lists take a chain of cold loads: 8 us.
#include <initializer_list>

#include "cagq_features.h"

namespace cagq {

namespace {

constexpr int kAtThreads = 256;
constexpr int kAtWaves = kAtThreads / kWave;
// Workgroups of a launch; they go round where there is more to do. Short lists:
// as many as the card holds at once, so that the waves of an XCD walk through
// its rows side by side and none starts late. Long ones: as many as there are,
// handed out as workgroups end.
constexpr int kAtBlocks = 256 * 3;
constexpr int kAtMany = 1 << 16;
constexpr int kAtLds = 144 << 10;    // LDS of a workgroup: edges, table, chunks, and the waves' gradient tables
constexpr int kCuLds = 160 << 10;    // what a workgroup can have at most
constexpr int kPoints = 16;          // most points in a row whose lists one slot walks (FLAT)
constexpr int kJoinFloats = 2048;    // H * D up to which a workgroup's waves join their parts in LDS
// Caps above it: see Score::products. Of 2-byte features a score is off by some
// 2^-9 of its products' sizes anyway.
template <typename T>
constexpr float kWideCap = sizeof(T) == 4 ? 0.0f : 64.0f;
// Groups whose |lse| is above it: beside such an lse the log of the weights'
// sum is (partly) rounded away - all of it where a whole group has scores of the
// type's lowest value - and weights exp(s - lse) sum up to as much as their
// number instead of 1. The gradients divide them by their sum. Below, a weight
// is off by less than 2^-16 by it.
constexpr float kFarLse = 256.0f;
constexpr float kNegInf = -__builtin_inff();
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// How a wave's lanes are laid over a row of `heads` heads of D channels.
struct Lanes {
    int32_t G;       // lanes per head, a power of two
    int32_t Hc;      // heads side by side
    int32_t S;       // slots: rows at once
    int32_t passes;  // launches' y: parts of a row's heads
};

template <typename T>
Lanes make_lanes(int32_t heads, int32_t D) {
    Lanes l;
    l.G = 1;
    while (l.G * kVec<T> < D) l.G <<= 1;
    const int32_t items = kWave / l.G;
    l.Hc = heads < items ? heads : items;
    l.S = items / l.Hc;
    l.passes = (heads + l.Hc - 1) / l.Hc;
    return l;
}

struct LaneAt {
    int slot, li, head, chan, n;  // slot, lane within it, head, first channel, channels
    bool on;                      // it has work

    __device__ __forceinline__ LaneAt(const Lanes& l, int heads, int D, int W) {
        const int lane = lane_id();
        const int item = lane / l.G;
        slot = item / l.Hc;
        li = lane - slot * l.Hc * l.G;
        head = (int)blockIdx.y * l.Hc + item - slot * l.Hc;
        chan = (lane & (l.G - 1)) * W;
        on = slot < l.S && head < heads;
        n = D - chan;
        n = !on || n < 0 ? 0 : n > W ? W : n;
        if (!on) head = 0;
    }
};

// The rows of one cloud. BUF: a buffer of at most kMostBytes, rows aligned to
// 16 bytes. An entry that is not there (kNone) and a lane without channels
// (kMostBytes) each bring an offset past its end, and so do both together:
// their sum stays below 2^32. Otherwise pointers, element by element.
constexpr uint32_t kNone = 0x80000000u;
constexpr uint32_t kMostBytes = kNone - 4096;

template <typename T, bool BUF>
struct Rows {
    __amdgpu_buffer_rsrc_t rsrc;
    const T* base;
    int64_t row;
    uint32_t lane_off;
    int n;

    // `first`: the cloud's first row; `bytes` of the cloud; the lane's head and channel.
    __device__ __forceinline__ Rows(const T* first, int64_t row_, uint32_t bytes, int lane_elem, int n_) {
        if constexpr (BUF) {
            rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)first, 0, (int)bytes, 0x00027000);
            lane_off = n_ > 0 ? (uint32_t)lane_elem * (uint32_t)sizeof(T) : kMostBytes;
        } else {
            base = first + lane_elem;
            row = row_;
            n = n_;
        }
    }
    // What an entry's lane makes of its row's index (negative: none), to hand to the row's lanes.
    static __device__ __forceinline__ uint32_t key(int32_t i, uint32_t row_bytes) {
        if constexpr (BUF) return i < 0 ? kNone : (uint32_t)i * row_bytes;
        else return (uint32_t)i;
    }
    // `elems`: elements further on, the same for the wave.
    __device__ __forceinline__ Raw load(uint32_t key, int elems = 0) const {
        if constexpr (BUF)
            return __builtin_amdgcn_raw_buffer_load_b128(rsrc, key + lane_off, elems * (int)sizeof(T), 0);
        else return load_channels<T, false>(base + (int64_t)(int32_t)key * row + elems, (int32_t)key >= 0 ? n : 0);
    }
    static __device__ __forceinline__ bool there(uint32_t key) { return (int32_t)key >= 0; }
};

// Rows to write, dense, past the caches, which the centers' rows are to keep
// (indoor scenes with gradients 519 -> 505 us).
template <typename T, bool BUF>
struct RowsOut {
    T* base;
    int64_t row;
    int n;

    __device__ __forceinline__ RowsOut(T* first, int64_t row_, int lane_elem, int n_)
        : base(first + lane_elem), row(row_), n(n_) {}
    __device__ __forceinline__ void store(int32_t i, const float (&x)[kVec<T>]) const {
        if constexpr (BUF)  // a cloud's rows take less than 2^31 bytes
            store_channels<T, BUF, true>((T*)((char*)base + (uint32_t)i * (uint32_t)(row * (int)sizeof(T))), n, x);
        else store_channels<T, BUF>(base + i * row, n, x);
    }
};

// Keeps the compiler from making a branch that is hardly ever taken into
// selects that always run.
__device__ __forceinline__ void rare() { asm volatile(""); }

// What all kernels know of the scores.
struct Score : PlaceBias {
    float mul;  // of a product: scale, or with a cap 2 log2 e scale / cap
    float cap, scale;

    __device__ __forceinline__ Score(const Bias& b, const Attn& a, float* s) : PlaceBias(b, s) {
        cap = a.cap;
        scale = a.scale;
        mul = cap > 0.0f ? 2.0f * kLog2e * a.scale / cap : a.scale;
    }

    // The scores of N products, s[0], s[BY], ..., before the bias:
    // cap * tanh(scale * x / cap) as cap - 2 cap / (1 + exp(2 scale x / cap)),
    // off by some 2^-24 of the cap, not of x. Of a cap above kWideCap that is
    // too much (a large one stands for hardly any cap; float32 features under a
    // cap of 45 came out 1.3e-6 off instead of 2.2e-7), and arguments y below
    // 1/4 take the series y - y^3/3 + 2y^5/15 - 17y^7/315 + 62y^9/2835, whose
    // next term is below 2^-26 of it. `e`: 1 / (1 + exp), of which the tanh's
    // slope is 4 e (1 - e).
    template <typename T, int N, int BY>
    __device__ __forceinline__ void products(float (&s)[N * BY], float (&e)[N]) const {
        if (cap > 0.0f) {
            float x[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[i] = s[i * BY];
                e[i] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x[i] * mul));
                s[i * BY] = fmaf(-2.0f * cap, e[i], cap);
            }
            if (cap > kWideCap<T>) {
                rare();
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float z = x[i] * scale, y = z / cap, w = y * y;
                    float p = fmaf(w, 62.0f / 2835.0f, -17.0f / 315.0f);
                    p = fmaf(w, fmaf(w, fmaf(w, p, 2.0f / 15.0f), -1.0f / 3.0f), 1.0f);
                    if (fabsf(y) < 0.25f) s[i * BY] = z * p;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                s[i * BY] *= mul;
                e[i] = 0.5f;  // of a tanh at its steepest
            }
        }
    }
    // 1 - tanh^2
    static __device__ __forceinline__ float slack(float e) { return 4.0f * e * (1.0f - e); }
};

// exp(x) of a difference of scores.
__device__ __forceinline__ float weight(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }
__device__ __forceinline__ float weight(float x, float log2_part) {
    return __builtin_amdgcn_exp2f(fmaf(x, kLog2e, log2_part));
}

// Of a row and head, from the gradient at the centers to the one at the points.
struct Stat {
    float z, delta, log_part;  // lse (infinity: none), sum p dp, log2 of what the weights are multiplied by
};

// log of a sum of weights.
__device__ __forceinline__ float log_sum(float x) { return kLn2 * __builtin_amdgcn_logf(x); }

// A chunk of a wave's entries in LDS, a row each: the bias of the wave's heads
// (where there is a bias), then fields. The entries' lanes write the rows and
// the slots' lanes read them; a wave's own LDS operations run in order. Rows
// that no entry's lane writes stay without an entry. Fields: the keys of the
// entry's two rows; at the points also that of its (lse, delta), its point
// (-1: no entry) and the keys of the point's own rows.
constexpr int kKey = 0, kKey2 = 1, kStat = 2, kPoint = 3, kPKey = 4, kPKey2 = 5, kPlace = 6, kDist = 7, kFields = 8;

struct Chunk {
    float* rows;
    int hp, stride;

    // Floats of a row: an odd number of groups of four, so that rows one after another start on different banks.
    static __host__ __device__ int row_floats(int hp) { return (hp + kFields) | 4; }
    static __host__ __device__ int floats(bool placed, int rows_n, int hp) {
        return rows_n * row_floats(placed ? (hp + 3) & ~3 : 0);
    }
    __device__ __forceinline__ Chunk(float* lds, int rows_n, const Score& sc, int hp_) {
        hp = sc.placed() ? (hp_ + 3) & ~3 : 0;
        stride = row_floats(hp);
        rows = lds + (threadIdx.x / kWave) * rows_n * stride;
        for (int r = lane_id(); r < rows_n; r += kWave) {
            rows[r * stride + hp + kKey] = __uint_as_float(kNone);
            rows[r * stride + hp + kKey2] = __uint_as_float(kNone);
            rows[r * stride + hp + kStat] = 0.0f;  // read at any entry
            rows[r * stride + hp + kPoint] = __int_as_float(-1);
            rows[r * stride + hp + kPKey] = __uint_as_float(kNone);
            rows[r * stride + hp + kPKey2] = __uint_as_float(kNone);
        }
    }
    __device__ __forceinline__ const float* row(int r) const { return rows + r * stride; }
    __device__ __forceinline__ uint32_t field(const float* r, int f) const { return __float_as_uint(r[hp + f]); }
    __device__ __forceinline__ void set(int r, int f, uint32_t v) { rows[r * stride + hp + f] = __uint_as_float(v); }

    // The lane's entry into row r: the keys of its rows, and the bias of heads h0 .. h0 + n.
    __device__ __forceinline__ void put(int r, uint32_t key, uint32_t key2, uint32_t u, float d, const Score& sc,
                                        int h0, int n) {
        float* o = rows + r * stride;
        set(r, kKey, key);
        set(r, kKey2, key2);
        if (!sc.placed() || (int32_t)key < 0) return;
        set(r, kPlace, u);
        o[hp + kDist] = d;
        if ((h0 & 3) == 0) {
            for (int h = 0; h < n; h += 4) *(f32x4*)(o + h) = sc.four(u, d, h0 + h);
        } else {
            for (int h = 0; h < n; ++h) o[h] = sc.one(u, d, h0 + h);
        }
    }
};

// Sum over the slots of a wave, in slot 0.
__device__ __forceinline__ float slots_sum(float v, int S, int step, int slot, int lane) {
    int top = 1;
    while (top < S) top <<= 1;
    for (int h = top >> 1; h > 0; h >>= 1) {
        const float o = __shfl(v, (lane + h * step) & 63, kWave);
        if (slot + h < S && slot < h) v += o;
    }
    return v;
}

__device__ __forceinline__ float slots_max(float v, int S, int step, int slot, int lane) {
    int top = 1;
    while (top < S) top <<= 1;
    for (int h = top >> 1; h > 0; h >>= 1) {
        const float o = __shfl(v, (lane + h * step) & 63, kWave);
        if (slot + h < S && slot < h) v = fmaxf(v, o);
    }
    return v;
}

// Which lists the waves take. A unit is a row, or S * P rows of a cloud (P for
// each slot). Units are laid out so that an XCD's workgroups walk through one
// range of them side by side: groups near each other share points, and share
// the XCD's L2.
struct Walk {
    int64_t units;
    int32_t per_cloud;  // units
    int32_t P;
    Magic by_cloud;
};

// `slots`: slots that take rows of their own (1: a row to the wave).
Walk make_walk(int32_t B, int32_t rows_per_cloud, int32_t slots, int32_t P) {
    Walk w;
    w.P = P;
    const int64_t per = (int64_t)slots * P;
    w.per_cloud = (int32_t)((rows_per_cloud + per - 1) / per);
    w.units = (int64_t)B * w.per_cloud;
    w.by_cloud = make_magic((uint32_t)w.per_cloud);
    return w;
}

// f(unit) for the units of this wave (or of this workgroup: per = 1).
template <typename F>
__device__ __forceinline__ void each_unit(int64_t units, int per, int mine, F f) {
    const int64_t x = blockIdx.x & 7, i = blockIdx.x >> 3, n = (gridDim.x + 7 - x) >> 3;
    const int64_t lo = units * x / 8, hi = units * (x + 1) / 8;
    for (int64_t u = lo + i * per + mine; u < hi; u += n * per) f((uint32_t)__builtin_amdgcn_readfirstlane((int)u));
}

// Rows loaded at once: U of each slot. Entries of a chunk: with EACH as many as
// a slot has lanes, else one per lane of the wave.
template <bool EACH, int U>
struct Rounds {
    static __host__ __device__ int slot_rows(const Lanes& l) { return (l.Hc * l.G + U - 1) / U * U; }
    static __host__ __device__ int rows_n(const Lanes& l) {
        if (EACH) return l.S * slot_rows(l);
        return U * l.S < kWave ? kWave : U * l.S;
    }
    int chunk, first, by, per;  // entries; the slot's first row; from one of the U rows to the next; a round's entries

    __device__ __forceinline__ Rounds(const Lanes& l, int slot) {
        const int s = slot < l.S ? slot : 0;
        first = EACH ? s * slot_rows(l) : s;
        by = EACH ? 1 : l.S;
        per = EACH ? U : U * l.S;
        chunk = EACH ? l.Hc * l.G : per < kWave ? kWave / per * per : kWave;  // of whole rounds
    }
};

// Partial softmax of a part of a list: maximum and sum, and the weighted sum's
// D channels, per row and head.
struct Partial {
    float* ml;   // [parts][rows][H][2]
    float* acc;  // [parts][rows][H][D]
    int32_t parts;
};

template <typename T>
__device__ __forceinline__ uint32_t cloud_bytes(int32_t rows, int64_t row, int32_t last) {
    return (uint32_t)(((rows - 1) * row + last) * (int64_t)sizeof(T));
}

template <int R>
constexpr int kUnroll = R == 4 ? 2 : 4;

// One pass over a list with the running maximum and sum; what bounds it and what
// it measured stands at the top.
// R: query heads a lane holds (they share the key's head).
template <typename T, bool BUF, int R, bool EACH, bool BLOCK>
__global__ __launch_bounds__(kAtThreads) void k_at(Groups g, Bias b, Attn a, Lanes l, Walk walk, T* __restrict__ out,
                                                   float* __restrict__ lse, Partial part) {
    constexpr int W = kVec<T>;
    constexpr int U = kUnroll<R>;
    struct Round {
        Raw k[U], v[U];
        float bias[U * R];
        bool there[U];
    };
    extern __shared__ __align__(16) float s_lds[];
    const Score sc(b, a, s_lds);
    const int lane = lane_id(), wave = threadIdx.x / kWave, waves_b = blockDim.x / kWave;
    const LaneAt at(l, a.H / R, a.D, W);
    const Rounds<EACH, U> rd(l, at.slot);
    const int rows_n = Rounds<EACH, U>::rows_n(l), hp = l.Hc * R, hw = (int)blockIdx.y * hp;
    const int hn = a.H - hw < hp ? a.H - hw : hp;  // heads of this pass
    Chunk ck(s_lds + Score::floats(b), rows_n, sc, hp);
    const int h0 = at.head * R, hl = at.on ? h0 - hw : 0;
    const int kvh = h0 / (a.H / a.Hkv);
    const int step = l.Hc * l.G;
    const uint32_t krb = (uint32_t)(a.k_row * (int64_t)sizeof(T)), vrb = (uint32_t)(a.v_row * (int64_t)sizeof(T));
    const uint32_t kbytes = cloud_bytes<T>(g.N, a.k_row, a.Hkv * a.D);
    const uint32_t vbytes = cloud_bytes<T>(g.N, a.v_row, a.Hkv * a.D);

    each_unit(walk.units, BLOCK ? 1 : waves_b, BLOCK ? 0 : wave, [&](uint32_t unit) {
        const uint32_t cloud = udiv(unit, walk.by_cloud);
        const uint32_t in = unit - cloud * (uint32_t)walk.per_cloud;
        const int32_t j = EACH ? (int32_t)in * l.S + at.slot : (int32_t)in;
        const bool live_row = !EACH || (j < g.M && at.slot < l.S);
        const int64_t row = (int64_t)cloud * g.M + (live_row ? j : 0);
        const int64_t p0 = (int64_t)cloud * g.N;
        const Rows<T, BUF> kr((const T*)a.k + p0 * a.k_row, a.k_row, kbytes, kvh * a.D + at.chan, at.n);
        const Rows<T, BUF> vr((const T*)a.v + p0 * a.v_row, a.v_row, vbytes, kvh * a.D + at.chan, at.n);
        Raw q[R];
        float acc[R][W] = {}, m[R], sum[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            q[r] = load_channels<T, BUF>((const T*)a.q + row * a.q_row + (h0 + r) * a.D + at.chan, at.n);
            m[r] = kNegInf;
            sum[r] = 0.0f;
        }
        float c[3] = {};
        if (sc.placed()) load_xyz(g.centers, row, c);
        int64_t beg, end;
        g.range((int32_t)row, beg, end);
        if (EACH && !live_row) end = beg;
        if (!EACH && (BLOCK || part.parts > 1)) {
            const int split = BLOCK ? waves_b * part.parts : part.parts;
            int64_t per = (end - beg + split - 1) / split;
            per = (per + rd.per - 1) / rd.per * rd.per;  // whole rounds
            beg += (BLOCK ? (int64_t)blockIdx.z * waves_b + wave : (int64_t)blockIdx.z) * per;
            end = end < beg + per ? end : beg + per;
        }
        const int e = EACH ? at.li : lane;
        int32_t next = beg + e < end ? g.idx[beg + e] : -1;  // of the next chunk
        for (int64_t s0 = beg; EACH ? __any(s0 < end) : s0 < end; s0 += rd.chunk) {
            const int n = end - s0 < rd.chunk ? (int)(end - s0) : rd.chunk;
            int32_t mine = next;
            uint32_t u = 0;
            float dist = 0.0f;
            next = s0 + rd.chunk + e < end ? g.idx[s0 + rd.chunk + e] : -1;
            if (e < n) {
                if ((uint32_t)mine >= (uint32_t)g.N) mine = -1;
                if (sc.placed() && mine >= 0) {
                    float p[3];
                    load_xyz(g.points, p0 + mine, p);
                    pair_place(sc.ed, sc.dist, p, c, u, dist);
                }
            }
            if (EACH ? at.slot < l.S : e < rd.chunk)
                ck.put(EACH ? rd.first + e : e, Rows<T, BUF>::key(mine, krb), Rows<T, BUF>::key(mine, vrb), u, dist, sc,
                       hw, hn);
            __builtin_amdgcn_wave_barrier();
            auto load = [&](Round& x, int t) {
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const float* r0 = ck.row(rd.first + t + i * rd.by);
                    const uint32_t key = ck.field(r0, kKey);
                    x.there[i] = Rows<T, BUF>::there(key);
                    x.k[i] = kr.load(key);
                    x.v[i] = vr.load(ck.field(r0, kKey2));
#pragma unroll
                    for (int r = 0; r < R; ++r) x.bias[i * R + r] = sc.placed() ? r0[hl + r] : 0.0f;
                }
            };
            auto add = [&](Round& x) {
                float s[U * R];
#pragma unroll
                for (int i = 0; i < U; ++i)
#pragma unroll
                    for (int r = 0; r < R; ++r) s[i * R + r] = dot<T>(q[r], x.k[i]);
                group_sums(s, l.G);
                float low = 0.0f, e2[U * R];
                sc.template products<T, U * R, 1>(s, e2);
#pragma unroll
                for (int i = 0; i < U; ++i) {
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const float sx = s[i * R + r] + x.bias[i * R + r];
                        s[i * R + r] = x.there[i] ? sx : kNegInf;
                        low = fminf(low, x.bias[i * R + r]);
                    }
                }
                if (__any(low == kNegInf)) {  // masked by the bias: whatever k and v hold
                    rare();
#pragma unroll
                    for (int i = 0; i < U; ++i)
#pragma unroll
                        for (int r = 0; r < R; ++r)
                            if (x.bias[i * R + r] == kNegInf) {
                                s[i * R + r] = kNegInf;
                                if (R == 1) x.v[i] = Raw{0, 0, 0, 0};
                            }
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float mn = m[r];
#pragma unroll
                    for (int i = 0; i < U; ++i) mn = fmaxf(mn, s[i * R + r]);
                    const float z = mn == kNegInf ? 0.0f : mn;
                    const float keep = weight(m[r] - z);
                    m[r] = mn;
                    sum[r] *= keep;
#pragma unroll
                    for (int w = 0; w < W; ++w) acc[r][w] *= keep;
#pragma unroll
                    for (int i = 0; i < U; ++i) {
                        const float p = weight(s[i * R + r] - z);
                        sum[r] += p;
                        if (R == 1) {
                            add_channels<T>(acc[r], p, x.v[i]);
                        } else {
                            // heads of their own biases share v: a masked one passes it over
                            const bool off = s[i * R + r] == kNegInf;
#pragma unroll
                            for (int w = 0; w < W; ++w)
                                acc[r][w] = fmaf(p, off ? 0.0f : channel<T>(x.v[i], w), acc[r][w]);
                        }
                    }
                }
            };
            for (int t = 0; EACH ? __any(t < n) : t < n; t += rd.per) {
                Round x;
                load(x, t);
                add(x);
            }
            __builtin_amdgcn_wave_barrier();
        }
        if (!EACH) {  // the slots' parts joined in slot 0
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float all = __shfl(slots_max(m[r], l.S, step, at.slot, lane), at.li, kWave);
                const float f = m[r] == kNegInf ? 0.0f : weight(m[r] - all);
                m[r] = all;
                sum[r] = slots_sum(sum[r] * f, l.S, step, at.slot, lane);
#pragma unroll
                for (int w = 0; w < W; ++w) acc[r][w] = slots_sum(acc[r][w] * f, l.S, step, at.slot, lane);
            }
        }
        const bool writes = EACH ? at.on && live_row : at.on && at.slot == 0;
        if constexpr (BLOCK) {
            // the waves' parts joined in LDS: [wave][heads of this pass][D + 2]
            const int D2 = a.D + 2;
            float* s_join = s_lds + Score::floats(b) + waves_b * Chunk::floats(sc.placed(), rows_n, hp);
            if (writes) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float* d = s_join + (wave * hp + hl + r) * D2;
                    if (at.chan == 0) {
                        d[0] = m[r];
                        d[1] = sum[r];
                    }
#pragma unroll
                    for (int w = 0; w < W; ++w)
                        if (w < at.n) d[2 + at.chan + w] = acc[r][w];
                }
            }
            __syncthreads();
            for (int e = threadIdx.x; e < hn * a.D; e += blockDim.x) {
                const int h = e / a.D, d = e - h * a.D;
                const float* s = s_join + h * D2;
                float mm = kNegInf;
                for (int w = 0; w < waves_b; ++w) mm = fmaxf(mm, s[w * hp * D2]);
                const float z = mm == kNegInf ? 0.0f : mm;
                float x = 0.0f, total = 0.0f;
                for (int w = 0; w < waves_b; ++w) {
                    const float f = weight(s[w * hp * D2] - z);
                    total = fmaf(s[w * hp * D2 + 1], f, total);
                    x = fmaf(s[w * hp * D2 + 2 + d], f, x);
                }
                const int64_t rh = row * a.H + hw + h;
                if (part.parts > 1) {
                    const int64_t prh = (int64_t)blockIdx.z * g.rows * a.H + rh;
                    if (d == 0) {
                        part.ml[2 * prh] = mm;
                        part.ml[2 * prh + 1] = total;
                    }
                    part.acc[prh * a.D + d] = x;
                } else {
                    out[rh * a.D + d] = (T)(total == 0.0f ? 0.0f : x / total);
                    if (lse && d == 0) lse[rh] = total == 0.0f ? kNegInf : mm + log_sum(total);
                }
            }
            __syncthreads();
            return;
        }
        if (!writes) return;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t rh = row * a.H + h0 + r;
            const bool some = sum[r] != 0.0f;
            const float inv = some ? 1.0f / sum[r] : 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) acc[r][w] = some ? acc[r][w] * inv : 0.0f;
            store_channels<T, BUF>(out + rh * a.D + at.chan, at.n, acc[r]);
            if (lse && at.chan == 0) lse[rh] = some ? m[r] + log_sum(sum[r]) : kNegInf;
        }
    });
}

// The parts of a row and head joined by a wave: their maxima and sums a part
// per lane, then a lane per channel.
template <typename T>
__global__ __launch_bounds__(kAtThreads) void k_at_join(Partial part, int64_t rows, Attn a, T* __restrict__ out,
                                                        float* __restrict__ lse) {
    const int lane = lane_id();
    const int64_t all_rh = rows * a.H, waves = (int64_t)gridDim.x * kAtWaves;
    for (int64_t rh = (int64_t)blockIdx.x * kAtWaves + threadIdx.x / kWave; rh < all_rh; rh += waves) {
        const bool mine = lane < part.parts;  // at most kWave parts
        const float pm = mine ? part.ml[2 * (lane * all_rh + rh)] : kNegInf;
        const float ps = mine ? part.ml[2 * (lane * all_rh + rh) + 1] : 0.0f;
        float m = pm;
        for (int h = 1; h < kWave; h <<= 1) m = fmaxf(m, __shfl_xor(m, h, kWave));
        const float f = pm == kNegInf ? 0.0f : weight(pm - m);
        float sum[1] = {ps * f};
        group_sums(sum, kWave);
        for (int d = lane; d < ((a.D + kWave - 1) & -kWave); d += kWave) {
            const float* at = part.acc + rh * a.D + (d < a.D ? d : 0);
            float x = 0.0f;
            for (int p = 0; p < part.parts; p += 8) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = p + i < part.parts ? at[(int64_t)(p + i) * all_rh * a.D] : 0.0f;
#pragma unroll
                for (int i = 0; i < 8; ++i) x = fmaf(v[i], __shfl(f, (p + i) & 63, kWave), x);
            }
            if (d < a.D) out[rh * a.D + d] = (T)(sum[0] == 0.0f ? 0.0f : x / sum[0]);
        }
        if (lse && lane == 0) lse[rh] = sum[0] == 0.0f ? kNegInf : m + log_sum(sum[0]);
    }
}

// Gradient at the centers. With da = ds (1 - t^2) (t the cap's tanh):
//   dq = scale * sum da k = scale * (sum p dp (1 - t^2) k - delta * sum p (1 - t^2) k),
// so that delta = sum p dp may come out only at the end of the one pass over
// the list, in fp32. The weights' sum is 1 but for the rounding of lse, which
// all of a list share; dividing delta by it keeps the sum of a list's ds at 0,
// on which the sums over many lists in the bias's gradient rely.
// stat: what the points need of each row and head.
template <typename T, bool BUF, bool EACH>
__global__ __launch_bounds__(kAtThreads) void k_at_back_c(Groups g, Bias b, Attn a, Lanes l, Walk walk,
                                                          const float* __restrict__ lse, const T* __restrict__ dout,
                                                          T* __restrict__ dq, Stat* __restrict__ stat) {
    constexpr int W = kVec<T>;
    constexpr int U = kUnroll<1>;
    extern __shared__ __align__(16) float s_lds[];
    const Score sc(b, a, s_lds);
    const int lane = lane_id(), wave = threadIdx.x / kWave, waves_b = blockDim.x / kWave;
    const LaneAt at(l, a.H, a.D, W);
    const Rounds<EACH, U> rd(l, at.slot);
    const int hw = (int)blockIdx.y * l.Hc, hn = a.H - hw < l.Hc ? a.H - hw : l.Hc, hl = at.on ? at.head - hw : 0;
    Chunk ck(s_lds + Score::floats(b), Rounds<EACH, U>::rows_n(l), sc, l.Hc);
    const int kvh = at.head / (a.H / a.Hkv);
    const int step = l.Hc * l.G;
    const uint32_t krb = (uint32_t)(a.k_row * (int64_t)sizeof(T)), vrb = (uint32_t)(a.v_row * (int64_t)sizeof(T));
    const uint32_t kbytes = cloud_bytes<T>(g.N, a.k_row, a.Hkv * a.D);
    const uint32_t vbytes = cloud_bytes<T>(g.N, a.v_row, a.Hkv * a.D);

    each_unit(walk.units, waves_b, wave, [&](uint32_t unit) {
        const uint32_t cloud = udiv(unit, walk.by_cloud);
        const uint32_t in = unit - cloud * (uint32_t)walk.per_cloud;
        const int32_t j = EACH ? (int32_t)in * l.S + at.slot : (int32_t)in;
        const bool live_row = !EACH || (j < g.M && at.slot < l.S);
        const int64_t row = (int64_t)cloud * g.M + (live_row ? j : 0);
        const int64_t p0 = (int64_t)cloud * g.N;
        const Rows<T, BUF> kr((const T*)a.k + p0 * a.k_row, a.k_row, kbytes, kvh * a.D + at.chan, at.n);
        const Rows<T, BUF> vr((const T*)a.v + p0 * a.v_row, a.v_row, vbytes, kvh * a.D + at.chan, at.n);
        const int64_t rh = row * a.H + at.head;
        const Raw q = load_channels<T, BUF>((const T*)a.q + row * a.q_row + at.head * a.D + at.chan, at.n);
        const Raw go = load_channels<T, BUF>(dout + rh * a.D + at.chan, at.n);
        float acc[W] = {}, acd[W] = {}, sum = 0.0f, ones = 0.0f;
        const float ls = lse[rh];
        const float z = ls == kNegInf ? __builtin_inff() : ls;  // no weights in an empty group
        float c[3] = {};
        if (sc.placed()) load_xyz(g.centers, row, c);
        int64_t beg, end;
        g.range((int32_t)row, beg, end);
        if (EACH && !live_row) end = beg;
        const int e = EACH ? at.li : lane;
        int32_t next = beg + e < end ? g.idx[beg + e] : -1;  // of the next chunk
        for (int64_t s0 = beg; EACH ? __any(s0 < end) : s0 < end; s0 += rd.chunk) {
            const int n = end - s0 < rd.chunk ? (int)(end - s0) : rd.chunk;
            int32_t mine = next;
            uint32_t u = 0;
            float dist = 0.0f;
            next = s0 + rd.chunk + e < end ? g.idx[s0 + rd.chunk + e] : -1;
            if (e < n) {
                if ((uint32_t)mine >= (uint32_t)g.N) mine = -1;
                if (sc.placed() && mine >= 0) {
                    float p[3];
                    load_xyz(g.points, p0 + mine, p);
                    pair_place(sc.ed, sc.dist, p, c, u, dist);
                }
            }
            if (EACH ? at.slot < l.S : e < rd.chunk)
                ck.put(EACH ? rd.first + e : e, Rows<T, BUF>::key(mine, krb), Rows<T, BUF>::key(mine, vrb), u, dist, sc,
                       hw, hn);
            __builtin_amdgcn_wave_barrier();
            for (int t = 0; EACH ? __any(t < n) : t < n; t += rd.per) {
                Raw k[U], v[U];
                float s[2 * U], bi[U];
                bool there[U];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const float* r0 = ck.row(rd.first + t + i * rd.by);
                    const uint32_t key = ck.field(r0, kKey);
                    there[i] = Rows<T, BUF>::there(key);
                    k[i] = kr.load(key);
                    v[i] = vr.load(ck.field(r0, kKey2));
                    bi[i] = sc.placed() ? r0[hl] : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    s[2 * i] = dot<T>(q, k[i]);
                    s[2 * i + 1] = dot<T>(go, v[i]);
                }
                group_sums(s, l.G);
                float e2[U];
                sc.template products<T, U, 2>(s, e2);
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const float dp = s[2 * i + 1], x = s[2 * i] + bi[i];
                    if (__any(bi[i] == kNegInf)) {  // masked by the bias: whatever k and v hold
                        rare();
                        if (bi[i] == kNegInf) {
                            k[i] = Raw{0, 0, 0, 0};
                            there[i] = false;
                        }
                    }
                    // an entry that is not there: its zeros times a q or dout that is not finite are none
                    const float p = there[i] ? weight(x - z) : 0.0f;
                    const float pdp = there[i] ? p * dp : 0.0f, sl = there[i] ? Score::slack(e2[i]) : 0.0f;
                    sum += pdp;
                    ones += p;
                    add_channels<T>(acc, pdp * sl, k[i]);
                    add_channels<T>(acd, p * sl, k[i]);
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
        if (!EACH) {
            sum = slots_sum(sum, l.S, step, at.slot, lane);
            ones = slots_sum(ones, l.S, step, at.slot, lane);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                acc[w] = slots_sum(acc[w], l.S, step, at.slot, lane);
                acd[w] = slots_sum(acd[w], l.S, step, at.slot, lane);
            }
        }
        if (!(EACH ? at.on && live_row : at.on && at.slot == 0)) return;
        const float delta = ones > 0.0f ? sum / ones : sum;
        const bool far = fabsf(z) > kFarLse;
        const float part = far && ones > 0.0f ? 1.0f / ones : 1.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) acc[w] = a.scale * part * fmaf(-delta, acd[w], acc[w]);
        store_channels<T, BUF>(dq + rh * a.D + at.chan, at.n, acc);
        if (at.chan == 0) stat[rh] = Stat{z, delta, far ? __builtin_amdgcn_logf(part) : 0.0f};
    });
}

// Gradient at the points, over the centers that hold each; and the bias's
// gradient, which a wave sums in a table of its own in LDS, of its pass's heads.
// FLAT: a slot takes P points in a row and walks through their lists as one
// (lists here are a few entries long: a list per slot would leave most of a
// round's rows empty, and the wave would wait for the longest). A round's rows
// are then of any of its points, so that each entry brings its point's k and v
// rows along, which the L1 holds; the sums are written when the point changes.
constexpr int kBackUnroll = 2;

template <typename T, bool BUF, bool FLAT, bool TAB>
__global__ __launch_bounds__(kAtThreads) void k_at_back_p(Groups g, Bias b, Attn a, Lanes l, Walk walk,
                                                          const int64_t* __restrict__ pt_off,
                                                          const int32_t* __restrict__ pt_center, int64_t capacity,
                                                          const Stat* __restrict__ stat, const T* __restrict__ dout,
                                                          T* __restrict__ dk, T* __restrict__ dv,
                                                          float* __restrict__ part) {
    constexpr int W = kVec<T>;
    constexpr int U = kBackUnroll;
    extern __shared__ __align__(16) float s_lds[];
    const Score sc(b, a, s_lds);
    const int lane = lane_id(), wave = threadIdx.x / kWave, waves_b = blockDim.x / kWave;
    const int Rq = a.H / a.Hkv;
    const LaneAt at(l, a.Hkv, a.D, W);
    const Rounds<FLAT, U> rd(l, at.slot);
    const int rows_n = Rounds<FLAT, U>::rows_n(l), hp = l.Hc * Rq, hw = (int)blockIdx.y * hp;
    const int hn = a.H - hw < hp ? a.H - hw : hp;
    Chunk ck(s_lds + Score::floats(b), rows_n, sc, hp);
    const int rows_t = 3 * b.nb + 1, entries = rows_t * hp;  // of a wave's table: this pass's heads
    float* s_tab = s_lds + Score::floats(b) + waves_b * Chunk::floats(sc.placed(), rows_n, hp);
    float* tab = s_tab + wave * entries;
    if constexpr (TAB) {
        for (int e = threadIdx.x; e < entries * waves_b; e += blockDim.x) s_tab[e] = 0.0f;
        __syncthreads();
    }
    const int step = l.Hc * l.G, slot = at.slot < l.S ? at.slot : 0;
    const uint32_t qrb = (uint32_t)(a.q_row * (int64_t)sizeof(T)), orb = (uint32_t)(a.H * a.D * (int)sizeof(T));
    const uint32_t krb = (uint32_t)(a.k_row * (int64_t)sizeof(T)), vrb = (uint32_t)(a.v_row * (int64_t)sizeof(T));
    const uint32_t kbytes = cloud_bytes<T>(g.N, a.k_row, a.Hkv * a.D);
    const uint32_t vbytes = cloud_bytes<T>(g.N, a.v_row, a.Hkv * a.D);
    const uint32_t qbytes = cloud_bytes<T>(g.M, a.q_row, a.H * a.D);
    const uint32_t gbytes = cloud_bytes<T>(g.M, (int64_t)a.H * a.D, a.H * a.D);

    each_unit(walk.units, waves_b, wave, [&](uint32_t unit) {
        const uint32_t cloud = udiv(unit, walk.by_cloud);
        const uint32_t in = unit - cloud * (uint32_t)walk.per_cloud;
        const int64_t p0 = (int64_t)cloud * g.N, c0 = (int64_t)cloud * g.M;
        // the slot's points: n0 of them from i0 on
        int32_t i0 = (int32_t)in, n0 = 1;
        if (FLAT) {
            const int64_t f = ((int64_t)in * l.S + at.slot) * walk.P;
            n0 = at.slot < l.S && f < g.N ? (g.N - f < walk.P ? (int32_t)(g.N - f) : walk.P) : 0;
            i0 = n0 ? (int32_t)f : 0;
        }
        const Rows<T, BUF> qr((const T*)a.q + c0 * a.q_row, a.q_row, qbytes, at.head * Rq * a.D + at.chan, at.n);
        const Rows<T, BUF> gr(dout + c0 * a.H * a.D, (int64_t)a.H * a.D, gbytes, at.head * Rq * a.D + at.chan, at.n);
        const Rows<T, BUF> kr((const T*)a.k + p0 * a.k_row, a.k_row, kbytes, at.head * a.D + at.chan, at.n);
        const Rows<T, BUF> vr((const T*)a.v + p0 * a.v_row, a.v_row, vbytes, at.head * a.D + at.chan, at.n);
        const int64_t kd = (int64_t)a.Hkv * a.D;
        const RowsOut<T, BUF> dkr(dk + p0 * kd, kd, at.head * a.D + at.chan, at.n);
        const RowsOut<T, BUF> dvr(dv + p0 * kd, kd, at.head * a.D + at.chan, at.n);
        const Stat* st0 = stat + c0 * a.H;
        auto clip = [&](int64_t x) { return x < 0 ? 0 : x > capacity ? capacity : x; };
        const int64_t beg = clip(pt_off[p0 + i0]);
        int64_t total = clip(pt_off[p0 + i0 + n0]) - beg;
        if (total < 0) total = 0;
        float gk[W] = {}, gv[W] = {}, gs = 0.0f;  // gs: the slope's, of a lane's one head
        Raw x, y;
        float p3[3] = {};
        int32_t starts = 0, cur = -1;  // FLAT: where the lane's point's list starts; the point the sums are of
        if (FLAT) {
            // points without an entry get zeros
            int64_t f = at.li < n0 ? clip(pt_off[p0 + i0 + at.li]) - beg : total;
            f = f < 0 ? 0 : f > total ? total : f;
            starts = (int32_t)f;
            int32_t next = __shfl(starts, (lane + 1) & 63, kWave);
            if (at.li + 1 >= n0 || at.li + 1 >= step) next = (int32_t)total;
            uint64_t none = __ballot(at.slot < l.S && at.li < n0 && starts >= next) >> (slot * step);
            none &= (1ull << n0) - 1;  // n0 <= kPoints
            while (__any(none != 0)) {
                if (none && at.on) {
                    const int32_t k = __ffsll((unsigned long long)none) - 1;
                    dkr.store(i0 + k, gk);
                    dvr.store(i0 + k, gv);
                }
                none &= none - 1;
            }
        } else {
            x = kr.load(Rows<T, BUF>::key(i0, krb));
            y = vr.load(Rows<T, BUF>::key(i0, vrb));
            if (sc.placed()) load_xyz(g.points, p0 + i0, p3);
        }
        auto write = [&](int32_t k) {
#pragma unroll
            for (int w = 0; w < W; ++w) gk[w] *= a.scale;
            dkr.store(i0 + k, gk);
            dvr.store(i0 + k, gv);
        };
        for (int64_t s0 = 0; FLAT ? __any(s0 < total) : s0 < total; s0 += rd.chunk) {
            const int n = total - s0 < rd.chunk ? (int)(total - s0) : rd.chunk;
            const int e = FLAT ? at.li : lane;
            int32_t mine = -1, k = 0;
            uint32_t u = 0;
            float dist = 0.0f;
            if (FLAT) {  // the last point whose list starts at or before the entry
#pragma unroll
                for (int h = kPoints / 2; h > 0; h >>= 1) {
                    const int32_t st = __shfl(starts, slot * step + (k + h < step ? k + h : 0), kWave);
                    if (k + h < n0 && st <= (int32_t)s0 + e) k += h;
                }
            }
            if (e < n) {
                mine = pt_center[beg + s0 + e];
                if ((uint32_t)mine >= (uint32_t)g.M) mine = -1;
                if (sc.placed() && mine >= 0) {
                    float c[3];
                    load_xyz(g.centers, c0 + mine, c);
                    if (FLAT) load_xyz(g.points, p0 + i0 + k, p3);
                    pair_place(sc.ed, sc.dist, p3, c, u, dist);
                }
            }
            if (FLAT ? at.slot < l.S : e < rd.chunk) {
                const int r = FLAT ? rd.first + e : e;
                ck.put(r, Rows<T, BUF>::key(mine, qrb), Rows<T, BUF>::key(mine, orb), u, dist, sc, hw, hn);
                if (BUF) ck.set(r, kStat, mine < 0 ? 0u : (uint32_t)mine * (uint32_t)a.H);
                if (FLAT) {
                    ck.set(r, kPoint, e < n ? (uint32_t)k : 0xFFFFFFFFu);
                    ck.set(r, kPKey, Rows<T, BUF>::key(i0 + k, krb));
                    ck.set(r, kPKey2, Rows<T, BUF>::key(i0 + k, vrb));
                }
            }
            __builtin_amdgcn_wave_barrier();
            // Entries one after another, the heads that share a key within each (FLAT: an entry's point must not
            // come back once the sums are another's).
            const int all = FLAT ? n * Rq : (n + rd.per - 1) / rd.per * Rq;
            for (int t = 0; FLAT ? __any(t < all) : t < all; t += FLAT ? U : 1) {
                int at_row[U], rr[U];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const int m = FLAT ? t + i : t, en = Rq == 1 ? m : m / Rq;
                    rr[i] = m - en * Rq;
                    at_row[i] = rd.first + (FLAT ? en : en * rd.per + i * rd.by);
                }
                Raw q[U], go[U], kx[U], vx[U];
                float s[2 * U], bi[U], pd[U];
                Stat st[U];
                uint32_t pu[U];
                int32_t pk[U];
                bool there[U];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const int h = at.head * Rq + rr[i];
                    const float* r0 = ck.row(at_row[i]);
                    const uint32_t key = ck.field(r0, kKey), key2 = ck.field(r0, kKey2);
                    there[i] = Rows<T, BUF>::there(key);
                    q[i] = qr.load(key, rr[i] * a.D);
                    go[i] = gr.load(key2, rr[i] * a.D);
                    if constexpr (BUF) st[i] = st0[ck.field(r0, kStat) + (uint32_t)h];
                    else st[i] = st0[(int64_t)(there[i] ? (int32_t)key : 0) * a.H + h];
                    pk[i] = 0;
                    if (FLAT) {
                        pk[i] = (int32_t)ck.field(r0, kPoint);
                        kx[i] = kr.load(ck.field(r0, kPKey));
                        vx[i] = vr.load(ck.field(r0, kPKey2));
                    } else {
                        kx[i] = x;
                        vx[i] = y;
                    }
                    bi[i] = sc.placed() ? r0[at.on ? h - hw : 0] : 0.0f;
                    pu[i] = ck.field(r0, kPlace);
                    pd[i] = r0[ck.hp + kDist];
                }
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    s[2 * i] = dot<T>(q[i], kx[i]);
                    s[2 * i + 1] = dot<T>(go[i], vx[i]);
                }
                group_sums(s, l.G);
                float e2[U];
                sc.template products<T, U, 2>(s, e2);
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const float dp = s[2 * i + 1], v = s[2 * i] + bi[i];
                    if (__any(bi[i] == kNegInf)) {
                        rare();
                        if (bi[i] == kNegInf) {
                            q[i] = go[i] = Raw{0, 0, 0, 0};
                            there[i] = false;  // nor lse, delta and a distance that overflows
                        }
                    }
                    const float p = there[i] ? weight(v - st[i].z, st[i].log_part) : 0.0f;
                    const float ds = there[i] ? p * (dp - st[i].delta) : 0.0f;
                    const float da = there[i] ? ds * Score::slack(e2[i]) : 0.0f;
                    if (FLAT) {
                        const bool change = pk[i] >= 0 && pk[i] != cur;
                        if (__any(change)) {
                            if (change) {
                                if (cur >= 0) write(cur);
#pragma unroll
                                for (int w = 0; w < W; ++w) gk[w] = gv[w] = 0.0f;
                                cur = pk[i];
                            }
                        }
                    }
                    add_channels<T>(gk, da, q[i]);
                    add_channels<T>(gv, p, go[i]);
                    if constexpr (TAB) {
                        if (at.chan == 0 && there[i] && at.on) {
                            const int h = at.head * Rq + rr[i] - hw;
                            if (b.nb > 0) {
                                lds_add(&tab[__umul24(pu[i] & 255u, (uint32_t)hp) + h], ds);
                                lds_add(&tab[__umul24(b.nb + (pu[i] >> 8 & 255u), (uint32_t)hp) + h], ds);
                                lds_add(&tab[__umul24(2 * b.nb + (pu[i] >> 16), (uint32_t)hp) + h], ds);
                            }
                            if (Rq == 1) gs = fmaf(ds, pd[i], gs);
                            else if (b.slope) lds_add(&tab[3 * b.nb * hp + h], ds * pd[i]);
                        }
                    }
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
        if constexpr (TAB) {
            if (Rq == 1 && b.slope && at.chan == 0 && at.on) lds_add(&tab[3 * b.nb * hp + at.head - hw], gs);
        }
        if (!FLAT) {
#pragma unroll
            for (int w = 0; w < W; ++w) {
                gk[w] = slots_sum(gk[w], l.S, step, at.slot, lane);
                gv[w] = slots_sum(gv[w], l.S, step, at.slot, lane);
            }
            if (at.on && at.slot == 0) write(0);
        } else if (at.on && cur >= 0) {
            write(cur);
        }
    });
    if constexpr (TAB) {
        __syncthreads();
        for (int e = threadIdx.x; e < rows_t * hn; e += blockDim.x) {
            const int r = e / hn, h = e - r * hn;
            float x = 0.0f;
            for (int w = 0; w < waves_b; ++w) x += s_tab[w * entries + r * hp + h];
            part[((int64_t)blockIdx.x * rows_t + r) * a.H + hw + h] = x;
        }
    }
}

// ------------------------------------------------------------------ host side

size_t stat_bytes(int64_t rh) { return ((size_t)rh * sizeof(Stat) + 255) & ~(size_t)255; }

// Whether every slot of a wave takes a list of its own: lists short, and the
// shorter the fewer of them that takes. (Mean lengths of 5 and 8, 5870 and 4542
// lists: 37 -> 14 and 19 -> 9 us forward; 1, 80 lists: 11 -> 7. Otherwise a wave's
// slots share a list: 470 ragged ones of 4 on the average 18 us against 30 with
// one each, 1024 x 8 of 20 in 4 slots with gradients 200 against 207.)
bool each_of(int64_t rows, int64_t slots, const Lanes& l) {
    if (l.S == 1) return true;
    const int64_t units = rows / l.S;
    return slots <= 2 * rows || (slots <= 8 * rows && units >= 64) || (slots <= 32 * rows && units >= 4096);
}

// The launch of a kernel: waves of a workgroup, such that what they keep in
// LDS fits, and LDS bytes.
struct Shape {
    int waves;
    size_t lds;
};

Shape shape_of(const Bias& b, size_t floats_per_wave) {
    const size_t base = (size_t)Score::floats(b) * 4;
    Shape r;
    r.waves = kAtWaves;
    while (r.waves > 1 && base + floats_per_wave * 4 * r.waves > kAtLds) r.waves >>= 1;
    r.lds = base + floats_per_wave * 4 * r.waves;
    return r;
}

bool placed(const Bias& b) { return b.nb > 0 || b.slope; }

// A workgroup to a list whose mean length gives each wave a chunk, where there
// are not lists enough to fill the card with a wave each; parts where there
// are few.
constexpr int kSplitRows = 4096;
struct Split {
    bool block;
    int32_t parts;
};

Split split_of(const Groups& g, int32_t HD) {
    Split s = {false, 1};
    const int64_t mean = g.idx_len / g.rows;  // of ragged lists only their mean is known here
    if (mean < 2 * kWave || HD > kJoinFloats || g.rows >= kSplitRows) return s;
    s.block = true;
    int64_t p = 1024 / g.rows;
    if (p > mean / kWave) p = mean / kWave;  // 16 entries to a wave
    s.parts = (int32_t)(p < 1 ? 1 : p > kWave ? kWave : p);
    return s;
}

template <typename T>
bool vectors(const Groups& g, const Attn& a, std::initializer_list<const void*> ptrs) {
    constexpr int W = kVec<T>;
    if (a.D % W || a.q_row % W || a.k_row % W || a.v_row % W) return false;
    for (const void* p : ptrs)
        if ((uintptr_t)p & 15) return false;
    // a cloud's rows in one buffer
    const int64_t most = (int64_t)kMostBytes / (int64_t)sizeof(T);
    const int64_t qd = (int64_t)a.H * a.D;
    return a.k_row <= most / g.N && a.v_row <= most / g.N && a.q_row <= most / g.M && qd <= most / g.M;
}

// Query heads per lane: those that share a key's head, while the pass's heads
// stay few (their biases of a chunk are in LDS).
template <typename T>
int heads_per_lane(const Attn& a) {
    const int r = a.H / a.Hkv;
    for (int R : {4, 2})
        if (r % R == 0 && make_lanes<T>(a.H / R, a.D).Hc * R <= 64) return R;
    return 1;
}

uint32_t blocks_of(int64_t units, int64_t per, int64_t most) {
    const int64_t n = (units + per - 1) / per;
    return (uint32_t)(n > most ? most : n < 8 ? 8 : (n + 7) & ~7ll);
}

template <typename K>
hipError_t allow_lds(K kern, size_t bytes) {
    if (bytes <= (48 << 10)) return hipSuccess;
    return hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <typename T, bool BUF, int R, bool EACH, bool BLOCK>
hipError_t forward_with(const Groups& g, int32_t B, const Attn& a, const Bias& b, const Lanes& l, const Partial& part,
                        void* out, float* lse, hipStream_t s) {
    const Walk w = make_walk(B, g.M, EACH ? l.S : 1, 1);
    size_t floats = Chunk::floats(placed(b), Rounds<EACH, kUnroll<R>>::rows_n(l), l.Hc * R);
    if (BLOCK) floats += (size_t)l.Hc * R * (a.D + 2);
    const Shape sh = shape_of(b, floats);
    auto kern = k_at<T, BUF, R, EACH, BLOCK>;
    hipError_t e = allow_lds(kern, sh.lds);
    if (e != hipSuccess) return e;
    const uint32_t blocks = blocks_of(w.units, BLOCK ? 1 : sh.waves, EACH ? kAtBlocks : kAtMany);
    kern<<<dim3(blocks, l.passes, part.parts), sh.waves * kWave, sh.lds, s>>>(
        g, b, a, l, w, (T*)out, lse, part);
    if (part.parts > 1) {
        const int64_t n = (int64_t)g.rows * a.H;
        k_at_join<T><<<blocks_of(n, kAtWaves, kAtMany), kAtThreads, 0, s>>>(part, g.rows, a, (T*)out, lse);
    }
    return hipGetLastError();
}

template <typename T, bool BUF, int R>
hipError_t forward_as(const Groups& g, int32_t B, const Attn& a, const Bias& b, void* out, float* lse, void* ws,
                      hipStream_t s) {
    const Lanes l = make_lanes<T>(a.H / R, a.D);
    const Split sp = split_of(g, a.H * a.D);
    Partial part = {nullptr, nullptr, sp.parts};
    if (part.parts > 1) {
        part.ml = (float*)ws;
        part.acc = part.ml + (size_t)part.parts * g.rows * a.H * 2;
    }
    auto f = sp.block ? forward_with<T, BUF, R, false, true>
             : each_of(g.rows, g.idx_len, l) ? forward_with<T, BUF, R, true, false>
                                             : forward_with<T, BUF, R, false, false>;
    return f(g, B, a, b, l, part, out, lse, s);
}

template <typename T>
hipError_t forward(const Groups& g, int32_t B, const Attn& a, const Bias& b, void* out, float* lse, void* ws,
                   hipStream_t s) {
    const bool buf = vectors<T>(g, a, {a.q, a.k, a.v, out});
    const int r = heads_per_lane<T>(a);
    auto f = buf ? (r == 4 ? forward_as<T, true, 4> : r == 2 ? forward_as<T, true, 2> : forward_as<T, true, 1>)
                 : forward_as<T, false, 1>;
    return f(g, B, a, b, out, lse, ws, s);
}

template <typename T, bool BUF, bool EACH>
hipError_t back_centers(const Groups& g, int32_t B, const Attn& a, const Bias& b, const Lanes& l, const float* lse,
                        const void* dout, void* dq, Stat* stat, hipStream_t s) {
    const Walk w = make_walk(B, g.M, EACH ? l.S : 1, 1);
    const Shape sh = shape_of(b, Chunk::floats(placed(b), Rounds<EACH, kUnroll<1>>::rows_n(l), l.Hc));
    auto kern = k_at_back_c<T, BUF, EACH>;
    hipError_t e = allow_lds(kern, sh.lds);
    if (e != hipSuccess) return e;
    kern<<<dim3(blocks_of(w.units, sh.waves, EACH ? kAtBlocks : kAtMany), l.passes), sh.waves * kWave, sh.lds, s>>>(
        g, b, a, l, w, lse, (const T*)dout, (T*)dq, stat);
    return hipGetLastError();
}

// Whether a slot walks lists at the points as one, rather than a wave one list
// after another: while a list does not fill a wave's round, or its rounds are
// few beside what a wave does once a list. (61341 points with 136 slots 165 -> 28 us,
// 28264 with 27180 137 -> 44, indoor scenes with gradients, 3 slots a point,
// 818 -> 369; 23 slots a point in 2 slots 54 -> 49. On the other side 27 slots a
// point, three query heads to a key's, 4 slots: 340 as lists, 573 as one, in
// which a wave waits for the longest.)
bool flat_of(int64_t points, int64_t slots, const Attn& a, const Lanes& l) {
    return slots < points * 2 * l.S || slots * (a.H / a.Hkv) < points * 32;
}

// The launch of the gradient at the points. Points are walked in a row by a
// slot where the places fit 32 bits; several of them where there are enough
// for more than two rounds of the card's waves. Fewer slots where one wave's
// chunk and table of the bias's gradient take more LDS than a CU has (128 heads
// of at most 16 bytes that share one key's, 64 buckets: 168 KB with 64 slots).
struct BackShape {
    bool flat;
    Lanes l;
    Walk walk;
    Shape sh;
    uint32_t blocks;
};

BackShape back_shape(const Groups& g, int32_t B, const Attn& a, const Bias& b, Lanes l, bool tab) {
    BackShape r;
    const int64_t points = (int64_t)B * g.N;
    r.flat = g.idx_len < (1ll << 31) && flat_of(points, g.idx_len, a, l);
    for (;; l.S >>= 1) {
        const int rows = r.flat ? Rounds<true, kBackUnroll>::rows_n(l) : Rounds<false, kBackUnroll>::rows_n(l);
        size_t floats = Chunk::floats(placed(b), rows, l.Hc * (a.H / a.Hkv));
        if (tab) floats += (size_t)(3 * b.nb + 1) * l.Hc * (a.H / a.Hkv);
        r.sh = shape_of(b, floats);
        if (r.sh.lds <= kCuLds || l.S == 1) break;
    }
    r.l = l;
    const int32_t step = l.Hc * l.G, most = step < kPoints ? step : kPoints;
    const int64_t P = points / ((int64_t)l.S * 8192);
    r.walk = r.flat ? make_walk(B, g.N, l.S, (int32_t)(P < 1 ? 1 : P > most ? most : P)) : make_walk(B, g.N, 1, 1);
    r.blocks = blocks_of(r.walk.units, r.sh.waves, r.flat || tab ? kAtBlocks : kAtMany);
    return r;
}

template <typename T, bool BUF>
auto points_kernel(bool flat, bool tab) {
    return flat ? (tab ? k_at_back_p<T, BUF, true, true> : k_at_back_p<T, BUF, true, false>)
                : (tab ? k_at_back_p<T, BUF, false, true> : k_at_back_p<T, BUF, false, false>);
}

template <typename T>
hipError_t backward(const Groups& g, int32_t B, const Attn& a, const Bias& b, const int64_t* pt_off,
                    const int32_t* pt_center, int64_t capacity, const float* lse, const void* dout, void* dq, void* dk,
                    void* dv, float* dtable, float* dslope, void* ws, hipStream_t s) {
    const Lanes lc = make_lanes<T>(a.H, a.D);
    const int64_t rh = (int64_t)g.rows * a.H;
    Stat* stat = (Stat*)ws;
    float* part = (float*)((char*)ws + stat_bytes(rh));
    const bool buf = vectors<T>(g, a, {a.q, a.k, a.v, dout, dq, dk, dv});
    const bool ec = each_of(g.rows, g.idx_len, lc), tab = dtable || dslope;
    // what can fail, before anything is enqueued
    const BackShape r = back_shape(g, B, a, b, make_lanes<T>(a.Hkv, a.D), tab);
    auto points = buf ? points_kernel<T, true>(r.flat, tab) : points_kernel<T, false>(r.flat, tab);
    hipError_t e = allow_lds(points, r.sh.lds);
    if (e != hipSuccess) return e;
    auto centers = buf ? (ec ? back_centers<T, true, true> : back_centers<T, true, false>)
                       : (ec ? back_centers<T, false, true> : back_centers<T, false, false>);
    e = centers(g, B, a, b, lc, lse, dout, dq, stat, s);
    if (e != hipSuccess) return e;
    points<<<dim3(r.blocks, r.l.passes), r.sh.waves * kWave, r.sh.lds, s>>>(
        g, b, a, r.l, r.walk, pt_off, pt_center, capacity, stat, (const T*)dout, (T*)dk, (T*)dv, part);
    e = hipGetLastError();
    if (e != hipSuccess || !tab) return e;
    return launch_bias_reduce(part, (int32_t)r.blocks, b, dtable, dslope, s);
}

Lanes lanes_of(int32_t dtype, int32_t heads, int32_t D) {
    return dtype == CAGQ_F32 ? make_lanes<float>(heads, D) : make_lanes<bf16>(heads, D);
}

}  // namespace

size_t group_attention_bytes(const Groups& g, int32_t B, const Attn& a, int32_t dtype, const Bias& b, bool backward) {
    if (!backward) {
        const Split sp = split_of(g, a.H * a.D);
        return sp.parts > 1 ? (size_t)sp.parts * g.rows * a.H * (2 + a.D) * 4 : 0;
    }
    const size_t stat = stat_bytes((int64_t)g.rows * a.H);
    if (!placed(b)) return stat;
    const Lanes l = lanes_of(dtype, a.Hkv, a.D);
    const BackShape r = back_shape(g, B, a, b, l, true);
    return stat + (size_t)r.blocks * (3 * b.nb + 1) * b.H * 4;
}

hipError_t launch_group_attention(const Groups& g, int32_t B, const Attn& a, int32_t dtype, const Bias& b, void* out,
                                  float* lse, void* ws, hipStream_t s) {
    auto f = dtype == CAGQ_F32 ? forward<float> : dtype == CAGQ_BF16 ? forward<bf16> : forward<f16>;
    return f(g, B, a, b, out, lse, ws, s);
}

hipError_t launch_group_attention_backward(const Groups& g, int32_t B, const Attn& a, int32_t dtype, const Bias& b,
                                           const int64_t* pt_off, const int32_t* pt_center, int64_t capacity,
                                           const float* lse, const void* dout, void* dq, void* dk, void* dv,
                                           float* dtable, float* dslope, void* ws, hipStream_t s) {
    auto f = dtype == CAGQ_F32 ? backward<float> : dtype == CAGQ_BF16 ? backward<bf16> : backward<f16>;
    return f(g, B, a, b, pt_off, pt_center, capacity, lse, dout, dq, dk, dv, dtable, dslope, ws, s);
}

}  // namespace cagq
