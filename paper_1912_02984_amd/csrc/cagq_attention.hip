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
//   - a list's indices, offsets and places in the bias are made a chunk at a
//     time, one entry per lane, and handed to the rows' lanes by permutes;
//   - kUnroll rows of each slot are loaded before the first is used. Loads go
//     through a bounds-checked buffer, in which an entry that is not there has
//     an offset past the end and reads as zeros, without a branch;
//   - two ways to share a wave: EACH, a list per slot (many short lists: no
//     slot waits for another list's end, nothing is joined), or one list for
//     all slots, joined by permutes at its end.
// Scores stay in natural units (times log2 e, a bias of the type's lowest
// value would become -infinity), and only differences of them are taken to
// base 2.
//
// The gradients take two passes: at the centers (dq, and delta = sum p dp) and
// at the points (dk, dv and the bias's), each recomputing the scores: that
// reads two rows a pair, as storing and fetching weights for every pair and
// head would need memory for them all.
#include <initializer_list>
#include <type_traits>

#include "cagq_features.h"

namespace cagq {

namespace {

constexpr int kAtThreads = 256;
constexpr int kAtWaves = kAtThreads / kWave;
constexpr int kAtBlocks = 256 * 8;   // workgroups of a launch; they go round where there is more to do
constexpr int kAtParts = 1024;       // workgroups of the gradient at the points, where the bias wants its own
constexpr int kAtLds = 144 << 10;    // LDS of a workgroup: edges, table, and the waves' gradient tables
constexpr int kJoinFloats = 2048;    // H * D up to which a workgroup's waves join their parts in LDS
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

// The rows of one cloud. BUF: a buffer of less than 2^31 bytes, rows aligned
// to 16 bytes; an offset of kNone is past its end whatever is added to it.
// Otherwise pointers, element by element.
constexpr uint32_t kNone = 0x80000000u;

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
            lane_off = n_ > 0 ? (uint32_t)lane_elem * (uint32_t)sizeof(T) : kNone;
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
    __device__ __forceinline__ Raw load(uint32_t key) const {
        if constexpr (BUF) return __builtin_amdgcn_raw_buffer_load_b128(rsrc, key + lane_off, 0, 0);
        else return load_channels<T, false>(base + (int64_t)(int32_t)key * row, (int32_t)key >= 0 ? n : 0);
    }
    static __device__ __forceinline__ bool there(uint32_t key) { return (int32_t)key >= 0; }
};

// What all kernels know of the scores.
struct Score {
    Edges ed;
    const float* table;  // LDS, [3][nb][H]
    int nb, H;
    bool dist;
    float mul;   // of a product: scale, or with a cap 2 log2 e scale / cap
    float cap;

    // Floats of LDS before the kernel's own.
    static __host__ __device__ int floats(const Bias& b) { return 3 * edges_size(b.nb) + 3 * b.nb * b.H; }

    // Every thread of the block; ends with a barrier.
    __device__ __forceinline__ Score(const Bias& b, const Attn& a, float* lds) {
        ed = stage_edges(b, lds);
        float* t = lds + 3 * ed.size;
        for (int e = threadIdx.x; e < 3 * b.nb * b.H; e += blockDim.x) t[e] = b.table[e];
        table = t;
        nb = b.nb;
        H = b.H;
        dist = b.slope != nullptr;
        cap = a.cap;
        mul = cap > 0.0f ? 2.0f * kLog2e * a.scale / cap : a.scale;
        __syncthreads();
    }
    __device__ __forceinline__ bool placed() const { return nb > 0 || dist; }

    // cap * tanh(scale * x / cap) as cap - 2 cap / (1 + exp(2 scale x / cap)):
    // off by some 2^-24 of the cap, not of x, which is what differences of
    // scores call for. `e`: 1 / (1 + exp), of which the tanh's slope is
    // 4 e (1 - e).
    __device__ __forceinline__ float product(float x, float& e) const {
        if (cap > 0.0f) {
            e = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * mul));
            return fmaf(-2.0f * cap, e, cap);
        }
        return x * mul;
    }
    // 1 - tanh^2
    __device__ __forceinline__ float slack(float e) const { return cap > 0.0f ? 4.0f * e * (1.0f - e) : 1.0f; }
    __device__ __forceinline__ float bias(int h, uint32_t u, float slope, float d) const {
        return bias_at(table, nb, H, slope, h, u, d);
    }
};

// exp(x) of a difference of scores.
__device__ __forceinline__ float weight(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// log of a sum of weights.
__device__ __forceinline__ float log_sum(float x) { return kLn2 * __builtin_amdgcn_logf(x); }

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

// Which lists the waves take. Units (a row, or S rows of a cloud with EACH)
// are laid out so that an XCD's workgroups walk through one range of them side
// by side: groups near each other share points, and share the XCD's L2.
struct Walk {
    int64_t units;     // per launch
    int32_t per_cloud; // EACH: units per cloud
    Magic by_cloud;
};

template <bool EACH>
Walk make_walk(int32_t B, int32_t rows_per_cloud, const Lanes& l) {
    Walk w;
    w.per_cloud = EACH ? (rows_per_cloud + l.S - 1) / l.S : rows_per_cloud;
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

// Partial softmax of a part of a list: maximum and sum, and the weighted sum's
// D channels, per row and head.
struct Partial {
    float* ml;   // [parts][rows][H][2]
    float* acc;  // [parts][rows][H][D]
    int32_t parts;
};

// R: query heads a lane holds (they share the key's head).
template <typename T, bool BUF, int R, bool EACH, bool BLOCK>
__global__ __launch_bounds__(kAtThreads) void k_at(Groups g, Bias b, Attn a, Lanes l, Walk walk, T* __restrict__ out,
                                                   float* __restrict__ lse, Partial part) {
    constexpr int W = kVec<T>;
    constexpr int U = R == 4 ? 2 : 4;
    extern __shared__ float s_lds[];
    const Score sc(b, a, s_lds);
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const LaneAt at(l, a.H / R, a.D, W);
    const int h0 = at.head * R;
    const int kvh = h0 / (a.H / a.Hkv);
    const int step = l.Hc * l.G;
    const uint32_t krb = (uint32_t)(a.k_row * (int64_t)sizeof(T)), vrb = (uint32_t)(a.v_row * (int64_t)sizeof(T));
    const bool same = krb == vrb;
    float slope[R];
#pragma unroll
    for (int r = 0; r < R; ++r) slope[r] = b.slope && at.on ? b.slope[h0 + r] : 0.0f;

    each_unit(walk.units, BLOCK ? 1 : kAtWaves, BLOCK ? 0 : wave, [&](uint32_t unit) {
        const uint32_t cloud = udiv(unit, walk.by_cloud);
        const uint32_t in = unit - cloud * (uint32_t)walk.per_cloud;
        const int32_t j = EACH ? (int32_t)in * l.S + at.slot : (int32_t)in;
        const bool live_row = !EACH || (j < g.M && at.slot < l.S);
        const int64_t row = (int64_t)cloud * g.M + (live_row ? j : 0);
        const int64_t p0 = (int64_t)cloud * g.N;
        const Rows<T, BUF> kr((const T*)a.k + p0 * a.k_row, a.k_row, (uint32_t)((g.N - 1) * (int64_t)krb) +
                              (uint32_t)(a.Hkv * a.D * (int)sizeof(T)), kvh * a.D + at.chan, at.n);
        const Rows<T, BUF> vr((const T*)a.v + p0 * a.v_row, a.v_row, (uint32_t)((g.N - 1) * (int64_t)vrb) +
                              (uint32_t)(a.Hkv * a.D * (int)sizeof(T)), kvh * a.D + at.chan, at.n);
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
        const int split = BLOCK ? kAtWaves * part.parts : part.parts;
        if (!EACH && split > 1) {
            const int64_t per = (end - beg + split - 1) / split;
            beg += (BLOCK ? (int64_t)blockIdx.z * kAtWaves + wave : (int64_t)blockIdx.z) * per;
            end = end < beg + per ? end : beg + per;
        }
        const int ch = EACH ? step : kWave;  // entries of a chunk
        const int first = EACH ? at.slot * step : at.slot;
        for (int64_t s0 = beg; EACH ? __any(s0 < end) : s0 < end; s0 += ch) {
            const int n = end - s0 < ch ? (int)(end - s0) : ch;
            int32_t mine = -1;
            uint32_t u = 0;
            float dist = 0.0f;
            const int e = EACH ? at.li : lane;
            if (e < n) {
                mine = g.idx[s0 + e];
                if ((uint32_t)mine >= (uint32_t)g.N) mine = -1;
                if (sc.placed() && mine >= 0) {
                    float p[3];
                    load_xyz(g.points, p0 + mine, p);
                    pair_place(sc.ed, sc.dist, p, c, u, dist);
                }
            }
            const uint32_t kkey = Rows<T, BUF>::key(mine, krb), vkey = Rows<T, BUF>::key(mine, vrb);
            for (int t = 0; EACH ? __any(t < n) : t < n; t += EACH ? U : U * l.S) {
                Raw k[U], v[U];
                uint32_t pu[U];
                float pd[U], s[U * R];
                bool there[U];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const int from = EACH ? t + i : t + i * l.S + at.slot;
                    const int src = (EACH ? first + from : from) & 63;
                    uint32_t key = (uint32_t)__shfl((int)kkey, src, kWave);
                    if (from >= n) key = 0xFFFFFFFFu & (BUF ? kNone : 0xFFFFFFFFu);
                    there[i] = Rows<T, BUF>::there(key);
                    k[i] = kr.load(key);
                    if (!BUF || same) {
                        v[i] = vr.load(key);
                    } else {
                        const uint32_t key2 = (uint32_t)__shfl((int)vkey, src, kWave);
                        v[i] = vr.load(there[i] ? key2 : kNone);
                    }
                    if (sc.nb > 0) pu[i] = (uint32_t)__shfl((int)u, src, kWave);
                    else pu[i] = 0;
                    pd[i] = sc.dist ? __shfl(dist, src, kWave) : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < U; ++i)
#pragma unroll
                    for (int r = 0; r < R; ++r) s[i * R + r] = dot<T>(q[r], k[i]);
                group_sums(s, l.G);
#pragma unroll
                for (int i = 0; i < U; ++i) {
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        float e2;
                        float x = sc.product(s[i * R + r], e2);
                        if (sc.placed()) {
                            const float bi = sc.bias(h0 + r, pu[i], slope[r], pd[i]);
                            x = bi == kNegInf ? kNegInf : x + bi;
                            if (R == 1 && __any(bi == kNegInf)) {  // masked by the bias: whatever v holds
                                if (bi == kNegInf) v[i] = Raw{0, 0, 0, 0};
                            }
                        }
                        s[i * R + r] = there[i] ? x : kNegInf;
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
                            add_channels<T>(acc[r], p, v[i]);
                        } else {
                            // heads of their own biases share v: a masked one passes it over
                            const bool off = s[i * R + r] == kNegInf;
#pragma unroll
                            for (int w = 0; w < W; ++w)
                                acc[r][w] = fmaf(p, off ? 0.0f : channel<T>(v[i], w), acc[r][w]);
                        }
                    }
                }
            }
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
            const int D2 = a.D + 2, hp = l.Hc * R;
            float* s_join = s_lds + Score::floats(b);
            if (writes) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float* d = s_join + (wave * hp + h0 - (int)blockIdx.y * hp + r) * D2;
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
            const int hq = a.H - (int)blockIdx.y * hp < hp ? a.H - (int)blockIdx.y * hp : hp;
            for (int e = threadIdx.x; e < hq * a.D; e += kAtThreads) {
                const int h = e / a.D, d = e - h * a.D;
                const float* s = s_join + h * D2;
                float mm = kNegInf;
#pragma unroll
                for (int w = 0; w < kAtWaves; ++w) mm = fmaxf(mm, s[w * hp * D2]);
                const float z = mm == kNegInf ? 0.0f : mm;
                float x = 0.0f, total = 0.0f;
#pragma unroll
                for (int w = 0; w < kAtWaves; ++w) {
                    const float f = weight(s[w * hp * D2] - z);
                    total = fmaf(s[w * hp * D2 + 1], f, total);
                    x = fmaf(s[w * hp * D2 + 2 + d], f, x);
                }
                const int64_t rh = row * a.H + (int)blockIdx.y * hp + h;
                if (part.parts > 1) {
                    const int64_t prh = (int64_t)blockIdx.z * g.rows * a.H + rh;
                    if (d == 0) {
                        part.ml[2 * prh] = mm;
                        part.ml[2 * prh + 1] = total;
                    }
                    part.acc[prh * a.D + d] = x;
                } else {
                    out[rh * a.D + d] = (T)(total == 0.0f ? 0.0f : x / total);
                    if (lse && d == 0)
                        lse[rh] = total == 0.0f ? kNegInf : mm + log_sum(total);
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
            float x = 0.0f;
            for (int p = 0; p < part.parts; ++p) {
                const float fp = __shfl(f, p, kWave);
                if (d < a.D && fp > 0.0f) x = fmaf(part.acc[(p * all_rh + rh) * a.D + d], fp, x);
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
// stat: (lse, delta) of each row and head, for the points.
template <typename T, bool BUF, bool EACH>
__global__ __launch_bounds__(kAtThreads) void k_at_back_c(Groups g, Bias b, Attn a, Lanes l, Walk walk,
                                                          const float* __restrict__ lse, const T* __restrict__ dout,
                                                          T* __restrict__ dq, float2* __restrict__ stat) {
    constexpr int W = kVec<T>;
    constexpr int U = 4;
    extern __shared__ float s_lds[];
    const Score sc(b, a, s_lds);
    const int lane = lane_id(), wave = threadIdx.x / kWave;
    const LaneAt at(l, a.H, a.D, W);
    const int kvh = at.head / (a.H / a.Hkv);
    const int step = l.Hc * l.G;
    const uint32_t krb = (uint32_t)(a.k_row * (int64_t)sizeof(T)), vrb = (uint32_t)(a.v_row * (int64_t)sizeof(T));
    const bool same = krb == vrb;
    const float slope = b.slope && at.on ? b.slope[at.head] : 0.0f;

    each_unit(walk.units, kAtWaves, wave, [&](uint32_t unit) {
        const uint32_t cloud = udiv(unit, walk.by_cloud);
        const uint32_t in = unit - cloud * (uint32_t)walk.per_cloud;
        const int32_t j = EACH ? (int32_t)in * l.S + at.slot : (int32_t)in;
        const bool live_row = !EACH || (j < g.M && at.slot < l.S);
        const int64_t row = (int64_t)cloud * g.M + (live_row ? j : 0);
        const int64_t p0 = (int64_t)cloud * g.N;
        const Rows<T, BUF> kr((const T*)a.k + p0 * a.k_row, a.k_row, (uint32_t)((g.N - 1) * (int64_t)krb) +
                              (uint32_t)(a.Hkv * a.D * (int)sizeof(T)), kvh * a.D + at.chan, at.n);
        const Rows<T, BUF> vr((const T*)a.v + p0 * a.v_row, a.v_row, (uint32_t)((g.N - 1) * (int64_t)vrb) +
                              (uint32_t)(a.Hkv * a.D * (int)sizeof(T)), kvh * a.D + at.chan, at.n);
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
        const int ch = EACH ? step : kWave;
        const int first = EACH ? at.slot * step : at.slot;
        for (int64_t s0 = beg; EACH ? __any(s0 < end) : s0 < end; s0 += ch) {
            const int n = end - s0 < ch ? (int)(end - s0) : ch;
            int32_t mine = -1;
            uint32_t u = 0;
            float dist = 0.0f;
            const int e = EACH ? at.li : lane;
            if (e < n) {
                mine = g.idx[s0 + e];
                if ((uint32_t)mine >= (uint32_t)g.N) mine = -1;
                if (sc.placed() && mine >= 0) {
                    float p[3];
                    load_xyz(g.points, p0 + mine, p);
                    pair_place(sc.ed, sc.dist, p, c, u, dist);
                }
            }
            const uint32_t kkey = Rows<T, BUF>::key(mine, krb), vkey = Rows<T, BUF>::key(mine, vrb);
            for (int t = 0; EACH ? __any(t < n) : t < n; t += EACH ? U : U * l.S) {
                Raw k[U], v[U];
                uint32_t pu[U];
                float pd[U], s[2 * U];
                bool there[U];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    const int from = EACH ? t + i : t + i * l.S + at.slot;
                    const int src = (EACH ? first + from : from) & 63;
                    uint32_t key = (uint32_t)__shfl((int)kkey, src, kWave);
                    if (from >= n) key = BUF ? kNone : 0xFFFFFFFFu;
                    there[i] = Rows<T, BUF>::there(key);
                    k[i] = kr.load(key);
                    if (!BUF || same) {
                        v[i] = vr.load(key);
                    } else {
                        const uint32_t key2 = (uint32_t)__shfl((int)vkey, src, kWave);
                        v[i] = vr.load(there[i] ? key2 : kNone);
                    }
                    if (sc.nb > 0) pu[i] = (uint32_t)__shfl((int)u, src, kWave);
                    else pu[i] = 0;
                    pd[i] = sc.dist ? __shfl(dist, src, kWave) : 0.0f;
                }
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    s[2 * i] = dot<T>(q, k[i]);
                    s[2 * i + 1] = dot<T>(go, v[i]);
                }
                group_sums(s, l.G);
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    float e2 = 0.0f, dp = s[2 * i + 1];
                    float x = sc.product(s[2 * i], e2);
                    if (sc.placed()) {
                        const float bi = sc.bias(at.head, pu[i], slope, pd[i]);
                        x += bi;
                        if (__any(bi == kNegInf)) {  // masked by the bias: whatever k and v hold
                            if (bi == kNegInf) {
                                k[i] = Raw{0, 0, 0, 0};
                                x = kNegInf;
                                dp = 0.0f;
                            }
                        }
                    }
                    const float p = there[i] ? weight(x - z) : 0.0f;
                    const float pdp = p * dp, sl = sc.slack(e2);
                    sum += pdp;
                    ones += p;
                    add_channels<T>(acc, pdp * sl, k[i]);
                    add_channels<T>(acd, p * sl, k[i]);
                }
            }
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
#pragma unroll
        for (int w = 0; w < W; ++w) acc[w] = a.scale * fmaf(-delta, acd[w], acc[w]);
        store_channels<T, BUF>(dq + rh * a.D + at.chan, at.n, acc);
        if (at.chan == 0) stat[rh] = make_float2(z, delta);
    });
}

// Gradient at the points, over the centers that hold each; and the bias's
// gradient, which a wave sums in a table of its own in LDS.
template <typename T, bool BUF, bool EACH, bool TAB>
__global__ __launch_bounds__(kAtThreads) void k_at_back_p(Groups g, Bias b, Attn a, Lanes l, Walk walk,
                                                          const int64_t* __restrict__ pt_off,
                                                          const int32_t* __restrict__ pt_center, int64_t capacity,
                                                          const float2* __restrict__ stat, const T* __restrict__ dout,
                                                          T* __restrict__ dk, T* __restrict__ dv,
                                                          float* __restrict__ part) {
    constexpr int W = kVec<T>;
    constexpr int U = 4;
    extern __shared__ float s_lds[];
    const Score sc(b, a, s_lds);
    const int lane = lane_id(), wave = threadIdx.x / kWave, waves_b = blockDim.x / kWave;
    const int entries = (3 * b.nb + 1) * a.H;
    float* s_tab = s_lds + Score::floats(b);
    float* tab = s_tab + wave * entries;
    if constexpr (TAB) {
        for (int e = threadIdx.x; e < entries * waves_b; e += blockDim.x) s_tab[e] = 0.0f;
        __syncthreads();
    }
    const LaneAt at(l, a.Hkv, a.D, W);
    const int Rq = a.H / a.Hkv;
    const int step = l.Hc * l.G;
    const uint32_t qrb = (uint32_t)(a.q_row * (int64_t)sizeof(T)), orb = (uint32_t)(a.H * a.D * (int)sizeof(T));
    const bool same = qrb == orb;

    each_unit(walk.units, waves_b, wave, [&](uint32_t unit) {
        const uint32_t cloud = udiv(unit, walk.by_cloud);
        const uint32_t in = unit - cloud * (uint32_t)walk.per_cloud;
        const int32_t i0 = EACH ? (int32_t)in * l.S + at.slot : (int32_t)in;
        const bool live_row = !EACH || (i0 < g.N && at.slot < l.S);
        const int64_t pt = (int64_t)cloud * g.N + (live_row ? i0 : 0);
        const int64_t c0 = (int64_t)cloud * g.M;
        const Raw x = load_channels<T, BUF>((const T*)a.k + pt * a.k_row + at.head * a.D + at.chan, at.n);
        const Raw y = load_channels<T, BUF>((const T*)a.v + pt * a.v_row + at.head * a.D + at.chan, at.n);
        float gk[W] = {}, gv[W] = {}, p3[3] = {};
        if (sc.placed()) load_xyz(g.points, pt, p3);
        int64_t beg = pt_off[pt], end = pt_off[pt + 1];
        beg = beg < 0 ? 0 : beg > capacity ? capacity : beg;
        end = end < beg ? beg : end > capacity ? capacity : end;
        if (EACH && !live_row) end = beg;
        const int ch = EACH ? step : kWave;
        const int first = EACH ? at.slot * step : at.slot;
        for (int64_t s0 = beg; EACH ? __any(s0 < end) : s0 < end; s0 += ch) {
            const int n = end - s0 < ch ? (int)(end - s0) : ch;
            int32_t mine = -1;
            uint32_t u = 0;
            float dist = 0.0f;
            const int e = EACH ? at.li : lane;
            if (e < n) {
                mine = pt_center[s0 + e];
                if ((uint32_t)mine >= (uint32_t)g.M) mine = -1;
                if (sc.placed() && mine >= 0) {
                    float c[3];
                    load_xyz(g.centers, c0 + mine, c);
                    pair_place(sc.ed, sc.dist, p3, c, u, dist);
                }
            }
            for (int r = 0; r < Rq; ++r) {
                const int h = at.head * Rq + r;
                const Rows<T, BUF> qr((const T*)a.q + c0 * a.q_row, a.q_row, (uint32_t)((g.M - 1) * (int64_t)qrb) + orb,
                                      h * a.D + at.chan, at.n);
                const Rows<T, BUF> gr(dout + c0 * a.H * a.D, (int64_t)a.H * a.D, (uint32_t)(g.M * (int64_t)orb),
                                      h * a.D + at.chan, at.n);
                const float slope = b.slope && at.on ? b.slope[h] : 0.0f;
                for (int t = 0; EACH ? __any(t < n) : t < n; t += EACH ? U : U * l.S) {
                    Raw q[U], go[U];
                    uint32_t pu[U];
                    float pd[U], s[2 * U];
                    float2 st[U];
                    bool there[U];
#pragma unroll
                    for (int i = 0; i < U; ++i) {
                        const int from = EACH ? t + i : t + i * l.S + at.slot;
                        const int src = (EACH ? first + from : from) & 63;
                        int32_t jj = __shfl(mine, src, kWave);
                        if (from >= n) jj = -1;
                        there[i] = jj >= 0;
                        const uint32_t key = Rows<T, BUF>::key(jj, qrb);
                        q[i] = qr.load(key);
                        go[i] = gr.load(!BUF || same ? key : Rows<T, BUF>::key(jj, orb));
                        st[i] = stat[(c0 + (there[i] ? jj : 0)) * a.H + h];
                        if (sc.nb > 0) pu[i] = (uint32_t)__shfl((int)u, src, kWave);
                        else pu[i] = 0;
                        pd[i] = sc.dist ? __shfl(dist, src, kWave) : 0.0f;
                    }
#pragma unroll
                    for (int i = 0; i < U; ++i) {
                        s[2 * i] = dot<T>(q[i], x);
                        s[2 * i + 1] = dot<T>(go[i], y);
                    }
                    group_sums(s, l.G);
#pragma unroll
                    for (int i = 0; i < U; ++i) {
                        float e2 = 0.0f, dp = s[2 * i + 1];
                        float v = sc.product(s[2 * i], e2);
                        if (sc.placed()) {
                            const float bi = sc.bias(h, pu[i], slope, pd[i]);
                            v += bi;
                            if (__any(bi == kNegInf)) {
                                if (bi == kNegInf) {
                                    q[i] = go[i] = Raw{0, 0, 0, 0};
                                    v = kNegInf;
                                    dp = 0.0f;
                                }
                            }
                        }
                        const float p = there[i] ? weight(v - st[i].x) : 0.0f;
                        const float ds = there[i] ? p * (dp - st[i].y) : 0.0f;
                        add_channels<T>(gk, ds * sc.slack(e2), q[i]);
                        add_channels<T>(gv, p, go[i]);
                        if constexpr (TAB) {
                            if (at.chan == 0 && there[i] && at.on) {
                                if (b.nb > 0) {
                                    lds_add(&tab[(pu[i] & 255u) * a.H + h], ds);
                                    lds_add(&tab[(b.nb + (pu[i] >> 8 & 255u)) * a.H + h], ds);
                                    lds_add(&tab[(2 * b.nb + (pu[i] >> 16)) * a.H + h], ds);
                                }
                                if (b.slope) lds_add(&tab[3 * b.nb * a.H + h], ds * pd[i]);
                            }
                        }
                    }
                }
            }
        }
        if (!EACH) {
#pragma unroll
            for (int w = 0; w < W; ++w) {
                gk[w] = slots_sum(gk[w], l.S, step, at.slot, lane);
                gv[w] = slots_sum(gv[w], l.S, step, at.slot, lane);
            }
        }
        if (!(EACH ? at.on && live_row : at.on && at.slot == 0)) return;
#pragma unroll
        for (int w = 0; w < W; ++w) gk[w] *= a.scale;
        const int64_t o = (pt * a.Hkv + at.head) * a.D + at.chan;
        store_channels<T, BUF>(dk + o, at.n, gk);
        store_channels<T, BUF>(dv + o, at.n, gv);
    });
    if constexpr (TAB) {
        __syncthreads();
        const int64_t blk = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
        for (int e = threadIdx.x; e < entries; e += blockDim.x) {
            float x = 0.0f;
            for (int w = 0; w < waves_b; ++w) x += s_tab[w * entries + e];
            part[blk * entries + e] = x;
        }
    }
}

// ------------------------------------------------------------------ host side

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Whether every slot of a wave takes a list of its own: lists short beside a
// chunk of the slot's lanes, and enough of them.
bool each_of(int64_t rows, int64_t slots, const Lanes& l) {
    if (l.S == 1) return true;
    return slots / rows <= 32 && rows / l.S >= 4096;
}

// A workgroup to a list whose mean length gives each wave a chunk; parts where
// there are few lists.
struct Split {
    bool block;
    int32_t parts;
};

Split split_of(const Groups& g, int32_t passes, int32_t HD) {
    Split s = {false, 1};
    const int64_t mean = g.idx_len / g.rows;  // of ragged lists only their mean is known here
    const int64_t rows = (int64_t)g.rows * passes;
    if (mean < 2 * kWave || HD > kJoinFloats) return s;
    s.block = true;
    int64_t p = 1024 / rows;
    if (p > mean / (2 * kWave)) p = mean / (2 * kWave);
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
    const int64_t most = (int64_t)(kNone - 4096) / (int64_t)sizeof(T);
    const int64_t qd = (int64_t)a.H * a.D;
    return a.k_row <= most / g.N && a.v_row <= most / g.N && a.q_row <= most / g.M && qd <= most / g.M;
}

int heads_per_lane(const Attn& a) {
    const int r = a.H / a.Hkv;
    return r % 4 == 0 ? 4 : r % 2 == 0 ? 2 : 1;
}

uint32_t blocks_of(int64_t units, int64_t per) {
    const int64_t n = (units + per - 1) / per;
    return (uint32_t)(n > kAtBlocks ? kAtBlocks : n < 8 ? 8 : (n + 7) & ~7ll);
}

template <typename K>
hipError_t allow_lds(K kern, size_t bytes) {
    if (bytes <= (48 << 10)) return hipSuccess;
    return hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}

template <typename T, bool BUF, int R>
hipError_t forward_as(const Groups& g, int32_t B, const Attn& a, const Bias& b, void* out, float* lse, void* ws,
                      hipStream_t s) {
    const Lanes l = make_lanes<T>(a.H / R, a.D);
    const Split sp = split_of(g, 1, a.H * a.D);
    Partial part = {nullptr, nullptr, sp.parts};
    if (part.parts > 1) {
        part.ml = (float*)ws;
        part.acc = part.ml + (size_t)part.parts * g.rows * a.H * 2;
    }
    size_t lds = (size_t)Score::floats(b) * 4;
    hipError_t e = hipSuccess;
    if (sp.block) {
        const Walk w = make_walk<false>(B, g.M, l);
        lds += (size_t)kAtWaves * l.Hc * R * (a.D + 2) * 4;
        auto kern = k_at<T, BUF, R, false, true>;
        if ((e = allow_lds(kern, lds)) != hipSuccess) return e;
        kern<<<dim3(blocks_of(w.units, 1), l.passes, sp.parts), kAtThreads, lds, s>>>(g, b, a, l, w, (T*)out, lse,
                                                                                     part);
    } else if (each_of(g.rows, g.idx_len, l)) {
        const Walk w = make_walk<true>(B, g.M, l);
        auto kern = k_at<T, BUF, R, true, false>;
        if ((e = allow_lds(kern, lds)) != hipSuccess) return e;
        kern<<<dim3(blocks_of(w.units, kAtWaves), l.passes), kAtThreads, lds, s>>>(g, b, a, l, w, (T*)out, lse, part);
    } else {
        const Walk w = make_walk<false>(B, g.M, l);
        auto kern = k_at<T, BUF, R, false, false>;
        if ((e = allow_lds(kern, lds)) != hipSuccess) return e;
        kern<<<dim3(blocks_of(w.units, kAtWaves), l.passes), kAtThreads, lds, s>>>(g, b, a, l, w, (T*)out, lse, part);
    }
    if (part.parts > 1) {
        const int64_t n = (int64_t)g.rows * a.H;
        k_at_join<T><<<blocks_of(n, kAtWaves), kAtThreads, 0, s>>>(part, g.rows, a, (T*)out, lse);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t forward(const Groups& g, int32_t B, const Attn& a, const Bias& b, void* out, float* lse, void* ws,
                   hipStream_t s) {
    const bool buf = vectors<T>(g, a, {a.q, a.k, a.v, out});
    const int r = heads_per_lane(a);
    auto f = buf ? (r == 4 ? forward_as<T, true, 4> : r == 2 ? forward_as<T, true, 2> : forward_as<T, true, 1>)
                 : forward_as<T, false, 1>;
    return f(g, B, a, b, out, lse, ws, s);
}

template <typename T, bool BUF, bool EACH>
hipError_t back_centers(const Groups& g, int32_t B, const Attn& a, const Bias& b, const Lanes& l, const float* lse,
                        const void* dout, void* dq, float2* stat, hipStream_t s) {
    const Walk w = make_walk<EACH>(B, g.M, l);
    const size_t lds = (size_t)Score::floats(b) * 4;
    auto kern = k_at_back_c<T, BUF, EACH>;
    hipError_t e = allow_lds(kern, lds);
    if (e != hipSuccess) return e;
    kern<<<dim3(blocks_of(w.units, kAtWaves), l.passes), kAtThreads, lds, s>>>(g, b, a, l, w, lse, (const T*)dout,
                                                                              (T*)dq, stat);
    return hipGetLastError();
}

// The launch of the gradient at the points: waves of a workgroup whose tables
// fit its LDS, and the workgroups, each with partial sums of its own.
struct BackShape {
    int waves;
    uint32_t blocks;
    size_t lds;
};

BackShape back_shape(int64_t units, int32_t passes, const Bias& b, bool tab) {
    BackShape r;
    const size_t base = (size_t)Score::floats(b) * 4, entries = (size_t)(3 * b.nb + 1) * b.H * 4;
    r.waves = kAtWaves;
    if (!tab) {
        r.blocks = blocks_of(units, r.waves);
        r.lds = base;
        return r;
    }
    while (r.waves > 1 && base + entries * r.waves > kAtLds) r.waves >>= 1;
    r.lds = base + entries * r.waves;
    r.blocks = blocks_of(units, r.waves);
    const uint32_t most = kAtParts / passes;
    if (r.blocks > most) r.blocks = most < 8 ? 8 : most & ~7u;
    return r;
}

bool points_each(const Groups& g, int32_t B, const Lanes& l) { return each_of((int64_t)B * g.N, g.idx_len, l); }

int64_t point_units(const Groups& g, int32_t B, const Lanes& l) {
    return points_each(g, B, l) ? make_walk<true>(B, g.N, l).units : make_walk<false>(B, g.N, l).units;
}

template <typename T, bool BUF, bool EACH, bool TAB>
hipError_t back_points(const Groups& g, int32_t B, const Attn& a, const Bias& b, const Lanes& l, const int64_t* pt_off,
                       const int32_t* pt_center, int64_t capacity, const float2* stat, const void* dout, void* dk,
                       void* dv, float* part, hipStream_t s) {
    const Walk w = make_walk<EACH>(B, g.N, l);
    const BackShape r = back_shape(w.units, l.passes, b, TAB);
    auto kern = k_at_back_p<T, BUF, EACH, TAB>;
    hipError_t e = allow_lds(kern, r.lds);
    if (e != hipSuccess) return e;
    kern<<<dim3(r.blocks, l.passes), r.waves * kWave, r.lds, s>>>(g, b, a, l, w, pt_off, pt_center, capacity, stat,
                                                                  (const T*)dout, (T*)dk, (T*)dv, part);
    return hipGetLastError();
}

template <typename T>
hipError_t backward(const Groups& g, int32_t B, const Attn& a, const Bias& b, const int64_t* pt_off,
                    const int32_t* pt_center, int64_t capacity, const float* lse, const void* dout, void* dq, void* dk,
                    void* dv, float* dtable, float* dslope, void* ws, hipStream_t s) {
    const Lanes lc = make_lanes<T>(a.H, a.D), lp = make_lanes<T>(a.Hkv, a.D);
    float2* stat = (float2*)ws;
    float* part = (float*)((char*)ws + align256((size_t)g.rows * a.H * 8));
    const bool buf = vectors<T>(g, a, {a.q, a.k, a.v, dout, dq, dk, dv});
    const bool ec = each_of(g.rows, g.idx_len, lc), ep = points_each(g, B, lp), tab = dtable || dslope;
    auto fc = buf ? (ec ? back_centers<T, true, true> : back_centers<T, true, false>)
                  : (ec ? back_centers<T, false, true> : back_centers<T, false, false>);
    hipError_t e = fc(g, B, a, b, lc, lse, dout, dq, stat, s);
    if (e != hipSuccess) return e;
    auto with = [&](auto bufc, auto tabc) {
        constexpr bool BUF = decltype(bufc)::value, TAB = decltype(tabc)::value;
        return (ep ? back_points<T, BUF, true, TAB> : back_points<T, BUF, false, TAB>)(
            g, B, a, b, lp, pt_off, pt_center, capacity, stat, dout, dk, dv, part, s);
    };
    const std::true_type yes;
    const std::false_type no;
    e = buf ? (tab ? with(yes, yes) : with(yes, no)) : (tab ? with(no, yes) : with(no, no));
    if (e != hipSuccess || !tab) return e;
    const BackShape r = back_shape(point_units(g, B, lp), lp.passes, b, true);
    return launch_bias_reduce(part, (int32_t)r.blocks * lp.passes, b, dtable, dslope, s);
}

Lanes lanes_of(int32_t dtype, int32_t heads, int32_t D) {
    return dtype == CAGQ_F32 ? make_lanes<float>(heads, D) : make_lanes<bf16>(heads, D);
}

}  // namespace

size_t group_attention_bytes(const Groups& g, int32_t B, const Attn& a, int32_t dtype, const Bias& b, bool backward) {
    if (!backward) {
        const Split sp = split_of(g, 1, a.H * a.D);
        return sp.parts > 1 ? (size_t)sp.parts * g.rows * a.H * (2 + a.D) * 4 : 0;
    }
    const size_t stat = align256((size_t)g.rows * a.H * 8);
    if (b.nb == 0 && !b.slope) return stat;
    const Lanes l = lanes_of(dtype, a.Hkv, a.D);
    const BackShape r = back_shape(point_units(g, B, l), l.passes, b, true);
    return stat + (size_t)r.blocks * l.passes * (3 * b.nb + 1) * b.H * 4;
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
