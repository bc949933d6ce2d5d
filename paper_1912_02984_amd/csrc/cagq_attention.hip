// Attention of each center over the features of its group, and its gradients
// (cagq_group_attention, cagq_group_attention_backward; the formulas are in
// include/cagq.h).
//
// A query here meets a list of its own, so there is no tile of queries that
// share keys and no matrix product to make of it: a pair costs 4 D flops and
// reads 2 D features. The work is gathering rows, and a wave takes the rows
// of one center at a time: G lanes to a head of a row (16 bytes of features
// each), the row's heads side by side, and as many rows at once as the wave
// has lanes for ("slots").
#include "cagq_features.h"

namespace cagq {

namespace {

constexpr int kAtThreads = 256;
constexpr int kAtWaves = kAtThreads / kWave;
constexpr int kAtParts = 1024;     // workgroups of the gradient at the points, where the bias wants its own
constexpr int kAtLds = 128 << 10;  // LDS of their tables, a table per wave

// How a wave's lanes are laid over a row of `heads` heads of D channels.
struct Lanes {
    int32_t G;      // lanes per head, a power of two
    int32_t Hc;     // heads side by side
    int32_t S;      // slots: rows at once
    int32_t passes; // waves to a row's heads
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
    int slot, head, chan, n;  // slot of the lane, its head, first channel, channels
    bool on;                  // it has work

    __device__ __forceinline__ LaneAt(const Lanes& l, int heads, int D, int W, int pass) {
        const int lane = lane_id();
        const int item = lane / l.G;
        slot = item / l.Hc;
        head = pass * l.Hc + item - slot * l.Hc;
        chan = (lane & (l.G - 1)) * W;
        on = slot < l.S && head < heads;
        n = D - chan;
        n = !on || n < 0 ? 0 : n > W ? W : n;
        if (!on) head = 0;
    }
};

template <int W>
__device__ __forceinline__ float dot(const float (&a)[W], const float (&b)[W]) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < W; ++i) s = fmaf(a[i], b[i], s);
    return s;
}

// Sum over the slots of a wave (lanes slot * step + i), in slot 0.
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

// cap * tanh(x / cap), and the tanh: 1 - 2 / (1 + exp(2 x / cap)), whose error
// is of the order of 2^-24 of 1, that is of cap, not of x: scores are only
// ever used by their differences.
__device__ __forceinline__ float capped(float x, float cap, float two_over_cap, float& t) {
    t = fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + __expf(x * two_over_cap)), 1.0f);
    return cap * t;
}

constexpr float kNegInf = -__builtin_inff();

// Partial softmax of a part of a list: maximum, sum, and the weighted sum's D
// channels, per row and head.
struct Partial {
    float* ml;   // [parts][rows][H][2]
    float* acc;  // [parts][rows][H][D]
    int32_t parts;
};

template <typename T, bool VEC>
__global__ __launch_bounds__(kAtThreads) void k_at(Groups g, Bias b, Attn a, Lanes l, T* __restrict__ out,
                                                   float* __restrict__ lse, Partial part) {
    constexpr int W = kVec<T>;
    const int lane = lane_id();
    const int64_t waves = (int64_t)gridDim.x * kAtWaves;
    const int64_t all_w = (int64_t)g.rows * part.parts * l.passes;
    for (int64_t w = (int64_t)blockIdx.x * kAtWaves + threadIdx.x / kWave; w < all_w; w += waves) {
        const int pass = (int)(w % l.passes);
        const int64_t rp = w / l.passes;
        const int pi = (int)(rp % part.parts);
        const int64_t row = rp / part.parts;
        const LaneAt at(l, a.H, a.D, W, pass);
        const int64_t cloud = (int64_t)udiv((uint32_t)row, g.mm) * g.N;
        const int kvh = at.head / (a.H / a.Hkv);
        const T* kp = (const T*)a.k + kvh * a.D + at.chan;
        const T* vp = (const T*)a.v + kvh * a.D + at.chan;
        float q[W], acc[W] = {}, m = kNegInf, sum = 0.0f;
        load_channels<T, VEC>((const T*)a.q + row * a.q_row + at.head * a.D + at.chan, at.n, q);
#pragma unroll
        for (int i = 0; i < W; ++i) q[i] *= a.scale;
        const bool placed = b.nb > 0 || b.slope;
        const float slope = b.slope && at.on ? b.slope[at.head] : 0.0f;
        const float two_over_cap = a.cap > 0.0f ? 2.0f / a.cap : 0.0f;
        float c[3] = {};
        if (placed) load_xyz(g.centers, row, c);
        int64_t beg, end;
        g.range((int32_t)row, beg, end);
        if (part.parts > 1) {
            const int64_t per = ((end - beg + part.parts - 1) / part.parts + kWave - 1) & -(int64_t)kWave;
            beg += pi * per;
            end = end < beg + per ? end : beg + per;
        }
        for (int64_t s0 = beg; s0 < end; s0 += kWave) {
            const int n = end - s0 < kWave ? (int)(end - s0) : kWave;
            int32_t mine = -1;
            uint32_t u = 0;
            float dist = 0.0f;
            if (lane < n) {
                mine = g.idx[s0 + lane];
                if ((uint32_t)mine >= (uint32_t)g.N) mine = -1;
                if (placed && mine >= 0) {
                    float p[3];
                    load_xyz(g.points, cloud + mine, p);
                    pair_place(b.edges, b.nb, b.slope != nullptr, p, c, u, dist);
                }
            }
            for (int t = 0; t < n; t += l.S) {
                const int from = t + at.slot;
                const int src = from < n ? from : 0;
                int32_t i = __shfl(mine, src, kWave);
                const uint32_t pu = (uint32_t)__shfl((int)u, src, kWave);
                const float pd = __shfl(dist, src, kWave);
                const bool live = at.on && from < n && i >= 0;
                float x[W];
                load_channels<T, VEC>(kp + (cloud + (live ? i : 0)) * a.k_row, live ? at.n : 0, x);
                float s = group_sum(dot<W>(q, x), l.G);
                if (!live) continue;
                if (a.cap > 0.0f) {
                    float th;
                    s = capped(s, a.cap, two_over_cap, th);
                }
                if (placed) s += bias_at(b.table, b.nb, a.H, slope, at.head, pu, pd);
                if (s == kNegInf) continue;
                const float mn = fmaxf(m, s);
                const float keep = __expf(m - mn), p = __expf(s - mn);
                m = mn;
                sum = fmaf(sum, keep, p);
                load_channels<T, VEC>(vp + (cloud + i) * a.v_row, at.n, x);
#pragma unroll
                for (int k = 0; k < W; ++k) acc[k] = fmaf(p, x[k], acc[k] * keep);
            }
        }
        // the slots' parts joined in slot 0
        const int step = l.Hc * l.G;
        const float all = __shfl(slots_max(m, l.S, step, at.slot, lane), lane - at.slot * step, kWave);
        const float f = m == kNegInf ? 0.0f : __expf(m - all);
        sum = slots_sum(sum * f, l.S, step, at.slot, lane);
#pragma unroll
        for (int k = 0; k < W; ++k) acc[k] = slots_sum(acc[k] * f, l.S, step, at.slot, lane);
        if (at.slot > 0 || !at.on) continue;
        const int64_t rh = row * a.H + at.head;
        if (part.parts > 1) {
            const int64_t prh = (int64_t)pi * g.rows * a.H + rh;
            if (at.chan == 0) {
                part.ml[2 * prh] = all;
                part.ml[2 * prh + 1] = sum;
            }
#pragma unroll
            for (int k = 0; k < W; ++k)
                if (k < at.n) part.acc[prh * a.D + at.chan + k] = acc[k];
            continue;
        }
        const bool some = all != kNegInf;
        const float inv = some ? 1.0f / sum : 0.0f;
#pragma unroll
        for (int k = 0; k < W; ++k) acc[k] = some ? acc[k] * inv : 0.0f;
        store_channels<T, VEC>(out + rh * a.D + at.chan, at.n, acc);
        if (lse && at.chan == 0) lse[rh] = some ? all + __logf(sum) : kNegInf;
    }
}

// The parts of each row and head joined, a thread per channel.
template <typename T>
__global__ __launch_bounds__(kAtThreads) void k_at_join(Partial part, int64_t rows, Attn a, T* __restrict__ out,
                                                        float* __restrict__ lse) {
    const int64_t all_rh = rows * a.H, step = (int64_t)gridDim.x * kAtThreads;
    for (int64_t t = (int64_t)blockIdx.x * kAtThreads + threadIdx.x; t < all_rh * a.D; t += step) {
        const int64_t rh = t / a.D;
        const int d = (int)(t - rh * a.D);
        float m = kNegInf;
        for (int p = 0; p < part.parts; ++p) m = fmaxf(m, part.ml[2 * (p * all_rh + rh)]);
        float sum = 0.0f, x = 0.0f;
        if (m != kNegInf) {
            for (int p = 0; p < part.parts; ++p) {
                const float pm = part.ml[2 * (p * all_rh + rh)];
                if (pm == kNegInf) continue;
                const float f = __expf(pm - m);
                sum = fmaf(part.ml[2 * (p * all_rh + rh) + 1], f, sum);
                x = fmaf(part.acc[(p * all_rh + rh) * a.D + d], f, x);
            }
            x /= sum;
        }
        out[t] = (T)x;
        if (lse && d == 0) lse[rh] = m == kNegInf ? kNegInf : m + __logf(sum);
    }
}

// Gradient at the centers. With da = ds (1 - t^2) (t the cap's tanh):
//   dq = scale * sum da k = scale * (sum p dp (1 - t^2) k - delta * sum p (1 - t^2) k),
// so that delta = sum p dp, which the gradient at the points needs as well, is
// known to fp32 only at the end of the one pass over the list.
template <typename T, bool VEC>
__global__ __launch_bounds__(kAtThreads) void k_at_back_c(Groups g, Bias b, Attn a, Lanes l,
                                                          const float* __restrict__ lse, const T* __restrict__ dout,
                                                          T* __restrict__ dq, float* __restrict__ delta) {
    constexpr int W = kVec<T>;
    const int lane = lane_id();
    const int64_t waves = (int64_t)gridDim.x * kAtWaves;
    for (int64_t w = (int64_t)blockIdx.x * kAtWaves + threadIdx.x / kWave; w < (int64_t)g.rows * l.passes; w += waves) {
        const int pass = (int)(w % l.passes);
        const int64_t row = w / l.passes;
        const LaneAt at(l, a.H, a.D, W, pass);
        const int64_t cloud = (int64_t)udiv((uint32_t)row, g.mm) * g.N;
        const int kvh = at.head / (a.H / a.Hkv);
        const T* kp = (const T*)a.k + kvh * a.D + at.chan;
        const T* vp = (const T*)a.v + kvh * a.D + at.chan;
        const int64_t rh = row * a.H + at.head;
        float q[W], go[W], acc[W] = {}, acd[W] = {}, sum = 0.0f;
        load_channels<T, VEC>((const T*)a.q + row * a.q_row + at.head * a.D + at.chan, at.n, q);
        load_channels<T, VEC>(dout + rh * a.D + at.chan, at.n, go);
#pragma unroll
        for (int i = 0; i < W; ++i) q[i] *= a.scale;
        const bool placed = b.nb > 0 || b.slope;
        const float slope = b.slope && at.on ? b.slope[at.head] : 0.0f;
        const float two_over_cap = a.cap > 0.0f ? 2.0f / a.cap : 0.0f;
        const float ls = at.on ? lse[rh] : kNegInf;
        float c[3] = {};
        if (placed) load_xyz(g.centers, row, c);
        int64_t beg, end;
        g.range((int32_t)row, beg, end);
        for (int64_t s0 = beg; s0 < end; s0 += kWave) {
            const int n = end - s0 < kWave ? (int)(end - s0) : kWave;
            int32_t mine = -1;
            uint32_t u = 0;
            float dist = 0.0f;
            if (lane < n) {
                mine = g.idx[s0 + lane];
                if ((uint32_t)mine >= (uint32_t)g.N) mine = -1;
                if (placed && mine >= 0) {
                    float p[3];
                    load_xyz(g.points, cloud + mine, p);
                    pair_place(b.edges, b.nb, b.slope != nullptr, p, c, u, dist);
                }
            }
            for (int t = 0; t < n; t += l.S) {
                const int from = t + at.slot;
                const int src = from < n ? from : 0;
                const int32_t i = __shfl(mine, src, kWave);
                const uint32_t pu = (uint32_t)__shfl((int)u, src, kWave);
                const float pd = __shfl(dist, src, kWave);
                const bool live = at.on && from < n && i >= 0;
                float x[W], y[W];
                load_channels<T, VEC>(kp + (cloud + (live ? i : 0)) * a.k_row, live ? at.n : 0, x);
                load_channels<T, VEC>(vp + (cloud + (live ? i : 0)) * a.v_row, live ? at.n : 0, y);
                float s = group_sum(dot<W>(q, x), l.G);
                const float dp = group_sum(dot<W>(go, y), l.G);
                if (!live) continue;
                float slack = 1.0f;
                if (a.cap > 0.0f) {
                    float th;
                    s = capped(s, a.cap, two_over_cap, th);
                    slack = 1.0f - th * th;
                }
                if (placed) s += bias_at(b.table, b.nb, a.H, slope, at.head, pu, pd);
                if (s == kNegInf) continue;
                const float p = __expf(s - ls);
                if (p == 0.0f) continue;
                const float pdp = p * dp, pt = p * slack;
                sum += pdp;
#pragma unroll
                for (int k = 0; k < W; ++k) {
                    acc[k] = fmaf(pdp * slack, x[k], acc[k]);
                    acd[k] = fmaf(pt, x[k], acd[k]);
                }
            }
        }
        const int step = l.Hc * l.G;
        sum = slots_sum(sum, l.S, step, at.slot, lane);
#pragma unroll
        for (int k = 0; k < W; ++k) {
            acc[k] = slots_sum(acc[k], l.S, step, at.slot, lane);
            acd[k] = slots_sum(acd[k], l.S, step, at.slot, lane);
        }
        if (at.slot > 0 || !at.on) continue;
#pragma unroll
        for (int k = 0; k < W; ++k) acc[k] = a.scale * fmaf(-sum, acd[k], acc[k]);
        store_channels<T, VEC>(dq + rh * a.D + at.chan, at.n, acc);
        if (at.chan == 0) delta[rh] = sum;
    }
}

// Gradient at the points: a wave per point over the centers that hold it, the
// scores computed again; and the bias's gradient, which a wave sums in a
// table of its own in LDS.
template <typename T, bool VEC, bool TAB>
__global__ __launch_bounds__(kAtThreads) void k_at_back_p(Groups g, Bias b, Attn a, Lanes l, int64_t points,
                                                          Magic mn, const int64_t* __restrict__ pt_off,
                                                          const int32_t* __restrict__ pt_center, int64_t capacity,
                                                          const float* __restrict__ lse,
                                                          const float* __restrict__ delta, const T* __restrict__ dout,
                                                          T* __restrict__ dk, T* __restrict__ dv,
                                                          float* __restrict__ part) {
    constexpr int W = kVec<T>;
    extern __shared__ float s_tab[];
    const int lane = lane_id();
    const int waves_b = blockDim.x / kWave;
    const int entries = (3 * b.nb + 1) * a.H;
    float* tab = s_tab + (threadIdx.x / kWave) * entries;
    if constexpr (TAB) {
        for (int e = threadIdx.x; e < entries * waves_b; e += blockDim.x) s_tab[e] = 0.0f;
        __syncthreads();
    }
    const int R = a.H / a.Hkv;
    const bool placed = b.nb > 0 || b.slope;
    const float two_over_cap = a.cap > 0.0f ? 2.0f / a.cap : 0.0f;
    const int64_t waves = (int64_t)gridDim.x * waves_b;
    const int step = l.Hc * l.G;
    for (int64_t w = (int64_t)blockIdx.x * waves_b + threadIdx.x / kWave; w < points * l.passes; w += waves) {
        const int pass = (int)(w % l.passes);
        const int64_t pt = w / l.passes;
        const LaneAt at(l, a.Hkv, a.D, W, pass);
        const int64_t cloud = (int64_t)udiv((uint32_t)pt, mn) * g.M;
        float x[W], y[W], gk[W] = {}, gv[W] = {};
        load_channels<T, VEC>((const T*)a.k + pt * a.k_row + at.head * a.D + at.chan, at.n, x);
        load_channels<T, VEC>((const T*)a.v + pt * a.v_row + at.head * a.D + at.chan, at.n, y);
        float p3[3] = {};
        if (placed) load_xyz(g.points, pt, p3);
        int64_t beg = pt_off[pt], end = pt_off[pt + 1];
        beg = beg < 0 ? 0 : beg > capacity ? capacity : beg;
        end = end < beg ? beg : end > capacity ? capacity : end;
        for (int64_t s0 = beg; s0 < end; s0 += kWave) {
            const int n = end - s0 < kWave ? (int)(end - s0) : kWave;
            int32_t mine = -1;
            uint32_t u = 0;
            float dist = 0.0f;
            if (lane < n) {
                mine = pt_center[s0 + lane];
                if ((uint32_t)mine >= (uint32_t)g.M) mine = -1;
                if (placed && mine >= 0) {
                    float c[3];
                    load_xyz(g.centers, cloud + mine, c);
                    pair_place(b.edges, b.nb, b.slope != nullptr, p3, c, u, dist);
                }
            }
            for (int t = 0; t < n; t += l.S) {
                const int from = t + at.slot;
                const int src = from < n ? from : 0;
                const int32_t j = __shfl(mine, src, kWave);
                const uint32_t pu = (uint32_t)__shfl((int)u, src, kWave);
                const float pd = __shfl(dist, src, kWave);
                const bool live = at.on && from < n && j >= 0;
                const int64_t row = cloud + (live ? j : 0);
                for (int r = 0; r < R; ++r) {
                    const int h = at.head * R + r;
                    float q[W], go[W];
                    load_channels<T, VEC>((const T*)a.q + row * a.q_row + h * a.D + at.chan, live ? at.n : 0, q);
                    load_channels<T, VEC>(dout + (row * a.H + h) * a.D + at.chan, live ? at.n : 0, go);
#pragma unroll
                    for (int k = 0; k < W; ++k) q[k] *= a.scale;
                    float s = group_sum(dot<W>(q, x), l.G);
                    const float dp = group_sum(dot<W>(go, y), l.G);
                    if (!live) continue;
                    float slack = 1.0f;
                    if (a.cap > 0.0f) {
                        float th;
                        s = capped(s, a.cap, two_over_cap, th);
                        slack = 1.0f - th * th;
                    }
                    if (placed) s += bias_at(b.table, b.nb, a.H, b.slope ? b.slope[h] : 0.0f, h, pu, pd);
                    if (s == kNegInf) continue;
                    const float p = __expf(s - lse[row * a.H + h]);
                    if (p == 0.0f) continue;
                    const float ds = p * (dp - delta[row * a.H + h]);
                    const float da = ds * slack;
#pragma unroll
                    for (int k = 0; k < W; ++k) {
                        gk[k] = fmaf(da, q[k], gk[k]);  // q holds the scale
                        gv[k] = fmaf(p, go[k], gv[k]);
                    }
                    if constexpr (TAB) {
                        if (at.chan == 0) {
                            if (b.nb > 0) {
                                lds_add(&tab[(pu & 255u) * a.H + h], ds);
                                lds_add(&tab[(b.nb + (pu >> 8 & 255u)) * a.H + h], ds);
                                lds_add(&tab[(2 * b.nb + (pu >> 16)) * a.H + h], ds);
                            }
                            if (b.slope) lds_add(&tab[3 * b.nb * a.H + h], ds * pd);
                        }
                    }
                }
            }
        }
#pragma unroll
        for (int k = 0; k < W; ++k) {
            gk[k] = slots_sum(gk[k], l.S, step, at.slot, lane);
            gv[k] = slots_sum(gv[k], l.S, step, at.slot, lane);
        }
        if (at.slot > 0 || !at.on) continue;
        const int64_t o = (pt * a.Hkv + at.head) * a.D + at.chan;
        store_channels<T, VEC>(dk + o, at.n, gk);
        store_channels<T, VEC>(dv + o, at.n, gv);
    }
    if constexpr (TAB) {
        __syncthreads();
        for (int e = threadIdx.x; e < entries; e += blockDim.x) {
            float x = 0.0f;
            for (int w = 0; w < waves_b; ++w) x += s_tab[w * entries + e];
            part[(int64_t)blockIdx.x * entries + e] = x;
        }
    }
}

// ------------------------------------------------------------------ host side

// Waves a launch wants at least before a list is worth splitting, and the
// shortest part.
constexpr int64_t kSplitWaves = 4096;
constexpr int64_t kSplitLen = 128;

int32_t parts_of(const Groups& g, int32_t passes) {
    const int64_t mean = g.idx_len / g.rows;  // of ragged lists only their mean is known here
    const int64_t waves = (int64_t)g.rows * passes;
    if (mean < 2 * kSplitLen || waves >= kSplitWaves) return 1;
    int64_t p = mean / kSplitLen;
    const int64_t most = kSplitWaves / waves;
    p = p < most ? p : most;
    return (int32_t)(p < 1 ? 1 : p > 256 ? 256 : p);
}

int32_t lanes_passes(int32_t dtype, int32_t heads, int32_t D) {
    return dtype == CAGQ_F32 ? make_lanes<float>(heads, D).passes : make_lanes<bf16>(heads, D).passes;
}

struct BackShape {
    int waves, blocks;
    size_t lds;
};

BackShape back_shape(int64_t points, int32_t passes, const Bias& b) {
    BackShape r;
    const size_t entries = (size_t)(3 * b.nb + 1) * b.H;
    r.waves = kAtWaves;
    while (r.waves > 1 && entries * 4 * r.waves > kAtLds) r.waves >>= 1;
    r.lds = entries * 4 * r.waves;
    const int64_t n = (points * passes + r.waves - 1) / r.waves;
    r.blocks = (int)(n > kAtParts ? kAtParts : n);
    return r;
}

// Workgroups for n items; the kernels go round where there are more.
uint32_t grid_of(int64_t n, int64_t per_block) {
    n = (n + per_block - 1) / per_block;
    return (uint32_t)(n > (1 << 20) ? (1 << 20) : n);
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

template <typename T>
bool vectors(const Attn& a, std::initializer_list<const void*> ptrs) {
    constexpr int W = kVec<T>;
    if (a.D % W || a.q_row % W || a.k_row % W || a.v_row % W) return false;
    for (const void* p : ptrs)
        if ((uintptr_t)p & 15) return false;
    return true;
}

template <typename T>
hipError_t forward(const Groups& g, const Attn& a, const Bias& b, void* out, float* lse, void* ws, hipStream_t s) {
    const Lanes l = make_lanes<T>(a.H, a.D);
    Partial part = {nullptr, nullptr, parts_of(g, l.passes)};
    if (part.parts > 1) {
        part.ml = (float*)ws;
        part.acc = part.ml + (size_t)part.parts * g.rows * a.H * 2;
    }
    const int64_t waves = (int64_t)g.rows * l.passes * part.parts;
    const uint32_t blocks = grid_of(waves, kAtWaves);
    if (vectors<T>(a, {a.q, a.k, a.v, out}))
        k_at<T, true><<<blocks, kAtThreads, 0, s>>>(g, b, a, l, (T*)out, lse, part);
    else
        k_at<T, false><<<blocks, kAtThreads, 0, s>>>(g, b, a, l, (T*)out, lse, part);
    if (part.parts > 1) {
        const int64_t n = (int64_t)g.rows * a.H * a.D;
        k_at_join<T><<<grid_of(n, kAtThreads), kAtThreads, 0, s>>>(part, g.rows, a, (T*)out, lse);
    }
    return hipGetLastError();
}

template <typename T, bool VEC, bool TAB>
hipError_t back_points(const Groups& g, const Attn& a, const Bias& b, const Lanes& l, int64_t points, Magic mn,
                       const int64_t* pt_off, const int32_t* pt_center, int64_t capacity, const float* lse,
                       const float* delta, const void* dout, void* dk, void* dv, float* part, hipStream_t s) {
    if (TAB) {
        const BackShape r = back_shape(points, l.passes, b);
        hipError_t e = hipFuncSetAttribute((const void*)k_at_back_p<T, VEC, TAB>,
                                           hipFuncAttributeMaxDynamicSharedMemorySize, kAtLds);
        if (e != hipSuccess) return e;
        k_at_back_p<T, VEC, TAB><<<r.blocks, r.waves * kWave, r.lds, s>>>(
            g, b, a, l, points, mn, pt_off, pt_center, capacity, lse, delta, (const T*)dout, (T*)dk, (T*)dv, part);
    } else {
        k_at_back_p<T, VEC, TAB><<<grid_of(points * l.passes, kAtWaves), kAtThreads, 0, s>>>(
            g, b, a, l, points, mn, pt_off, pt_center, capacity, lse, delta, (const T*)dout, (T*)dk, (T*)dv, part);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t backward(const Groups& g, int32_t B, const Attn& a, const Bias& b, const int64_t* pt_off,
                    const int32_t* pt_center, int64_t capacity, const float* lse, const void* dout, void* dq, void* dk,
                    void* dv, float* dtable, float* dslope, void* ws, hipStream_t s) {
    const Lanes lc = make_lanes<T>(a.H, a.D), lp = make_lanes<T>(a.Hkv, a.D);
    const int64_t points = (int64_t)B * g.N;
    float* delta = (float*)ws;
    float* part = (float*)((char*)ws + align256((size_t)g.rows * a.H * 4));
    const bool vec = vectors<T>(a, {a.q, a.k, a.v, dout, dq, dk, dv});
    const uint32_t blocks = grid_of((int64_t)g.rows * lc.passes, kAtWaves);
    if (vec)
        k_at_back_c<T, true><<<blocks, kAtThreads, 0, s>>>(g, b, a, lc, lse, (const T*)dout, (T*)dq, delta);
    else
        k_at_back_c<T, false><<<blocks, kAtThreads, 0, s>>>(g, b, a, lc, lse, (const T*)dout, (T*)dq, delta);
    const bool tab = dtable || dslope;
    const Magic mn = make_magic((uint32_t)g.N);
    auto f = vec ? (tab ? back_points<T, true, true> : back_points<T, true, false>)
                 : (tab ? back_points<T, false, true> : back_points<T, false, false>);
    hipError_t e = f(g, a, b, lp, points, mn, pt_off, pt_center, capacity, lse, delta, dout, dk, dv, part, s);
    if (e != hipSuccess || !tab) return e;
    return launch_bias_reduce(part, back_shape(points, lp.passes, b).blocks, b, dtable, dslope, s);
}

}  // namespace

size_t group_attention_bytes(const Groups& g, int32_t B, const Attn& a, int32_t dtype, const Bias& b, bool backward) {
    if (!backward) {
        const int32_t parts = parts_of(g, lanes_passes(dtype, a.H, a.D));
        return parts > 1 ? (size_t)parts * g.rows * a.H * (2 + a.D) * 4 : 0;
    }
    const size_t delta = align256((size_t)g.rows * a.H * 4);
    if (b.nb == 0 && !b.slope) return delta;
    return delta + (size_t)back_shape((int64_t)B * g.N, lanes_passes(dtype, a.Hkv, a.D), b).blocks *
                       (3 * b.nb + 1) * b.H * 4;
}

hipError_t launch_group_attention(const Groups& g, const Attn& a, int32_t dtype, const Bias& b, void* out, float* lse,
                                  void* ws, hipStream_t s) {
    if (dtype == CAGQ_F32) return forward<float>(g, a, b, out, lse, ws, s);
    if (dtype == CAGQ_BF16) return forward<bf16>(g, a, b, out, lse, ws, s);
    return forward<f16>(g, a, b, out, lse, ws, s);
}

hipError_t launch_group_attention_backward(const Groups& g, int32_t B, const Attn& a, int32_t dtype, const Bias& b,
                                           const int64_t* pt_off, const int32_t* pt_center, int64_t capacity,
                                           const float* lse, const void* dout, void* dq, void* dk, void* dv,
                                           float* dtable, float* dslope, void* ws, hipStream_t s) {
    auto f = dtype == CAGQ_F32 ? backward<float> : dtype == CAGQ_BF16 ? backward<bf16> : backward<f16>;
    return f(g, B, a, b, pt_off, pt_center, capacity, lse, dout, dq, dk, dv, dtable, dslope, ws, s);
}

}  // namespace cagq
