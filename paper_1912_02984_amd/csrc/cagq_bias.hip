// The relative position bias alone, and its gradient (cagq_relative_bias,
// cagq_relative_bias_backward; the definition is in include/cagq.h).
#include "cagq_features.h"

namespace cagq {

namespace {

constexpr int kRbThreads = 256;
constexpr int kRbWaves = kRbThreads / kWave;
constexpr int kRedThreads = 1024;
constexpr int kRbParts = 1024;   // workgroups of the gradient, each with partial sums of its own
constexpr int kRbLds = 128 << 10;  // LDS of their tables, a table per wave

// Fixed groups: 64 slots in a row are a wave's. Ragged ones: a group is a
// wave's, 64 slots at a time. f(first slot, number of slots, row, u, dist,
// counts) with the lane's own slot's row, place and whether it counts.
template <typename F>
__device__ __forceinline__ void each_chunk(const Groups& g, const Bias& b, const Edges& ed, F f) {
    const int lane = lane_id();
    const int waves_b = blockDim.x / kWave;
    const int64_t waves = (int64_t)gridDim.x * waves_b;
    const int64_t w0 = (int64_t)blockIdx.x * waves_b + threadIdx.x / kWave;
    auto chunk = [&](int64_t s0, int n, int64_t s, int32_t row, bool counts) {
        uint32_t u = 0;
        float dist = 0.0f;
        if (counts) {
            const int32_t i = g.idx[s];
            counts = (uint32_t)i < (uint32_t)g.N;
            if (counts) {
                float p[3], c[3];
                load_xyz(g.points, (int64_t)udiv((uint32_t)row, g.mm) * g.N + i, p);
                load_xyz(g.centers, row, c);
                pair_place(ed, b.slope != nullptr, p, c, u, dist);
            }
        }
        f(s0, n, u, dist, counts);
    };
    if (g.K > 0) {
        for (int64_t s0 = w0 * kWave; s0 < g.idx_len; s0 += waves * kWave) {
            const int n = g.idx_len - s0 < kWave ? (int)(g.idx_len - s0) : kWave;
            const int64_t s = s0 + (lane < n ? lane : 0);
            const int32_t row = (int32_t)(s / g.K);
            int64_t beg, end;
            g.range(row, beg, end);
            chunk(s0, n, s, row, lane < n && s < end);
        }
    } else {
        for (int64_t row = w0; row < g.rows; row += waves) {
            int64_t beg, end;
            g.range((int32_t)row, beg, end);
            for (int64_t s0 = beg; s0 < end; s0 += kWave) {
                const int n = end - s0 < kWave ? (int)(end - s0) : kWave;
                chunk(s0, n, s0 + lane, (int32_t)row, lane < n);
            }
        }
    }
}

template <typename T>
__global__ __launch_bounds__(kRbThreads) void k_rb(Groups g, Bias b, T* __restrict__ out) {
    __shared__ float s_edges[3 * (CAGQ_MAX_BUCKETS - 1)];
    const int lane = lane_id();
    const Edges ed = stage_edges(b, s_edges);
    __syncthreads();
    each_chunk(g, b, ed, [&](int64_t s0, int n, uint32_t u, float dist, bool counts) {
        const uint64_t live = __ballot(counts);
        for (int e = lane; e < ((n * b.H + kWave - 1) & -kWave); e += kWave) {
            const int p = e / b.H, h = e - p * b.H;
            const uint32_t pu = (uint32_t)__shfl((int)u, p & 63, kWave);
            const float pd = __shfl(dist, p & 63, kWave);
            if (p >= n) continue;
            float x = 0.0f;
            if (live >> p & 1) x = bias_at(b.table, b.nb, b.H, b.slope ? b.slope[h] : 0.0f, h, pu, pd);
            out[s0 * b.H + e] = (T)x;
        }
    });
}

// Ragged entries outside every group.
template <typename T>
__global__ __launch_bounds__(kRbThreads) void k_rb_outside(Groups g, int32_t H, T* __restrict__ out) {
    int64_t first, x, last;
    g.range(0, first, x);
    g.range(g.rows - 1, x, last);
    const int64_t step = (int64_t)gridDim.x * kRbThreads;
    for (int64_t e = (int64_t)blockIdx.x * kRbThreads + threadIdx.x; e < first * H; e += step) out[e] = (T)0.0f;
    for (int64_t e = last * H + (int64_t)blockIdx.x * kRbThreads + threadIdx.x; e < g.idx_len * H; e += step)
        out[e] = (T)0.0f;
}

// A wave adds its slots into a table of its own in LDS; the workgroup's tables
// are added up in the order of its waves.
template <typename T>
__global__ __launch_bounds__(kRbThreads) void k_rb_back(Groups g, Bias b, const T* __restrict__ dbias,
                                                        float* __restrict__ part) {
    extern __shared__ float s_tab[];
    __shared__ float s_edges[3 * (CAGQ_MAX_BUCKETS - 1)];
    const int lane = lane_id();
    const Edges ed = stage_edges(b, s_edges);
    const int entries = (3 * b.nb + 1) * b.H;
    const int waves_b = blockDim.x / kWave;
    for (int e = threadIdx.x; e < entries * waves_b; e += blockDim.x) s_tab[e] = 0.0f;
    __syncthreads();
    float* tab = s_tab + (threadIdx.x / kWave) * entries;
    each_chunk(g, b, ed, [&](int64_t s0, int n, uint32_t u, float dist, bool counts) {
        const uint64_t live = __ballot(counts);
        for (int e = lane; e < ((n * b.H + kWave - 1) & -kWave); e += kWave) {
            const int p = e / b.H, h = e - p * b.H;
            const uint32_t pu = (uint32_t)__shfl((int)u, p & 63, kWave);
            const float pd = __shfl(dist, p & 63, kWave);
            if (p >= n || !(live >> p & 1)) continue;
            const float x = to_float(dbias[s0 * b.H + e]);
            if (b.nb > 0) {
                lds_add(&tab[(pu & 255u) * b.H + h], x);
                lds_add(&tab[(b.nb + (pu >> 8 & 255u)) * b.H + h], x);
                lds_add(&tab[(2 * b.nb + (pu >> 16)) * b.H + h], x);
            }
            if (b.slope) lds_add(&tab[3 * b.nb * b.H + h], x * pd);
        }
    });
    __syncthreads();
    for (int e = threadIdx.x; e < entries; e += blockDim.x) {
        float x = 0.0f;
        for (int w = 0; w < waves_b; ++w) x += s_tab[w * entries + e];
        part[(int64_t)blockIdx.x * entries + e] = x;
    }
}

// Waves of a workgroup take the parts in turn, their lanes 64 entries in a row.
__global__ __launch_bounds__(kRedThreads) void k_bias_reduce(const float* __restrict__ part, int32_t parts,
                                                             int entries, int tab, float* __restrict__ dtable,
                                                             float* __restrict__ dslope) {
    constexpr int kWaves = kRedThreads / kWave;
    __shared__ float s[kWaves][kWave];
    const int lane = lane_id(), w = threadIdx.x / kWave;
    const int e = blockIdx.x * kWave + lane;
    float x[4] = {};
    if (e < entries) {
        int p = w;
        for (; p + 3 * kWaves < parts; p += 4 * kWaves) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] += part[(int64_t)(p + i * kWaves) * entries + e];
        }
        for (; p < parts; p += kWaves) x[0] += part[(int64_t)p * entries + e];
    }
    s[w][lane] = (x[0] + x[1]) + (x[2] + x[3]);
    __syncthreads();
    if (w > 0 || e >= entries) return;
    float sum = 0.0f;
    for (int i = 0; i < kWaves; ++i) sum += s[i][lane];
    if (e < tab) {
        if (dtable) dtable[e] = sum;
    } else if (dslope) {
        dslope[e - tab] = sum;
    }
}

// Waves of a workgroup whose tables fit its LDS, and the workgroups.
struct RbShape {
    int waves, parts;
    size_t lds;
};

RbShape rb_shape(const Groups& g, const Bias& b) {
    RbShape r;
    const size_t entries = (size_t)(3 * b.nb + 1) * b.H;
    r.waves = kRbWaves;
    while (r.waves > 1 && entries * 4 * r.waves > kRbLds) r.waves >>= 1;
    r.lds = entries * 4 * r.waves;
    const int64_t work = g.K > 0 ? (g.idx_len + kWave - 1) / kWave : g.rows;
    const int64_t blocks = (work + r.waves - 1) / r.waves;
    r.parts = (int)(blocks < 1 ? 1 : blocks > kRbParts ? kRbParts : blocks);
    return r;
}

template <typename T>
hipError_t rb_forward(const Groups& g, const Bias& b, void* out, hipStream_t s) {
    const int64_t work = g.K > 0 ? (g.idx_len + kWave - 1) / kWave : g.rows;
    int64_t blocks = (work + kRbWaves - 1) / kRbWaves;
    blocks = blocks < 1 ? 1 : blocks > 65536 ? 65536 : blocks;
    k_rb<T><<<(uint32_t)blocks, kRbThreads, 0, s>>>(g, b, (T*)out);
    if (g.K == 0) k_rb_outside<T><<<64, kRbThreads, 0, s>>>(g, b.H, (T*)out);
    return hipGetLastError();
}

template <typename T>
hipError_t rb_backward(const Groups& g, const Bias& b, const void* dbias, float* dtable, float* dslope, void* ws,
                       hipStream_t s) {
    const RbShape r = rb_shape(g, b);
    hipError_t e = hipFuncSetAttribute((const void*)k_rb_back<T>, hipFuncAttributeMaxDynamicSharedMemorySize, kRbLds);
    if (e != hipSuccess) return e;
    k_rb_back<T><<<r.parts, r.waves * kWave, r.lds, s>>>(g, b, (const T*)dbias, (float*)ws);
    return launch_bias_reduce((const float*)ws, r.parts, b, dtable, dslope, s);
}

}  // namespace

hipError_t launch_bias_reduce(const float* part, int32_t parts, const Bias& b, float* dtable, float* dslope,
                              hipStream_t s) {
    const int entries = (3 * b.nb + 1) * b.H;
    k_bias_reduce<<<(entries + kWave - 1) / kWave, kRedThreads, 0, s>>>(part, parts, entries, 3 * b.nb * b.H, dtable,
                                                                        b.slope ? dslope : nullptr);
    return hipGetLastError();
}

size_t relative_bias_bytes(const Groups& g, const Bias& b) {
    return (size_t)rb_shape(g, b).parts * (3 * b.nb + 1) * b.H * sizeof(float);
}

hipError_t launch_relative_bias(const Groups& g, const Bias& b, int32_t dtype, void* out, hipStream_t s) {
    if (dtype == CAGQ_F32) return rb_forward<float>(g, b, out, s);
    if (dtype == CAGQ_BF16) return rb_forward<bf16>(g, b, out, s);
    return rb_forward<f16>(g, b, out, s);
}

hipError_t launch_relative_bias_backward(const Groups& g, const Bias& b, int32_t dtype, const void* dbias,
                                         float* dtable, float* dslope, void* ws, hipStream_t s) {
    if (dtype == CAGQ_F32) return rb_backward<float>(g, b, dbias, dtable, dslope, ws, s);
    if (dtype == CAGQ_BF16) return rb_backward<bf16>(g, b, dbias, dtable, dslope, ws, s);
    return rb_backward<f16>(g, b, dbias, dtable, dslope, ws, s);
}

}  // namespace cagq
