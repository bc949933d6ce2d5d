// The relative position bias alone, and its gradient (cagq_relative_bias,
// cagq_relative_bias_backward; the definition is in include/cagq.h).
// Indoor scenes (2^20 slots, 8 heads in bfloat16): 17 us for the bias, of which
// 16.8 MB of stores and 13 MB of reads would take 6 at the card's copy rate. It
// reads 37 MB past the L2, which with the stores makes 11 of it; a lane's searches
// in the edges and its three table rows in LDS are the rest. The gradient takes 44
// us and the sum over its workgroups' tables 7.
#include "cagq_features.h"

namespace cagq {

namespace {

constexpr int kRbThreads = 256;
constexpr int kRbMost = 256;       // threads of a workgroup of the gradient
constexpr int kRbParts = 1024;     // workgroups of the gradient, each with partial sums of its own
constexpr int kRbLds = 128 << 10;  // LDS of their tables, one per wave for 16 heads
constexpr int kRedThreads = 1024;

// A slot is a lane's: fixed groups 64 slots in a row to a wave, ragged ones a
// group to a wave, 64 slots at a time. f(slot, u, dist, counts) for every lane
// with a slot.
template <typename F>
__device__ __forceinline__ void each_slot(const Groups& g, const PlaceBias& pb, Magic by_k, F f) {
    const int lane = lane_id();
    const int waves_b = blockDim.x / kWave;
    const int64_t waves = (int64_t)gridDim.x * waves_b;
    const int64_t w0 = (int64_t)blockIdx.x * waves_b + threadIdx.x / kWave;
    auto slot = [&](int64_t s, int32_t row, bool counts) {
        uint32_t u = 0;
        float dist = 0.0f;
        if (counts) {
            const int32_t i = g.idx[s];
            counts = (uint32_t)i < (uint32_t)g.N;
            if (counts) {
                float p[3], c[3];
                load_xyz(g.points, (int64_t)udiv((uint32_t)row, g.mm) * g.N + i, p);
                load_xyz(g.centers, row, c);
                pair_place(pb.ed, pb.dist, p, c, u, dist);
            }
        }
        f(s, u, dist, counts);
    };
    if (g.K > 0) {
        for (int64_t s = w0 * kWave + lane; s < g.idx_len; s += waves * kWave) {
            const int32_t row = (int32_t)udiv((uint32_t)s, by_k);
            int32_t n = g.K;
            if (g.n_valid) n = g.n_valid[row];
            slot(s, row, (int32_t)(s - (int64_t)row * g.K) < n);
        }
    } else {
        for (int64_t row = w0; row < g.rows; row += waves) {
            int64_t beg, end;
            g.range((int32_t)row, beg, end);
            for (int64_t s = beg + lane; s < end; s += kWave) slot(s, (int32_t)row, true);
        }
    }
}

// V heads at once: V of the slot's heads lie 16-byte aligned (V: what 16 bytes
// hold), or V = 1.
template <typename T, int V>
__global__ __launch_bounds__(kRbThreads) void k_rb(Groups g, Bias b, Magic by_k, T* __restrict__ out) {
    extern __shared__ __align__(16) float s_lds[];
    const PlaceBias pb(b, s_lds);
    each_slot(g, pb, by_k, [&](int64_t s, uint32_t u, float dist, bool counts) {
        T* o = out + s * b.H;
        if constexpr (V == 1) {
            for (int h = 0; h < b.H; ++h) o[h] = (T)(counts ? pb.one(u, dist, h) : 0.0f);
        } else {
            for (int h = 0; h < b.H; h += V) {
                float x[V] = {};
                if (counts) {
#pragma unroll
                    for (int i = 0; i < V; i += 4) {
                        const f32x4 y = pb.four(u, dist, h + i);
                        x[i] = y[0], x[i + 1] = y[1], x[i + 2] = y[2], x[i + 3] = y[3];
                    }
                }
                store_channels<T, true>(o + h, V, x);
            }
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

// The gradient is a product: the table's is (bucket one-hot) x dbias, summed
// over the slots, one for each axis, and the slope's a row of distances x
// dbias. The matrix units take it, 32 slots at a time: 16 rows of buckets
// (TA such tiles an axis) x 32 slots times 32 slots x 16 heads. bfloat16
// operands lose nothing: a one-hot is 0 or 1, and a value of a wider type goes
// in as the exact sum of two (float16) or three (float32, distances) of them.
// Values that are not finite, which would meet the zeros, go by LDS adds
// instead. (Adding every slot's heads to a table in LDS: 64 lanes meet in a few
// buckets, 180 cycles an instruction: 185 us for the indoor scenes' 2^20 slots
// and 8 heads in bfloat16, where this takes 42.)
// Few large workgroups: their tables are what the sum over all of them reads.
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kNoSlot = 0xFFFFFFFFu;  // no bucket is 255

template <typename T>
constexpr int kSplits = sizeof(T) == 4 ? 3 : __is_same(T, f16) ? 2 : 1;

// x as a sum of N bfloat16, exactly: the top 8 bits of what is left each time.
template <int N>
__device__ __forceinline__ void split(float x, uint32_t (&hi)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        hi[i] = __float_as_uint(x) & 0xFFFF0000u;
        x -= __uint_as_float(hi[i]);
    }
}

// Eight of them, the upper halves of a, as an operand.
__device__ __forceinline__ bf16x8 pack8(const uint32_t (&a)[8]) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (a[2 * i] >> 16) | a[2 * i + 1];
    return __builtin_bit_cast(bf16x8, r);
}

template <typename T, int TA>
__global__ __launch_bounds__(kRbMost, 4) void k_rb_back(Groups g, Bias b, Magic by_k, const T* __restrict__ dbias,
                                                     float* __restrict__ part) {
    constexpr int NS = kSplits<T>;
    constexpr int TN = TA > 0 ? 3 * TA : 1;
    extern __shared__ __align__(16) float s_lds[];
    const PlaceBias pb(b, s_lds, false);
    const int lane = lane_id(), wave = threadIdx.x / kWave, waves_b = blockDim.x / kWave;
    const int h0 = (int)blockIdx.y * 16, nh = b.H - h0 < 16 ? b.H - h0 : 16;
    const int rows = 3 * b.nb + 1, cells = rows * 16;
    float* s_odd = s_lds + PlaceBias::floats(b, false);       // [rows][16]: what is not finite
    float* s_place = s_odd + cells + wave * 2 * kWave;        // [64] places, [64] distances
    float* s_sum = s_odd + cells + waves_b * 2 * kWave;       // [wave][rows][16]
    for (int e = threadIdx.x; e < cells; e += blockDim.x) s_odd[e] = 0.0f;
    __syncthreads();
    f32x4_t acc[TN] = {}, accd = {};
    const int col = lane & 15, k0 = (lane >> 4) * 8;

    auto chunk = [&](int64_t s0, int n, int32_t row, bool counts) {  // slots s0 .. s0 + n, the lane's own and its row
        float v[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int k = (j >> 3) * 32 + k0 + (j & 7);
            v[j] = k < n && col < nh ? to_float(dbias[(s0 + k) * b.H + h0 + col]) : 0.0f;
        }
        uint32_t u = kNoSlot;
        float dist = 0.0f;
        if (counts) {
            const int32_t i = g.idx[s0 + lane];
            if ((uint32_t)i < (uint32_t)g.N) {
                float p[3], c[3];
                load_xyz(g.points, (int64_t)udiv((uint32_t)row, g.mm) * g.N + i, p);
                load_xyz(g.centers, row, c);
                pair_place(pb.ed, pb.dist, p, c, u, dist);
            }
        }
        s_place[lane] = __uint_as_float(u);
        s_place[kWave + lane] = dist;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t pu[8], w[8][NS];
            float d[8];
            bool odd = false;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                pu[j] = __float_as_uint(s_place[half * 32 + k0 + j]);
                d[j] = s_place[kWave + half * 32 + k0 + j];
                float x = pu[j] == kNoSlot ? 0.0f : v[half * 8 + j];
                odd = odd || !(fabsf(x) < __builtin_inff());
                v[half * 8 + j] = x;
            }
            if (__any(odd)) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    float& x = v[half * 8 + j];
                    if (fabsf(x) < __builtin_inff()) continue;
                    if (TA > 0) {
                        atomicAdd(&s_odd[pb.x_row(pu[j]) * 16 + col], x);
                        atomicAdd(&s_odd[pb.y_row(pu[j]) * 16 + col], x);
                        atomicAdd(&s_odd[pb.z_row(pu[j]) * 16 + col], x);
                    }
                    atomicAdd(&s_odd[3 * b.nb * 16 + col], x * d[j]);
                    x = 0.0f;
                    if (!(fabsf(d[j]) < __builtin_inff())) d[j] = 0.0f;  // added, and not once more below
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) split<NS>(v[half * 8 + j], w[j]);
            bf16x8 val[NS];
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                uint32_t t[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] = w[j][i];
                val[i] = pack8(t);
            }
            if constexpr (TA > 0) {
#pragma unroll
                for (int a = 0; a < 3; ++a) {
                    int r[8];  // the slot's bucket, from the lane's row of the first tile on
#pragma unroll
                    for (int j = 0; j < 8; ++j) r[j] = (int)(pu[j] >> (8 * a) & 255u) - col;
#pragma unroll
                    for (int t = 0; t < TA; ++t) {
                        uint32_t one[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) one[j] = r[j] == 16 * t ? 0x3F800000u : 0u;
                        const bf16x8 hot = pack8(one);
#pragma unroll
                        for (int i = 0; i < NS; ++i)
                            acc[a * TA + t] =
                                __builtin_amdgcn_mfma_f32_16x16x32_bf16(hot, val[i], acc[a * TA + t], 0, 0, 0);
                    }
                }
            }
            if (pb.dist) {  // rows 0 to 2: the distance's three parts
                uint32_t t[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    uint32_t w3[3];
                    split<3>(fabsf(d[j]) < __builtin_inff() ? d[j] : 0.0f, w3);
                    t[j] = col == 0 ? w3[0] : col == 1 ? w3[1] : col == 2 ? w3[2] : 0u;
                }
                const bf16x8 far = pack8(t);
#pragma unroll
                for (int i = 0; i < NS; ++i)
                    accd = __builtin_amdgcn_mfma_f32_16x16x32_bf16(far, val[i], accd, 0, 0, 0);
                // a distance that is not finite
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (!(fabsf(d[j]) < __builtin_inff()) && pu[j] != kNoSlot && col < nh)
                        atomicAdd(&s_odd[3 * b.nb * 16 + col], d[j] * v[half * 8 + j]);
            }
        }
        __builtin_amdgcn_wave_barrier();
    };

    const int64_t waves = (int64_t)gridDim.x * waves_b;
    const int64_t w0 = (int64_t)blockIdx.x * waves_b + wave;
    if (g.K > 0) {
        for (int64_t s0 = w0 * kWave; s0 < g.idx_len; s0 += waves * kWave) {
            const int n = g.idx_len - s0 < kWave ? (int)(g.idx_len - s0) : kWave;
            const int64_t s = s0 + (lane < n ? lane : 0);
            const int32_t row = (int32_t)udiv((uint32_t)s, by_k);
            const int32_t nv = g.n_valid ? g.n_valid[row] : g.K;
            chunk(s0, n, row, lane < n && (int32_t)(s - (int64_t)row * g.K) < nv);
        }
    } else {
        for (int64_t row = w0; row < g.rows; row += waves) {
            int64_t beg, end;
            g.range((int32_t)row, beg, end);
            for (int64_t s0 = beg; s0 < end; s0 += kWave) {
                const int n = end - s0 < kWave ? (int)(end - s0) : kWave;
                chunk(s0, n, (int32_t)row, lane < n);
            }
        }
    }
    // the wave's sums: element r of a tile is row 4 (lane / 16) + r, column lane % 16
    float* mine = s_sum + wave * cells;
    if constexpr (TA > 0) {
#pragma unroll
        for (int t = 0; t < TN; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int u = (t % TA) * 16 + (lane >> 4) * 4 + r;
                if (u < b.nb) mine[((t / TA) * b.nb + u) * 16 + col] = acc[t][r];
            }
    }
    if (lane < 16) mine[3 * b.nb * 16 + col] = (accd[0] + accd[1]) + accd[2];
    __syncthreads();
    const int entries = rows * b.H;
    for (int e = threadIdx.x; e < rows * nh; e += blockDim.x) {
        const int r = e / nh, h = e - r * nh;
        float x = s_odd[r * 16 + h];
        for (int w = 0; w < waves_b; ++w) x += s_sum[w * cells + r * 16 + h];
        part[(int64_t)blockIdx.x * entries + r * b.H + h0 + h] = x;
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
    const size_t cells = (size_t)(3 * b.nb + 1) * 16;
    const size_t base = (PlaceBias::floats(b, false) + cells) * 4, per = (2 * kWave + cells) * 4;
    const int64_t work = g.K > 0 ? (g.idx_len + kWave - 1) / kWave : g.rows;
    r.waves = kRbMost / kWave;
    while (r.waves > 1 && (base + per * r.waves > kRbLds || work < (int64_t)kRbParts * r.waves / 2)) r.waves >>= 1;
    r.lds = base + per * r.waves;
    const int64_t blocks = (work + r.waves - 1) / r.waves;
    r.parts = (int)(blocks < 1 ? 1 : blocks > kRbParts ? kRbParts : blocks);
    return r;
}

template <typename T>
bool rb_vectors(const Bias& b, const void* p) {
    return b.H % kVec<T> == 0 && ((uintptr_t)p & 15) == 0;
}

template <typename T>
hipError_t rb_forward(const Groups& g, const Bias& b, void* out, hipStream_t s) {
    const int64_t work = g.K > 0 ? (g.idx_len + kWave - 1) / kWave : g.rows;
    const int waves = kRbThreads / kWave;
    int64_t blocks = (work + waves - 1) / waves;
    blocks = blocks < 1 ? 1 : blocks > 2048 ? 2048 : blocks;
    const Magic by_k = make_magic(g.K > 0 ? (uint32_t)g.K : 1u);
    const size_t lds = (size_t)PlaceBias::floats(b) * 4;
    auto kern = rb_vectors<T>(b, out) ? k_rb<T, kVec<T>> : k_rb<T, 1>;
    kern<<<(uint32_t)blocks, kRbThreads, lds, s>>>(g, b, by_k, (T*)out);
    if (g.K == 0) k_rb_outside<T><<<64, kRbThreads, 0, s>>>(g, b.H, (T*)out);
    return hipGetLastError();
}

template <typename T>
hipError_t rb_backward(const Groups& g, const Bias& b, const void* dbias, float* dtable, float* dslope, void* ws,
                       hipStream_t s) {
    const RbShape r = rb_shape(g, b);
    const Magic by_k = make_magic(g.K > 0 ? (uint32_t)g.K : 1u);
    const int ta = (b.nb + 15) / 16;
    auto kern = ta == 0 ? k_rb_back<T, 0> : ta == 1 ? k_rb_back<T, 1> : ta == 2 ? k_rb_back<T, 2>
                : ta == 3 ? k_rb_back<T, 3> : k_rb_back<T, 4>;
    hipError_t e = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, kRbLds);
    if (e != hipSuccess) return e;
    kern<<<dim3(r.parts, (b.H + 15) / 16), r.waves * kWave, r.lds, s>>>(g, b, by_k, (const T*)dbias, (float*)ws);
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
