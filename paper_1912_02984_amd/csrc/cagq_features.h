// What the operators on point features share (attention over groups, the
// turned groups, the relative position bias): the groups as the kernels see
// them, feature types, the place of a pair in the bias, and how a wave's
// lanes are laid over rows of heads.
#pragma once

#include "cagq_internal.h"

namespace cagq {

// cagq_groups as the kernels take it.
struct Groups {
    const int32_t* idx;
    const int32_t* n_valid;
    const int64_t* off;
    const float* points;
    const float* centers;
    int64_t idx_len;  // slots
    int32_t N, M, K;
    int32_t rows;     // B * M
    Magic mm;         // division by M

    // Slots [beg, end) of group `row` that count.
    __device__ __forceinline__ void range(int32_t row, int64_t& beg, int64_t& end) const {
        if (K > 0) {
            beg = (int64_t)row * K;
            int32_t n = K;
            if (n_valid) {
                n = n_valid[row];
                n = n < 0 ? 0 : n > K ? K : n;
            }
            end = beg + n;
        } else {
            beg = off[row];
            end = off[row + 1];
            beg = beg < 0 ? 0 : beg > idx_len ? idx_len : beg;
            end = end < beg ? beg : end > idx_len ? idx_len : end;
        }
    }
};

// cagq_bias as the kernels take it.
struct Bias {
    const float* table;
    const float* edges;
    const float* slope;
    int32_t nb;  // buckets (0: no table)
    int32_t H;
};

// ------------------------------------------------------------------ feature types

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16;
typedef _Float16 f16;

// Channels a lane holds of a head: 16 bytes of features.
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(f16 x) { return (float)x; }
__device__ __forceinline__ float to_float(bf16 x) {
    return __uint_as_float((uint32_t)__builtin_bit_cast(uint16_t, x) << 16);
}

// n channels (of kVec) at p; the others are 0. VEC: p is 16-byte aligned and
// all kVec channels are there (or none is wanted, n = 0).
template <typename T, bool VEC>
__device__ __forceinline__ void load_channels(const T* p, int n, float (&x)[kVec<T>]) {
    constexpr int W = kVec<T>;
    if constexpr (VEC) {
        u32x4 r = {0, 0, 0, 0};
        if (n > 0) r = *reinterpret_cast<const u32x4*>(p);
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(r[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = to_float(__builtin_bit_cast(T, (uint16_t)(r[i] & 0xFFFFu)));
                x[2 * i + 1] = to_float(__builtin_bit_cast(T, (uint16_t)(r[i] >> 16)));
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) x[i] = i < n ? to_float(p[i]) : 0.0f;
    }
}

// The one rounding to the features' type, to nearest even.
template <typename T, bool VEC>
__device__ __forceinline__ void store_channels(T* p, int n, const float (&x)[kVec<T>]) {
    constexpr int W = kVec<T>;
    if constexpr (VEC) {
        if (n <= 0) return;
        u32x4 r;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(x[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                r[i] = (uint32_t)__builtin_bit_cast(uint16_t, (T)x[2 * i]) |
                       (uint32_t)__builtin_bit_cast(uint16_t, (T)x[2 * i + 1]) << 16;
        }
        *reinterpret_cast<u32x4*>(p) = r;
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < n) p[i] = (T)x[i];
    }
}

__device__ __forceinline__ float xlane_f(float v, int j) { return __uint_as_float(xlane(__float_as_uint(v), j)); }

// Sum over groups of G lanes (a power of two, the same for the launch), in
// every lane of the group.
__device__ __forceinline__ float group_sum(float v, int G) {
    if (G > 1) v += xlane_f(v, 1);
    if (G > 2) v += xlane_f(v, 2);
    if (G > 4) v += xlane_f(v, 4);
    if (G > 8) v += xlane_f(v, 8);
    if (G > 16) v += xlane_f(v, 16);
    if (G > 32) v += xlane_f(v, 32);
    return v;
}

// ------------------------------------------------------------------ the bias of a pair

// Number of the n ascending edges that are <= d (n < CAGQ_MAX_BUCKETS).
__device__ __forceinline__ uint32_t bucket_of(const float* edges, int n, float d) {
    uint32_t u = 0;
#pragma unroll
    for (int s = CAGQ_MAX_BUCKETS / 2; s > 0; s >>= 1)
        if ((int)u + s <= n && edges[u + s - 1] <= d) u += s;
    return u;
}

// Where a pair lies: its buckets on the axes, a byte each, and its distance.
// `edges`: [3][nb - 1], global memory or LDS.
__device__ __forceinline__ void pair_place(const float* edges, int nb, bool want_dist, const float (&p)[3],
                                           const float (&c)[3], uint32_t& u, float& dist) {
    const float dx = p[0] - c[0], dy = p[1] - c[1], dz = p[2] - c[2];
    u = 0;
    dist = 0.0f;
    if (nb > 1) {
        const int n = nb - 1;
        u = bucket_of(edges, n, dx) | bucket_of(edges + n, n, dy) << 8 | bucket_of(edges + 2 * n, n, dz) << 16;
    }
    if (want_dist) dist = sqrtf((dx * dx + dy * dy) + dz * dz);
}

// Bias of head h at a place. `table`: [3][nb][H], global memory or LDS.
__device__ __forceinline__ float bias_at(const float* table, int nb, int H, float slope, int h, uint32_t u,
                                         float dist) {
    float b = 0.0f;
    if (nb > 0) {
        const float x = table[(u & 255u) * H + h];
        const float y = table[(nb + (u >> 8 & 255u)) * H + h];
        const float z = table[(2 * nb + (u >> 16)) * H + h];
        b = x + y + z;
    }
    return fmaf(slope, dist, b);
}

__device__ __forceinline__ void load_xyz(const float* p, int64_t i, float (&x)[3]) {
    x[0] = p[3 * i];
    x[1] = p[3 * i + 1];
    x[2] = p[3 * i + 2];
}

// LDS sum without a return value. A wave's own LDS operations run in order,
// and lanes of one instruction that meet in a word are added in a fixed
// order, so a table that one wave alone adds to does not vary from run to run.
__device__ __forceinline__ void lds_add(float* p, float v) {
    __hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT);
}

// ------------------------------------------------------------------ launches

hipError_t launch_point_lists(const Groups& g, int32_t B, int64_t* pt_off, int32_t* pt_center, int64_t capacity,
                              void* ws, hipStream_t s);
size_t point_lists_bytes(const Groups& g, int32_t B);

// The gradient of the bias: the partial sums of `parts` workgroups, entry e of
// part p at part[p * entries + e] (entries = 3 nb H table sums, then H slope
// sums), added up in the order of the parts.
hipError_t launch_bias_reduce(const float* part, int32_t parts, const Bias& b, float* dtable, float* dslope,
                              hipStream_t s);
size_t relative_bias_bytes(const Groups& g, const Bias& b);
hipError_t launch_relative_bias(const Groups& g, const Bias& b, int32_t dtype, void* out, hipStream_t s);
hipError_t launch_relative_bias_backward(const Groups& g, const Bias& b, int32_t dtype, const void* dbias,
                                         float* dtable, float* dslope, void* ws, hipStream_t s);

struct Attn {
    const void* q;
    const void* k;
    const void* v;
    int64_t q_row, k_row, v_row;
    int32_t H, Hkv, D;
    float scale, cap;
};

size_t group_attention_bytes(const Groups& g, int32_t B, const Attn& a, int32_t dtype, const Bias& b, bool backward);
hipError_t launch_group_attention(const Groups& g, const Attn& a, int32_t dtype, const Bias& b, void* out, float* lse,
                                  void* ws, hipStream_t s);
hipError_t launch_group_attention_backward(const Groups& g, int32_t B, const Attn& a, int32_t dtype, const Bias& b,
                                           const int64_t* pt_off, const int32_t* pt_center, int64_t capacity,
                                           const float* lse, const void* dout, void* dq, void* dk, void* dv,
                                           float* dtable, float* dslope, void* ws, hipStream_t s);

}  // namespace cagq
