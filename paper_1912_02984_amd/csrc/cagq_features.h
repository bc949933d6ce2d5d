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

// The 16 bytes of a lane's channels as they are stored, so that products of
// bfloat16 can be taken two at a time.
typedef u32x4 Raw;

// n channels (of kVec) at p; the others are 0. VEC: p is 16-byte aligned and
// all kVec channels are there (or none is wanted, n = 0).
template <typename T, bool VEC>
__device__ __forceinline__ Raw load_channels(const T* p, int n) {
    Raw r = {0, 0, 0, 0};
    if constexpr (VEC) {
        if (n > 0) r = *reinterpret_cast<const u32x4*>(p);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) r[i] = __builtin_bit_cast(uint32_t, p[i]);
    } else {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) r[i / 2] |= (uint32_t)h[i] << (16 * (i & 1));
    }
    return r;
}

// Channel i (known at compile time) as a float.
template <typename T>
__device__ __forceinline__ float channel(const Raw& r, int i) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(r[i]);
    else if constexpr (__is_same(T, bf16))
        return __uint_as_float(i & 1 ? r[i / 2] & 0xFFFF0000u : r[i / 2] << 16);
    else
        return (float)__builtin_bit_cast(f16, (uint16_t)(i & 1 ? r[i / 2] >> 16 : r[i / 2] & 0xFFFFu));
}

// The lane's part of a product of two heads. bfloat16: two products and the
// sum in one instruction (v_dot2_f32_bf16, within 2^-24 of the products'
// magnitudes on subnormal inputs too). float16: one by one, mixed with fp32
// (v_dot2_f32_f16 was off by 35 * 2^-24 with subnormal inputs).
template <typename T>
__device__ __forceinline__ float dot(const Raw& a, const Raw& b) {
    float s = 0.0f;
    if constexpr (__is_same(T, bf16)) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (uint32_t)a[i]),
                                                __builtin_bit_cast(bf16x2, (uint32_t)b[i]), s, false);
    } else {
#pragma unroll
        for (int i = 0; i < kVec<T>; ++i) s = fmaf(channel<T>(a, i), channel<T>(b, i), s);
    }
    return s;
}

// acc += w * channels
template <typename T>
__device__ __forceinline__ void add_channels(float (&acc)[kVec<T>], float w, const Raw& r) {
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) acc[i] = fmaf(w, channel<T>(r, i), acc[i]);
}

// The one rounding to the features' type, to nearest even.
// ONCE: larger than the caches and not read again here.
template <typename T, bool VEC, bool ONCE = false>
__device__ __forceinline__ void store_channels(T* p, int n, const float (&x)[kVec<T>]) {
    constexpr int W = kVec<T>;
    if constexpr (VEC) {
        if (n <= 0) return;
        u32x4 r;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = __float_as_uint(x[i]);
        } else {
            typedef float f32x2 __attribute__((ext_vector_type(2)));
            typedef T t2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int i = 0; i < 4; ++i)
                r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2 * i], x[2 * i + 1]}), t2));
        }
        if constexpr (ONCE) __builtin_nontemporal_store(r, reinterpret_cast<u32x4*>(p));
        else *reinterpret_cast<u32x4*>(p) = r;
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < n) p[i] = (T)x[i];
    }
}

// ------------------------------------------------------------------ lanes

// Sums over groups of G lanes (a power of two, the same for the launch), in
// every lane of the group; every lane of the wave must be active. After the
// first steps the lanes of a quad, then of eight, hold the same value, so that
// a mirrored row serves as the exchange at distance 4 and 8.
template <int C>
__device__ __forceinline__ float dpp_f(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), C, 0xF, 0xF, true));
}
template <int N>
__device__ __forceinline__ void group_sums(float (&v)[N], int G) {
    if (G > 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += dpp_f<0xB1>(v[i]);  // quad_perm 1,0,3,2
    }
    if (G > 2) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += dpp_f<0x4E>(v[i]);  // quad_perm 2,3,0,1
    }
    if (G > 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += dpp_f<0x141>(v[i]);  // row_half_mirror
    }
    if (G > 8) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += dpp_f<0x140>(v[i]);  // row_mirror
    }
    if (G > 16) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __uint_as_float(xlane(__float_as_uint(v[i]), 16));
    }
    if (G > 32) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __uint_as_float(xlane(__float_as_uint(v[i]), 32));
    }
}

// ------------------------------------------------------------------ the bias of a pair

// The edges in LDS, each axis's filled up to one less than a power of two by
// values no distance reaches (NaN), and the steps of a search among them.
struct Edges {
    const float* at;  // [3][size]
    int size;         // 2^k - 1 >= nb - 1
};

inline __host__ __device__ int edges_size(int nb) {
    int n = 1;
    while (n < nb) n <<= 1;
    return n - 1;
}

// Copies them (every thread of the block; the caller synchronises).
__device__ __forceinline__ Edges stage_edges(const Bias& b, float* lds) {
    const int size = edges_size(b.nb), n = b.nb - 1;
    for (int e = threadIdx.x; e < 3 * size; e += blockDim.x) {
        const int axis = e / size, k = e - axis * size;
        lds[e] = k < n ? b.edges[axis * n + k] : __builtin_nanf("");
    }
    return Edges{lds, size};
}

// Where a pair lies: the number of edges <= d on each axis, a byte each, and
// its distance. The three searches' steps are read together.
__device__ __forceinline__ void pair_place(const Edges& ed, bool want_dist, const float (&p)[3], const float (&c)[3],
                                           uint32_t& u, float& dist) {
    const float dx = p[0] - c[0], dy = p[1] - c[1], dz = p[2] - c[2];
    int x = 0, y = 0, z = 0;
    for (int s = (ed.size + 1) >> 1; s > 0; s >>= 1) {
        const float ex = ed.at[x + s - 1], ey = ed.at[ed.size + y + s - 1], ez = ed.at[2 * ed.size + z + s - 1];
        x += ex <= dx ? s : 0;
        y += ey <= dy ? s : 0;
        z += ez <= dz ? s : 0;
    }
    u = (uint32_t)x | (uint32_t)y << 8 | (uint32_t)z << 16;
    dist = want_dist ? sqrtf((dx * dx + dy * dy) + dz * dz) : 0.0f;
}

constexpr int kTableFloats = 8192;  // largest table that a workgroup copies to LDS

// The bias as a workgroup holds it: edges and slopes in LDS, the table as well
// where it takes at most kTableFloats, its rows rounded up to four heads, so
// that a lane reads four at once.
struct PlaceBias {
    Edges ed;
    const float* table;  // [3][nb][H], the caller's
    const float* lds;    // [3][nb][Hp] (lds_table)
    const float* slope;  // [Hp], zeros where there is none
    int nb, H, Hp;
    bool dist, lds_table;

    // Floats of LDS it takes (a multiple of 4). with_table false: places alone.
    static __host__ __device__ int floats(const Bias& b, bool with_table = true) {
        if (b.nb == 0 && !b.slope) return 0;
        const int hp = (b.H + 3) & ~3, t = with_table ? 3 * b.nb * hp : 0;
        return ((t <= kTableFloats ? t : 0) + hp + 3 * edges_size(b.nb) + 3) & ~3;
    }

    // Every thread of the block; ends with a barrier. `s`: 16-byte aligned.
    __device__ __forceinline__ PlaceBias(const Bias& b, float* s, bool with_table = true) {
        nb = b.nb;
        H = b.H;
        Hp = (H + 3) & ~3;
        dist = b.slope != nullptr;
        const int t = with_table ? 3 * nb * Hp : 0;
        lds_table = t <= kTableFloats;
        table = b.table;
        lds = s;
        if (!placed()) return;
        if (lds_table) {
            if (Hp == H) {
                for (int e = threadIdx.x; e < t; e += blockDim.x) s[e] = b.table[e];
            } else {
                for (int e = threadIdx.x; e < t; e += blockDim.x) {
                    const int r = e / Hp, h = e - r * Hp;
                    s[e] = h < H ? b.table[r * H + h] : 0.0f;
                }
            }
            s += t;
        }
        slope = s;
        for (int e = threadIdx.x; e < Hp; e += blockDim.x) s[e] = b.slope && e < H ? b.slope[e] : 0.0f;
        ed = stage_edges(b, s + Hp);
        __syncthreads();
    }
    __device__ __forceinline__ bool placed() const { return nb > 0 || dist; }

    __device__ __forceinline__ uint32_t x_row(uint32_t u) const { return u & 255u; }
    __device__ __forceinline__ uint32_t y_row(uint32_t u) const { return nb + (u >> 8 & 255u); }
    __device__ __forceinline__ uint32_t z_row(uint32_t u) const { return 2 * nb + (u >> 16); }

    // Bias of head h at a place.
    __device__ __forceinline__ float one(uint32_t u, float d, int h) const {
        float b = slope[h] * d;
        if (nb == 0) return b;
        if (lds_table)
            return b + ((lds[x_row(u) * Hp + h] + lds[y_row(u) * Hp + h]) + lds[z_row(u) * Hp + h]);
        return b + ((table[x_row(u) * H + h] + table[y_row(u) * H + h]) + table[z_row(u) * H + h]);
    }
    // Of heads h to h + 3 (h a multiple of 4).
    __device__ __forceinline__ f32x4 four(uint32_t u, float d, int h) const {
        f32x4 b = *(const f32x4*)(slope + h);
        b *= d;
        if (nb == 0) return b;
        if (lds_table) {
            const f32x4 x = *(const f32x4*)(lds + __umul24(x_row(u), (uint32_t)Hp) + h);
            const f32x4 y = *(const f32x4*)(lds + __umul24(y_row(u), (uint32_t)Hp) + h);
            const f32x4 z = *(const f32x4*)(lds + __umul24(z_row(u), (uint32_t)Hp) + h);
            return b + ((x + y) + z);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (h + i < H) b[i] = one(u, d, h + i);
        return b;
    }
};

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
hipError_t launch_group_attention(const Groups& g, int32_t B, const Attn& a, int32_t dtype, const Bias& b, void* out,
                                  float* lse, void* ws, hipStream_t s);
hipError_t launch_group_attention_backward(const Groups& g, int32_t B, const Attn& a, int32_t dtype, const Bias& b,
                                           const int64_t* pt_off, const int32_t* pt_center, int64_t capacity,
                                           const float* lse, const void* dout, void* dq, void* dk, void* dv,
                                           float* dtable, float* dslope, void* ws, hipStream_t s);

}  // namespace cagq
