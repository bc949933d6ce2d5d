// C ABI of the operators on point features (declared in include/cagq.h):
// argument validation on the host, before anything is enqueued.
#include <math.h>

#include "cagq_features.h"

namespace cagq {

namespace {

constexpr int64_t kMaxSlots = 2147483647;

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// The groups' sizes and what `need_places` asks for; sizes only when `sizes`.
bool make_groups(const cagq_groups* c, bool need_places, bool sizes, Groups* g) {
    if (!c || c->B < 1 || c->N < 1 || c->M < 1 || c->K < 0) return false;
    if ((int64_t)c->B * c->N > 2147483647LL || (int64_t)c->B * c->M > 2147483647LL) return false;
    g->rows = c->B * c->M;
    if (c->K > 0) {
        if (c->off || c->idx_len != 0) return false;
        if ((int64_t)g->rows > kMaxSlots / c->K) return false;
        g->idx_len = (int64_t)g->rows * c->K;
    } else {
        if (c->n_valid || c->idx_len < 0 || c->idx_len > kMaxSlots) return false;
        if (!sizes && (!c->off || !aligned(c->off, 8))) return false;
        g->idx_len = c->idx_len;
    }
    g->idx = c->idx;
    g->n_valid = c->n_valid;
    g->off = c->off;
    g->points = c->points;
    g->centers = c->centers;
    g->N = c->N;
    g->M = c->M;
    g->K = c->K;
    g->mm = make_magic((uint32_t)c->M);
    if (sizes) return true;
    if ((!c->idx && g->idx_len > 0) || !aligned(c->idx, 4) || !aligned(c->n_valid, 4)) return false;
    if (need_places && (!c->points || !c->centers || !aligned(c->points, 4) || !aligned(c->centers, 4))) return false;
    return true;
}

// `b` may be null: no bias.
bool make_bias(const cagq_bias* b, int32_t H, bool sizes, Bias* out) {
    *out = Bias{nullptr, nullptr, nullptr, 0, H};
    if (!b) return true;
    if (b->buckets < 0 || b->buckets > CAGQ_MAX_BUCKETS) return false;
    if (!sizes) {
        if ((b->buckets > 0) != (b->table != nullptr)) return false;
        if (b->buckets > 1 && !b->edges) return false;
        if (!aligned(b->table, 4) || !aligned(b->edges, 4) || !aligned(b->slope, 4)) return false;
    }
    out->table = b->table;
    out->edges = b->edges;
    out->slope = b->slope;
    out->nb = b->buckets;
    return true;
}

bool make_attn(const cagq_attn* a, Attn* out) {
    if (!a || a->dtype < CAGQ_F32 || a->dtype > CAGQ_F16) return false;
    if (a->H < 1 || a->H > CAGQ_MAX_HEADS || a->Hkv < 1 || a->H % a->Hkv) return false;
    if (a->D < 1 || a->D > CAGQ_MAX_HEAD_DIM) return false;
    if (!isfinite(a->scale) || !isfinite(a->cap) || a->cap < 0.0f) return false;
    // what the kernels make of them: twice the cap, and scale / cap to base 2
    if (a->cap > 0.0f && (!isfinite(2.0f * a->cap) || !isfinite(3.0f * a->scale / a->cap))) return false;
    const int64_t qd = (int64_t)a->H * a->D, kd = (int64_t)a->Hkv * a->D;
    out->q_row = a->q_row ? a->q_row : qd;
    out->k_row = a->k_row ? a->k_row : kd;
    out->v_row = a->v_row ? a->v_row : kd;
    constexpr int64_t kMaxRow = 1ll << 31;  // times 2^31 rows and 4 bytes stays below 2^63
    if (out->q_row < qd || out->k_row < kd || out->v_row < kd) return false;
    if (out->q_row > kMaxRow || out->k_row > kMaxRow || out->v_row > kMaxRow) return false;
    out->q = out->k = out->v = nullptr;
    out->H = a->H;
    out->Hkv = a->Hkv;
    out->D = a->D;
    out->scale = a->scale;
    out->cap = a->cap;
    return true;
}

size_t type_bytes(int32_t dtype) { return dtype == CAGQ_F32 ? 4 : 2; }

int check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return CAGQ_OK;
    if (!ws || !aligned(ws, 256)) return CAGQ_ERR_INVALID_ARG;
    return have < need ? CAGQ_ERR_WORKSPACE_TOO_SMALL : CAGQ_OK;
}

int hip_status(hipError_t e) { return e == hipSuccess ? CAGQ_OK : CAGQ_ERR_HIP; }

}  // namespace

}  // namespace cagq

using namespace cagq;

extern "C" {

int cagq_group_attention_workspace(const cagq_groups* g, const cagq_attn* a, const cagq_bias* bias, int32_t backward,
                                   size_t* bytes) {
    Groups gr;
    Bias b;
    Attn at;
    if (!bytes || (backward != 0 && backward != 1) || !make_groups(g, false, true, &gr) || !make_attn(a, &at) ||
        !make_bias(bias, at.H, true, &b))
        return CAGQ_ERR_INVALID_ARG;
    *bytes = group_attention_bytes(gr, g->B, at, a->dtype, b, backward != 0);
    return CAGQ_OK;
}

int cagq_group_attention(const cagq_groups* g, const cagq_attn* a, const cagq_bias* bias, const void* q, const void* k,
                         const void* v, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    Groups gr;
    Bias b;
    Attn at;
    if (!make_attn(a, &at) || !make_bias(bias, at.H, false, &b) ||
        !make_groups(g, b.nb > 0 || b.slope, false, &gr))
        return CAGQ_ERR_INVALID_ARG;
    const size_t e = type_bytes(a->dtype);
    if (!q || !k || !v || !out || !aligned(q, e) || !aligned(k, e) || !aligned(v, e) || !aligned(out, e) ||
        !aligned(lse, 4))
        return CAGQ_ERR_INVALID_ARG;
    at.q = q;
    at.k = k;
    at.v = v;
    const int rc = check_workspace(workspace, workspace_bytes, group_attention_bytes(gr, g->B, at, a->dtype, b, false));
    if (rc != CAGQ_OK) return rc;
    return hip_status(launch_group_attention(gr, g->B, at, a->dtype, b, out, lse, workspace, (hipStream_t)stream));
}

int cagq_point_lists_workspace(const cagq_groups* g, size_t* bytes) {
    Groups gr;
    if (!bytes || !make_groups(g, false, true, &gr)) return CAGQ_ERR_INVALID_ARG;
    *bytes = point_lists_bytes(gr, g->B);
    return CAGQ_OK;
}

int cagq_point_lists(const cagq_groups* g, int64_t* pt_off, int32_t* pt_center, int64_t capacity, void* workspace,
                     size_t workspace_bytes, void* stream) {
    Groups gr;
    if (!make_groups(g, false, false, &gr) || !pt_off || !aligned(pt_off, 8) || !aligned(pt_center, 4) ||
        capacity < 0 || (!pt_center && capacity > 0))
        return CAGQ_ERR_INVALID_ARG;
    if (capacity < gr.idx_len) return CAGQ_ERR_CAPACITY;
    const int rc = check_workspace(workspace, workspace_bytes, point_lists_bytes(gr, g->B));
    if (rc != CAGQ_OK) return rc;
    return hip_status(launch_point_lists(gr, g->B, pt_off, pt_center, capacity, workspace, (hipStream_t)stream));
}

int cagq_group_attention_backward(const cagq_groups* g, const cagq_attn* a, const cagq_bias* bias,
                                  const int64_t* pt_off, const int32_t* pt_center, int64_t capacity, const void* q,
                                  const void* k, const void* v, const float* lse, const void* dout, void* dq, void* dk,
                                  void* dv, float* dtable, float* dslope, void* workspace, size_t workspace_bytes,
                                  void* stream) {
    Groups gr;
    Bias b;
    Attn at;
    if (!make_attn(a, &at) || !make_bias(bias, at.H, false, &b) ||
        !make_groups(g, b.nb > 0 || b.slope, false, &gr))
        return CAGQ_ERR_INVALID_ARG;
    const size_t e = type_bytes(a->dtype);
    for (const void* p : {q, k, v, dout, (const void*)dq, (const void*)dk, (const void*)dv})
        if (!p || !aligned(p, e)) return CAGQ_ERR_INVALID_ARG;
    if (!lse || !aligned(lse, 4) || !pt_off || !aligned(pt_off, 8) || !aligned(pt_center, 4) || capacity < 0 ||
        (!pt_center && capacity > 0) || !aligned(dtable, 4) || !aligned(dslope, 4))
        return CAGQ_ERR_INVALID_ARG;
    if ((dtable && b.nb == 0) || (dslope && !b.slope)) return CAGQ_ERR_INVALID_ARG;
    at.q = q;
    at.k = k;
    at.v = v;
    const int rc = check_workspace(workspace, workspace_bytes, group_attention_bytes(gr, g->B, at, a->dtype, b, true));
    if (rc != CAGQ_OK) return rc;
    return hip_status(launch_group_attention_backward(gr, g->B, at, a->dtype, b, pt_off, pt_center, capacity, lse,
                                                      dout, dq, dk, dv, dtable, dslope, workspace,
                                                      (hipStream_t)stream));
}

static bool bias_call(const cagq_groups* g, const cagq_bias* bias, int32_t H, int32_t dtype, bool sizes, Groups* gr,
                      Bias* b) {
    if (!bias || H < 1 || H > CAGQ_MAX_HEADS || dtype < CAGQ_F32 || dtype > CAGQ_F16) return false;
    if (!make_bias(bias, H, sizes, b) || !make_groups(g, true, sizes, gr)) return false;
    return sizes || b->nb > 0 || b->slope;
}

int cagq_relative_bias(const cagq_groups* g, const cagq_bias* bias, int32_t H, int32_t dtype, void* out,
                       void* stream) {
    Groups gr;
    Bias b;
    if (!bias_call(g, bias, H, dtype, false, &gr, &b) || !aligned(out, type_bytes(dtype)) ||
        (!out && gr.idx_len > 0))
        return CAGQ_ERR_INVALID_ARG;
    if (gr.idx_len == 0) return CAGQ_OK;
    return hip_status(launch_relative_bias(gr, b, dtype, out, (hipStream_t)stream));
}

int cagq_relative_bias_workspace(const cagq_groups* g, const cagq_bias* bias, int32_t H, size_t* bytes) {
    Groups gr;
    Bias b;
    if (!bytes || !bias_call(g, bias, H, CAGQ_F32, true, &gr, &b)) return CAGQ_ERR_INVALID_ARG;
    *bytes = relative_bias_bytes(gr, b);
    return CAGQ_OK;
}

int cagq_relative_bias_backward(const cagq_groups* g, const cagq_bias* bias, int32_t H, int32_t dtype,
                                const void* dbias, float* dtable, float* dslope, void* workspace,
                                size_t workspace_bytes, void* stream) {
    Groups gr;
    Bias b;
    if (!bias_call(g, bias, H, dtype, false, &gr, &b) || !aligned(dbias, type_bytes(dtype)) ||
        (!dbias && gr.idx_len > 0) || !aligned(dtable, 4) || !aligned(dslope, 4) || (!dtable && !dslope))
        return CAGQ_ERR_INVALID_ARG;
    if ((dtable && b.nb == 0) || (dslope && !b.slope)) return CAGQ_ERR_INVALID_ARG;
    const int rc = check_workspace(workspace, workspace_bytes, relative_bias_bytes(gr, b));
    if (rc != CAGQ_OK) return rc;
    return hip_status(launch_relative_bias_backward(gr, b, dtype, dbias, dtable, dslope, workspace,
                                                    (hipStream_t)stream));
}

}  // extern "C"
