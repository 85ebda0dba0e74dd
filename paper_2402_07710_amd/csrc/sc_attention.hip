// Attention over packed scenes: checks of the calls and the choice of kernels (sc_attention.h).
#include <initializer_list>

#include "sc_heads.h"
#include "sc_attention.h"

namespace sc {
int launch_attention_f16(const Attention& p, AttentionShape shape, hipStream_t s);
int launch_attention_bf16(const Attention& p, AttentionShape shape, hipStream_t s);
int launch_attention_f32(const Attention& p, AttentionShape shape, hipStream_t s);
int launch_attention_grad_f16(const Attention& p, bool alone, hipStream_t s);
int launch_attention_grad_bf16(const Attention& p, bool alone, hipStream_t s);
int launch_attention_grad_f32(const Attention& p, bool alone, hipStream_t s);

namespace {

bool sizes_ok(int64_t q_rows, int64_t k_rows, int scenes, int q_heads, int k_heads, int D, int dtype) {
    if (dtype != SC_F32 && dtype != SC_F16 && dtype != SC_BF16) return false;
    if (q_rows < 0 || q_rows > SC_N_MAX || k_rows < 0 || k_rows > SC_N_MAX || scenes < 1 || scenes > SC_SCENES_MAX || D < 1 || D > SC_ATTENTION_HEAD_MAX) return false;
    if (q_heads < 1 || q_heads > SC_GROUPS_MAX || k_heads < 1 || q_heads % k_heads != 0) return false;
    return q_rows * (q_heads / k_heads) <= INT32_MAX - 4096;
}
struct Plan {
    AttentionShape shape;
    int parts;
};
// bytes of a row in LDS
int row_bytes(int D, int dtype) { return (D <= 32 ? 32 : D <= 64 ? 64 : D <= 128 ? 128 : 256) * (dtype == SC_F32 ? 4 : 2); }
Plan plan_of(int64_t q_rows, int64_t k_rows, int scenes, int q_heads, int k_heads, int D, int dtype) {
    const int64_t columns = q_rows * (q_heads / k_heads);
    Plan plan{attention_shape(columns, scenes, k_heads, k_rows, row_bytes(D, dtype)), 1};
    plan.parts = q_rows == 0 ? 1 : attention_parts(plan.shape, columns, scenes, k_heads, k_rows, dtype == SC_F32);
    return plan;
}
struct GradPlan {
    bool alone;
    int parts, k_parts;
    size_t sums, part, k_part;         // bytes in the workspace: exponents or deltas, partial gradients of queries, of keys (and as much of values)
};
size_t up16(size_t n) { return (n + 15) / 16 * 16; }
GradPlan grad_plan_of(int64_t q_rows, int64_t k_rows, int scenes, int q_heads, int k_heads, int D, int dtype) {
    const int64_t per = q_heads / k_heads, columns = q_rows * per;
    GradPlan plan{attention_grad_alone(columns, scenes, k_heads, k_rows, row_bytes(D, dtype), dtype == SC_F32), 1, 1, 0, 0, 0};
    if (q_rows > 0 && k_rows > 0) {
        plan.parts = attention_grad_parts(plan.alone, columns, scenes, k_heads, k_rows, dtype == SC_F32);
        plan.k_parts = attention_grad_parts(plan.alone, k_rows, scenes, k_heads, columns, dtype == SC_F32);
    }
    plan.sums = up16((size_t)q_rows * q_heads * sizeof(float));
    plan.part = plan.parts > 1 ? up16((size_t)plan.parts * q_rows * q_heads * D * sizeof(float)) : 0;
    plan.k_part = plan.k_parts > 1 ? up16((size_t)plan.k_parts * k_rows * k_heads * D * sizeof(float)) : 0;
    return plan;
}
// A tile's rows are 63 strides apart at most, in an offset of 32 bits.
bool strides_ok(std::initializer_list<const sc_heads*> all) {
    for (const sc_heads* h : all)
        if (h->row > SC_ATTENTION_LD_MAX) return false;
    return true;
}
HeadRows rows_of(const sc_heads* h, int dtype) {
    const int size = dtype == SC_F32 ? 4 : 2;
    return HeadRows{(char*)h->data, h->row * size, h->head * size};
}
int check_attention(const sc_heads* q, const sc_heads* k, const sc_heads* v, int64_t q_rows, int64_t k_rows, int D, const int32_t* q_starts, const int32_t* k_starts,
                    const int32_t* k_lens, int scenes, int causal, float scale, const sc_heads* out, const float* lse, int dtype) {
    if (dtype != SC_F32 && dtype != SC_F16 && dtype != SC_BF16) return SC_EINVAL;
    if (!heads_ok(q, dtype) || !heads_ok(k, dtype) || !heads_ok(v, dtype) || !heads_ok(out, dtype)) return SC_EINVAL;
    if (!sizes_ok(q_rows, k_rows, scenes, q->heads, k->heads, D, dtype) || v->heads != k->heads || out->heads != q->heads) return SC_EINVAL;
    if (!strides_ok({q, k, v, out})) return SC_EINVAL;
    if (((uintptr_t)q_starts & 3) != 0 || ((uintptr_t)k_starts & 3) != 0 || ((uintptr_t)k_lens & 3) != 0 || ((uintptr_t)lse & 3) != 0) return SC_EINVAL;
    if (q_starts == nullptr && (k_starts != nullptr || scenes != 1)) return SC_EINVAL;
    if (q_starts != nullptr && k_starts == nullptr && q_rows != k_rows) return SC_EINVAL;
    if (causal != 0 && causal != 1) return SC_EINVAL;
    return scale > 0.f && scale <= SC_ATTENTION_SCALE_MAX ? SC_OK : SC_EINVAL;
}
// An output that shares elements with what other workgroups still read, or with another output, is refused; one in the very place of an operand that only its own
// columns are read from is not.
bool output_apart(const sc_heads* out, const sc_heads* q, const sc_heads* k, const sc_heads* v, int64_t q_rows, int64_t k_rows, int D, int dtype) {
    return !heads_meet(out, q_rows, k, k_rows, D, dtype) && !heads_meet(out, q_rows, v, k_rows, D, dtype) &&
           (heads_same(out, q, q_rows) || !heads_meet(out, q_rows, q, q_rows, D, dtype));
}
bool gradients_apart(const sc_heads* dout, const sc_heads* q, const sc_heads* k, const sc_heads* v, const sc_heads* out, const sc_heads* dq, const sc_heads* dk,
                     const sc_heads* dv, int64_t q_rows, int64_t k_rows, int D, int dtype) {
    if (heads_meet(dk, k_rows, dv, k_rows, D, dtype) || heads_meet(dq, q_rows, q, q_rows, D, dtype) || heads_meet(dq, q_rows, dout, q_rows, D, dtype)) return false;
    if (!heads_same(dq, out, q_rows) && heads_meet(dq, q_rows, out, q_rows, D, dtype)) return false;
    for (const sc_heads* of_keys : {k, v, dk, dv})
        if (heads_meet(dq, q_rows, of_keys, k_rows, D, dtype)) return false;
    for (const sc_heads* grad : {dk, dv}) {
        if (heads_meet(grad, k_rows, q, q_rows, D, dtype) || heads_meet(grad, k_rows, dout, q_rows, D, dtype)) return false;
        for (const sc_heads* own : {k, v})
            if (!heads_same(grad, own, k_rows) && heads_meet(grad, k_rows, own, k_rows, D, dtype)) return false;
    }
    return true;
}
Attention attention_of(const sc_heads* q, const sc_heads* k, const sc_heads* v, int64_t q_rows, int64_t k_rows, int D, const int32_t* q_starts, const int32_t* k_starts,
                       const int32_t* k_lens, int scenes, int causal, float scale, const sc_heads* out, float* lse, int dtype) {
    Attention p{};
    p.q = rows_of(q, dtype);
    p.k = rows_of(k, dtype);
    p.v = rows_of(v, dtype);
    p.out = rows_of(out, dtype);
    p.lse = lse;
    p.q_starts = q_starts;
    p.k_starts = k_starts != nullptr ? k_starts : q_starts;
    p.k_lens = k_lens;
    p.scenes = scenes;
    p.q_rows = q_rows;
    p.k_rows = k_rows;
    p.D = D;
    p.per = q->heads / k->heads;
    int log2 = 1;
    while (1 << log2 < p.per) ++log2;
    p.per_magic = (uint32_t)((((uint64_t)1 << (31 + log2)) + p.per - 1) / p.per);
    p.per_shift = log2 - 1;
    p.k_heads = k->heads;
    p.causal = causal;
    p.scale = scale;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.parts = 1;
    return p;
}
}  // namespace
}  // namespace sc

using namespace sc;

extern "C" size_t sc_attention_workspace_bytes(int64_t q_rows, int64_t k_rows, int scenes, int q_heads, int k_heads, int D, int dtype) {
    if (!sizes_ok(q_rows, k_rows, scenes, q_heads, k_heads, D, dtype)) return 0;
    const Plan plan = plan_of(q_rows, k_rows, scenes, q_heads, k_heads, D, dtype);
    if (plan.parts == 1) return 0;
    const size_t entries = (size_t)plan.parts * q_rows * q_heads;
    return up16(entries * sizeof(float2)) + entries * D * sizeof(float);
}

extern "C" int sc_attention_fwd(const sc_heads* q, const sc_heads* k, const sc_heads* v, int64_t q_rows, int64_t k_rows, int D, const int32_t* d_q_starts,
                                const int32_t* d_k_starts, const int32_t* d_k_lens, int scenes, int causal, float scale, const sc_heads* out, float* d_lse, int dtype,
                                void* d_workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_attention(q, k, v, q_rows, k_rows, D, d_q_starts, d_k_starts, d_k_lens, scenes, causal, scale, out, d_lse, dtype);
    if (rc != SC_OK) return rc;
    if (!heads_apart(out, q_rows, D)) return SC_EINVAL;
    const size_t need = sc_attention_workspace_bytes(q_rows, k_rows, scenes, q->heads, k->heads, D, dtype);
    if (need > 0 && (d_workspace == nullptr || !aligned16(d_workspace))) return SC_EINVAL;
    if (workspace_bytes < need) return SC_ECAP;
    if (!output_apart(out, q, k, v, q_rows, k_rows, D, dtype)) return SC_EINVAL;
    if (q_rows == 0) return SC_OK;
    const Plan plan = plan_of(q_rows, k_rows, scenes, q->heads, k->heads, D, dtype);
    Attention p = attention_of(q, k, v, q_rows, k_rows, D, d_q_starts, d_k_starts, d_k_lens, scenes, causal, scale, out, d_lse, dtype);
    p.parts = plan.parts;
    p.part_keys = attention_part_keys(dtype == SC_F32);
    if (plan.parts > 1) {
        p.part_sums = (float2*)d_workspace;
        p.part_out = (float*)((char*)d_workspace + up16((size_t)plan.parts * q_rows * q->heads * sizeof(float2)));
    }
    hipStream_t s = (hipStream_t)stream;
    return dtype == SC_F32 ? launch_attention_f32(p, plan.shape, s) : dtype == SC_F16 ? launch_attention_f16(p, plan.shape, s) : launch_attention_bf16(p, plan.shape, s);
}

extern "C" size_t sc_attention_bwd_workspace_bytes(int64_t q_rows, int64_t k_rows, int scenes, int q_heads, int k_heads, int D, int dtype) {
    if (!sizes_ok(q_rows, k_rows, scenes, q_heads, k_heads, D, dtype)) return 0;
    const GradPlan plan = grad_plan_of(q_rows, k_rows, scenes, q_heads, k_heads, D, dtype);
    return 2 * plan.sums + plan.part + 2 * plan.k_part;
}

extern "C" int sc_attention_bwd(const sc_heads* dout, const sc_heads* q, const sc_heads* k, const sc_heads* v, const sc_heads* out, const float* d_lse, int64_t q_rows,
                                int64_t k_rows, int D, const int32_t* d_q_starts, const int32_t* d_k_starts, const int32_t* d_k_lens, int scenes, int causal, float scale,
                                const sc_heads* dq, const sc_heads* dk, const sc_heads* dv, int dtype, void* d_workspace, size_t workspace_bytes, void* stream) {
    const int rc = check_attention(q, k, v, q_rows, k_rows, D, d_q_starts, d_k_starts, d_k_lens, scenes, causal, scale, out, d_lse, dtype);
    if (rc != SC_OK) return rc;
    if (d_lse == nullptr || !heads_ok(dout, dtype) || !heads_ok(dq, dtype) || !heads_ok(dk, dtype) || !heads_ok(dv, dtype)) return SC_EINVAL;
    if (dout->heads != q->heads || dq->heads != q->heads || dk->heads != k->heads || dv->heads != k->heads) return SC_EINVAL;
    if (!strides_ok({dout, dq, dk, dv})) return SC_EINVAL;
    if (!heads_apart(dq, q_rows, D) || !heads_apart(dk, k_rows, D) || !heads_apart(dv, k_rows, D)) return SC_EINVAL;
    const size_t need = sc_attention_bwd_workspace_bytes(q_rows, k_rows, scenes, q->heads, k->heads, D, dtype);
    if (need > 0 && (d_workspace == nullptr || !aligned16(d_workspace))) return SC_EINVAL;
    if (workspace_bytes < need) return SC_ECAP;
    if (!gradients_apart(dout, q, k, v, out, dq, dk, dv, q_rows, k_rows, D, dtype)) return SC_EINVAL;
    Attention p = attention_of(q, k, v, q_rows, k_rows, D, d_q_starts, d_k_starts, d_k_lens, scenes, causal, scale, out, const_cast<float*>(d_lse), dtype);
    p.dout = rows_of(dout, dtype);
    p.dq = rows_of(dq, dtype);
    p.dk = rows_of(dk, dtype);
    p.dv = rows_of(dv, dtype);
    const GradPlan plan = grad_plan_of(q_rows, k_rows, scenes, q->heads, k->heads, D, dtype);
    char* const space = (char*)d_workspace;
    p.against = (float*)space;
    p.delta = (float*)(space + plan.sums);
    p.part_out = (float*)(space + 2 * plan.sums);
    p.part_dk = (float*)(space + 2 * plan.sums + plan.part);
    p.part_dv = (float*)(space + 2 * plan.sums + plan.part + plan.k_part);
    p.parts = plan.parts;
    p.k_parts = plan.k_parts;
    p.part_keys = p.part_rows = attention_part_rows(plan.alone, dtype == SC_F32);
    hipStream_t s = (hipStream_t)stream;
    return dtype == SC_F32 ? launch_attention_grad_f32(p, plan.alone, s) : dtype == SC_F16 ? launch_attention_grad_f16(p, plan.alone, s) : launch_attention_grad_bf16(p, plan.alone, s);
}
