// C ABI of the norm and rotation of heads (k_heads.hip): parameter checks and launches.
#include "api_util.hpp"
#include "sla_kernels.hpp"

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>

using sla::aligned;
using sla::align_up;
using sla::fail;

namespace {

constexpr double kQuarterTurn = 1.5707963267948966192313216916398;

sla_status_t make_args(const sla_heads_params_t *p, sla::HeadsArgs &a)
{
    if (!p) return fail(SLA_ERR_INVALID_ARG, "params is NULL");
    if (p->B < 0 || p->H < 0 || p->N < 0) return fail(SLA_ERR_INVALID_ARG, "B, H, N must be >= 0 (got %d, %d, %d)", p->B, p->H, p->N);
    if (p->D != 64) return fail(SLA_ERR_UNSUPPORTED, "head dim D = %d; only 64 is implemented", p->D);
    if ((long)p->B * p->N > 0x7FFFFF00L) return fail(SLA_ERR_UNSUPPORTED, "B*N = %ld is too large", (long)p->B * p->N);
    if (p->H > 65535) return fail(SLA_ERR_UNSUPPORTED, "H = %d; at most 65535 are implemented", p->H);
    if ((long)p->B * p->H > 65535) return fail(SLA_ERR_UNSUPPORTED, "B*H = %ld exceeds 65535", (long)p->B * p->H);
    if (p->norm < SLA_NORM_NONE || p->norm > SLA_NORM_LAYER) return fail(SLA_ERR_INVALID_ARG, "unknown norm %d", p->norm);
    if (p->norm_per_head != 0 && p->norm_per_head != 1) return fail(SLA_ERR_INVALID_ARG, "norm_per_head must be 0 or 1");
    if (p->axes < 0 || p->axes > 2) return fail(SLA_ERR_INVALID_ARG, "axes = %d; must be 0, 1 or 2", p->axes);
    if (p->pairing != SLA_PAIR_HALVES && p->pairing != SLA_PAIR_ADJACENT) return fail(SLA_ERR_INVALID_ARG, "unknown pairing %d", p->pairing);
    if (p->pos_per_item != 0 && p->pos_per_item != 1) return fail(SLA_ERR_INVALID_ARG, "pos_per_item must be 0 or 1");
    if (p->layout != SLA_LAYOUT_BHND && p->layout != SLA_LAYOUT_BNHD) return fail(SLA_ERR_INVALID_ARG, "unknown layout %d", p->layout);
    if (p->norm != SLA_NORM_NONE && !(p->eps >= FLT_MIN && std::isfinite(p->eps))) return fail(SLA_ERR_INVALID_ARG, "eps must be a finite normal number > 0");
    if (p->axes && !(p->base >= 1.0 && std::isfinite(p->base))) return fail(SLA_ERR_INVALID_ARG, "base must be finite and >= 1");
    memset(&a, 0, sizeof a);
    a.B = p->B; a.H = p->H; a.N = p->N;
    a.norm = p->norm; a.per_head = p->norm_per_head; a.eps = p->eps;
    a.axes = p->axes; a.adjacent = p->pairing == SLA_PAIR_ADJACENT; a.pos_per_item = p->pos_per_item;
    a.bs = p->batch_stride; a.ts = p->token_stride; a.hs = p->head_stride;
    if (a.B && a.H && a.N) {
        // strides of dimensions of one element do not matter; from the smallest stride on, each of the others has to span all rows
        // that the smaller ones reach
        const long lim = 1L << 48;
        struct Dim { const char *name; long n; long *s; } dims[3] = {{"head_stride", a.H, &a.hs}, {"token_stride", a.N, &a.ts}, {"batch_stride", a.B, &a.bs}};
        for (Dim &d : dims) {
            if (d.n == 1) *d.s = 0;
            else if (*d.s < 64 || *d.s % 8 != 0 || *d.s > lim / d.n)
                return fail(SLA_ERR_INVALID_ARG, "%s = %ld; must be a multiple of 8 and at least 64", d.name, *d.s);
        }
        std::sort(dims, dims + 3, [](const Dim &x, const Dim &y) { return *x.s < *y.s; });
        long span = 64;
        for (const Dim &d : dims) {
            if (d.n == 1) continue;
            if (*d.s < span) return fail(SLA_ERR_INVALID_ARG, "%s = %ld; the rows of smaller strides reach over %ld elements: rows overlap or interleave", d.name, *d.s, span);
            span += (d.n - 1) * *d.s;
        }
    }
    const sla::RowMap out = sla::make_rowmap(p->layout == SLA_LAYOUT_BNHD, p->H, p->N);
    a.obs = out.bs; a.ots = out.ts; a.ohs = out.hs;
    if (p->axes)
        for (int j = 0, per = 32 / p->axes; j < 32; ++j) a.turn[j] = std::pow(p->base, -(double)(j % per) / per) / kQuarterTurn;
    return SLA_OK;
}

bool empty(const sla::HeadsArgs &a) { return a.B == 0 || a.H == 0 || a.N == 0; }

sla_status_t set_inputs(sla::HeadsArgs &a, const void *q, const void *k, const void *v, const float *q_weight, const float *q_bias,
                        const float *k_weight, const float *k_bias, const int32_t *pos)
{
    SLA_REQ_PTR(q); SLA_REQ_PTR(k);
    SLA_OPT_PTR(v); SLA_OPT_PTR(q_weight); SLA_OPT_PTR(q_bias); SLA_OPT_PTR(k_weight); SLA_OPT_PTR(k_bias);
    if (a.norm == 0 && (q_weight || q_bias || k_weight || k_bias)) return fail(SLA_ERR_INVALID_ARG, "weights and biases belong to a norm; SLA_NORM_NONE takes none");
    if (a.axes && !pos) return fail(SLA_ERR_INVALID_ARG, "pos is NULL");
    if (a.axes && !aligned(pos, 4)) return fail(SLA_ERR_INVALID_ARG, "pos must be 4-byte aligned");
    a.x[0] = (const uint16_t *)q; a.x[1] = (const uint16_t *)k; a.x[2] = (const uint16_t *)v;
    a.w[0] = q_weight; a.w[1] = k_weight; a.b[0] = q_bias; a.b[1] = k_bias;
    a.pos = pos;
    a.tensors = v ? 3 : 2;
    return SLA_OK;
}

}  // namespace

extern "C" {

sla_status_t sla_qk_norm_rope(const sla_heads_params_t *p, const void *q, const void *k, const void *v, const float *q_weight,
                              const float *q_bias, const float *k_weight, const float *k_bias, const int32_t *pos, void *Q, void *K,
                              void *V, void *stream)
{
    sla::HeadsArgs a;
    sla_status_t s = make_args(p, a);
    if (s != SLA_OK || empty(a)) return s;
    if ((s = set_inputs(a, q, k, v, q_weight, q_bias, k_weight, k_bias, pos)) != SLA_OK) return s;
    SLA_REQ_PTR(Q); SLA_REQ_PTR(K); SLA_OPT_PTR(V);
    if (!v != !V) return fail(SLA_ERR_INVALID_ARG, "v and V must both be given or both be NULL");
    a.y[0] = Q; a.y[1] = K; a.y[2] = V;
    SLA_HIP(sla::launch_heads(a, 0, (hipStream_t)stream));
    return SLA_OK;
}

sla_status_t sla_qk_norm_rope_e4m3(const sla_heads_params_t *p, const void *q, const void *k, const void *v, const float *q_weight,
                                   const float *q_bias, const float *k_weight, const float *k_bias, const int32_t *pos, int32_t bq,
                                   void *Q8, void *K8, void *V8, float *sQ, float *sK, float *sV, void *stream)
{
    sla::HeadsArgs a;
    sla_status_t s = make_args(p, a);
    if (s != SLA_OK) return s;
    if (bq != 64 && bq != 128) return fail(SLA_ERR_UNSUPPORTED, "query block bq = %d; only 64 and 128 are implemented", bq);
    if (empty(a)) return SLA_OK;
    if ((s = set_inputs(a, q, k, v, q_weight, q_bias, k_weight, k_bias, pos)) != SLA_OK) return s;
    SLA_REQ_PTR(Q8); SLA_REQ_PTR(K8); SLA_OPT_PTR(V8);
    if (!v != !V8 || !v != !sV) return fail(SLA_ERR_INVALID_ARG, "v, V8 and sV must all be given or all be NULL");
    if (!sQ || !sK) return fail(SLA_ERR_INVALID_ARG, "a scale output is NULL");
    a.y[0] = Q8; a.y[1] = K8; a.y[2] = V8;
    a.scales[0] = sQ; a.scales[1] = sK; a.scales[2] = sV;
    SLA_HIP(sla::launch_heads(a, bq, (hipStream_t)stream));
    return SLA_OK;
}

sla_status_t sla_qk_norm_rope_grad_workspace_bytes(const sla_heads_params_t *p, size_t *bytes)
{
    sla::HeadsArgs a;
    sla_status_t s = make_args(p, a);
    if (s != SLA_OK) return s;
    if (!bytes) return fail(SLA_ERR_INVALID_ARG, "bytes is NULL");
    // with and without v the heads are split over another number of workgroups
    size_t two = 0, three = 0;
    if (a.norm != 0 && !empty(a)) {
        two = sla::heads_grad_part_bytes(a.B, a.H, a.N, 2, a.per_head);
        three = sla::heads_grad_part_bytes(a.B, a.H, a.N, 3, a.per_head);
    }
    *bytes = align_up(two > three ? two : three, 256);
    return SLA_OK;
}

sla_status_t sla_qk_norm_rope_grad(const sla_heads_params_t *p, const void *q, const void *k, const float *q_weight, const float *k_weight,
                                   const int32_t *pos, const void *dQ, const void *dK, const void *dV, void *dq, void *dk, void *dv,
                                   float *dq_weight, float *dq_bias, float *dk_weight, float *dk_bias, void *workspace,
                                   size_t workspace_bytes, void *stream)
{
    sla::HeadsArgs a;
    size_t need = 0;
    sla_status_t s = make_args(p, a);
    if (s != SLA_OK) return s;
    SLA_OPT_PTR(dq_weight); SLA_OPT_PTR(dq_bias); SLA_OPT_PTR(dk_weight); SLA_OPT_PTR(dk_bias);
    const bool wanted = dq_weight || dq_bias || dk_weight || dk_bias;
    if (a.norm == 0 && wanted) return fail(SLA_ERR_INVALID_ARG, "weights and biases belong to a norm; SLA_NORM_NONE has none");
    sla::HeadsGrads d = {};
    d.dw[0] = dq_weight; d.dw[1] = dk_weight; d.db[0] = dq_bias; d.db[1] = dk_bias;
    if (empty(a)) {                      // no rows: the gradients of the weights are zero
        a.N = 0;
        if (wanted && (a.H > 0 || !a.per_head)) SLA_HIP(sla::launch_heads_grad(a, d, (hipStream_t)stream));
        return SLA_OK;
    }
    if ((s = set_inputs(a, q, k, nullptr, q_weight, nullptr, k_weight, nullptr, pos)) != SLA_OK) return s;
    SLA_REQ_PTR(dQ); SLA_REQ_PTR(dK); SLA_OPT_PTR(dV); SLA_REQ_PTR(dq); SLA_REQ_PTR(dk); SLA_OPT_PTR(dv);
    if (!dV != !dv) return fail(SLA_ERR_INVALID_ARG, "dV and dv must both be given or both be NULL");
    if (wanted) {
        if ((s = sla_qk_norm_rope_grad_workspace_bytes(p, &need)) != SLA_OK) return s;
        if (!workspace) return fail(SLA_ERR_WORKSPACE, "workspace is NULL (%zu bytes needed)", need);
        if (!aligned(workspace, 256)) return fail(SLA_ERR_WORKSPACE, "workspace must be 256-byte aligned");
        if (workspace_bytes < need) return fail(SLA_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
        d.part = (float *)workspace;
    }
    a.tensors = dV ? 3 : 2;
    d.g[0] = (const uint16_t *)dQ; d.g[1] = (const uint16_t *)dK; d.g[2] = (const uint16_t *)dV;
    d.dx[0] = (uint16_t *)dq; d.dx[1] = (uint16_t *)dk; d.dx[2] = (uint16_t *)dv;
    SLA_HIP(sla::launch_heads_grad(a, d, (hipStream_t)stream));
    return SLA_OK;
}

}  // extern "C"
