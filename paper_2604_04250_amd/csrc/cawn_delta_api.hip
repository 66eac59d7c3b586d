// Gated delta rule: argument checks, sizes and the choice of a form.
#include "cawn_delta.hpp"

using namespace cawn;
using namespace cawn::ops;
using cawn::delta::Args;

namespace {

int check(const cawn_delta_desc *d, Args *a)
{
    if (!d || d->B < 0 || d->L < 0 || d->H <= 0 || d->Hk < 0 || d->K <= 0 || d->V <= 0 || (d->bf16 & ~1) || (d->qk_norm & ~1)) return CAWN_EINVAL;
    const int Hk = d->Hk ? d->Hk : d->H;
    if (d->H % Hk) return CAWN_EINVAL;
    if (d->K > 128) return CAWN_EUNSUPPORTED;
    *a = Args{};
    a->B = d->B, a->L = d->L, a->H = d->H, a->Hk = Hk, a->K = d->K, a->V = d->V, a->norm = d->qk_norm;
    a->scale = d->scale, a->eps = d->norm_eps;
    const long long qrow = (long long)Hk * d->K, vrow = (long long)d->H * d->V;
    a->qst = d->qk_stride_t ? d->qk_stride_t : qrow, a->vst = d->v_stride_t ? d->v_stride_t : vrow, a->ost = d->o_stride_t ? d->o_stride_t : vrow;
    if (a->qst < qrow || a->vst < vrow || a->ost < vrow) return CAWN_EINVAL;
    a->qsb = d->qk_stride_b ? d->qk_stride_b : a->qst * d->L, a->vsb = d->v_stride_b ? d->v_stride_b : a->vst * d->L;
    a->osb = d->o_stride_b ? d->o_stride_b : a->ost * d->L;
    a->chunks = (int)ceil_div(d->L, delta::CHUNK);
    return CAWN_OK;
}

bool misaligned(const cawn_delta_desc *d, const void *p) { return !aligned_to(p, d->bf16 ? 2 : 4); }

} // namespace

extern "C" {

size_t cawn_delta_state_bytes(const cawn_delta_desc *d)
{
    Args a;
    return check(d, &a) != CAWN_OK ? 0 : (size_t)a.B * a.H * a.K * a.V * 4;
}

size_t cawn_delta_ckpt_bytes(const cawn_delta_desc *d)
{
    Args a;
    return check(d, &a) != CAWN_OK ? 0 : (size_t)a.B * a.H * a.chunks * (a.K + delta::CHUNK) * a.V * 4;
}

size_t cawn_delta_workspace_bytes(const cawn_delta_desc *d)
{
    Args a;
    return check(d, &a) != CAWN_OK ? 0 : 256;
}

int cawn_delta_rule_fwd(const cawn_delta_desc *d, const void *q, const void *k, const void *v, const float *decay, const float *beta, const int32_t *lengths,
                        const void *state_in, void *o, void *state_out, void *ckpt, void *workspace, size_t workspace_bytes, void *stream)
{
    Args a;
    if (int r = check(d, &a)) return r;
    if (a.B == 0) return CAWN_OK;
    if (a.L > 0 && (!q || !k || !v || !decay || !beta || !o)) return CAWN_EINVAL;
    if (misaligned(d, q) || misaligned(d, k) || misaligned(d, v) || misaligned(d, o) || !aligned_to(decay, 4) || !aligned_to(beta, 4) || !aligned_to(lengths, 4) ||
        !aligned_to(state_in, 4) || !aligned_to(state_out, 4) || !aligned_to(ckpt, 16)) return CAWN_EINVAL;
    a.q = q, a.k = k, a.v = v, a.decay = decay, a.beta = beta, a.lengths = lengths, a.state_in = (const float *)state_in, a.o = o, a.state_out = (float *)state_out;
    a.vec4 = a.V % 4 == 0 && aligned_to(state_in, 16) && aligned_to(state_out, 16);
    (void)workspace, (void)workspace_bytes;
    return delta::launch_token(a, d->bf16, (hipStream_t)stream);
}

int cawn_delta_rule_bwd(const cawn_delta_desc *d, const void *q, const void *k, const void *v, const float *decay, const float *beta, const int32_t *lengths,
                        const void *ckpt, const void *dO, const void *dstate_out, void *dq, void *dk, void *dv, float *ddecay, float *dbeta, void *dstate_in,
                        void *workspace, size_t workspace_bytes, void *stream)
{
    return CAWN_EUNSUPPORTED;
}

} // extern "C"
