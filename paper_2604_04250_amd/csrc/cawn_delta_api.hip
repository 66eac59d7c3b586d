// Gated delta rule: argument checks, sizes and the choice of a form.
#include "cawn_delta.hpp"

using namespace cawn;
using namespace cawn::ops;
using cawn::delta::Args;

using cawn::delta::Sizes;
using cawn::delta::StateArgs;

namespace {

constexpr size_t SPAN_BYTES = 128u << 20;

// How a row's chunks are cut into segments.  A segment costs each of its chunks twice (what it makes of a state, then its outputs) and
// one link of the join, so two segments gain nothing; many shorten the two passes until the chip is full or the links cost as much.
void cut(Args *a)
{
    const long long groups = (long long)a->B * a->H * ceil_div(a->VT, 4);
    const long long want = groups > 0 ? 768 / groups : 1;
    a->segments = 1, a->seg_chunks = a->chunks;
    if (want < 3 || a->chunks < 6) return;
    long long m = ceil_div(a->chunks, want);
    while (m * m * 13 < a->chunks) ++m;
    const long long segments = ceil_div(a->chunks, m);
    if (segments < 3) return;
    a->segments = (int)segments, a->seg_chunks = (int)m;
}

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
    a->VT = (int)ceil_div(d->V, 16);
    if ((long long)d->B * d->H * ceil_div(d->V, 16) > 0x7fffffffLL) return CAWN_EUNSUPPORTED;
    cut(a);
    return CAWN_OK;
}

// Chunks that the launches of a call treat at once: what they hand on to each other through the workspace is then still in the
// 256 MiB memory-side cache, and the workspace does not grow with the sequence.
int span_of(const Args &a, size_t per_chunk)
{
    const long long room = (long long)(SPAN_BYTES / ((size_t)a.B * a.H * per_chunk));
    return (int)(room < 1 ? 1 : room < a.chunks ? room : a.chunks > 1 ? a.chunks : 1);
}

struct Layout { size_t t, a, b, s, slots, carry, bytes; int span; };
Layout forward_layout(const Args &a, const Sizes &z)
{
    Layout l{};
    const size_t rows = (size_t)a.B * a.H;
    l.t = (rows * a.chunks * delta::GATE_FLOATS * 4 + 1023) / 1024 * 1024;
    l.a = l.t + rows * a.chunks * 18 * 1024;
    l.b = l.a + (a.segments > 1 ? rows * a.segments * z.KP * z.KP * 4 : 0);
    l.s = l.b + (a.segments > 1 ? rows * a.segments * z.st * 1024 : 0);
    l.bytes = l.s + (a.segments > 1 ? rows * a.segments * z.st * 1024 : 0);
    return l;
}

Layout backward_layout(const Args &a, const Sizes &z)
{
    Layout l{};
    const size_t rows = (size_t)a.B * a.H;
    l.span = span_of(a, z.bslot);
    l.slots = rows * l.span * z.bslot;
    l.carry = rows * z.st * 1024;
    l.bytes = l.slots + l.carry;
    return l;
}

// states [B H][chunks + 1], then u [B H][chunks], in tiles
size_t ckpt_bytes(const Args &a, const Sizes &z) { return (size_t)a.B * a.H * ((size_t)(a.chunks + 1) * z.st + (size_t)a.chunks * z.ut) * 1024; }

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
    return check(d, &a) != CAWN_OK ? 0 : ckpt_bytes(a, Sizes(a.K, a.V, 1));
}

size_t cawn_delta_workspace_bytes(const cawn_delta_desc *d)
{
    Args a;
    if (check(d, &a) != CAWN_OK) return 0;
    const Sizes z(a.K, a.V, d->bf16 ? 1 : 3);
    const size_t f = forward_layout(a, z).bytes, r = backward_layout(a, z).bytes, bytes = f > r ? f : r;
    return bytes > 256 ? bytes : 256;
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
    hipStream_t s = (hipStream_t)stream;
    // token by token up to TOKEN_MAX
    if (a.L <= delta::TOKEN_MAX && !ckpt) return delta::launch_token(a, d->bf16, s);
    const int e = d->bf16 ? 2 : 4, w = 16 / e;
    const Sizes z(a.K, a.V, d->bf16 ? 1 : 3);
    const Layout l = forward_layout(a, z);
    if (!workspace || workspace_bytes < l.bytes || !aligned_to(workspace, 256)) return CAWN_EWORKSPACE;
    if ((long long)a.B * a.H * (a.segments > a.chunks ? a.segments : a.chunks) * ceil_div(a.VT + z.KP / 16, 4) > 0x7fffffffLL) return CAWN_EUNSUPPORTED;
    a.vecq = a.K % w == 0 && a.qst % w == 0 && a.qsb % w == 0 && aligned_to(q, 16) && aligned_to(k, 16);
    a.veco = a.V % 4 == 0 && a.ost % 4 == 0 && a.osb % 4 == 0 && aligned_to(o, 4 * e);
    char *ws = (char *)workspace;
    a.gates = (float *)ws, a.t_ops = ws + l.t, a.seg_a = ws + l.a, a.seg_b = ws + l.b, a.seg_s = ws + l.s;
    if (ckpt) {
        a.s_tiles = (char *)ckpt, a.s_chunk = (size_t)z.st * 1024, a.s_row = (size_t)(a.chunks + 1) * a.s_chunk;
        a.u_tiles = a.s_tiles + (size_t)a.B * a.H * a.s_row, a.u_chunk = (size_t)z.ut * 1024, a.u_row = (size_t)a.chunks * a.u_chunk;
    }
    if (int r = delta::launch_system(a, d->bf16, s)) return r;
    return delta::launch_scan(a, d->bf16, s);
}

int cawn_delta_rule_bwd(const cawn_delta_desc *d, const void *q, const void *k, const void *v, const float *decay, const float *beta, const int32_t *lengths,
                        const void *ckpt, const void *dO, const void *dstate_out, void *dq, void *dk, void *dv, float *ddecay, float *dbeta, void *dstate_in,
                        void *workspace, size_t workspace_bytes, void *stream)
{
    Args a;
    if (int r = check(d, &a)) return r;
    if (a.B == 0) return CAWN_OK;
    if (a.L > 0 && (!q || !k || !v || !decay || !beta || !ckpt || !dO)) return CAWN_EINVAL;
    if (misaligned(d, q) || misaligned(d, k) || misaligned(d, v) || misaligned(d, dO) || misaligned(d, dq) || misaligned(d, dk) || misaligned(d, dv) ||
        !aligned_to(decay, 4) || !aligned_to(beta, 4) || !aligned_to(lengths, 4) || !aligned_to(ckpt, 16) || !aligned_to(dstate_out, 4) ||
        !aligned_to(ddecay, 4) || !aligned_to(dbeta, 4) || !aligned_to(dstate_in, 4)) return CAWN_EINVAL;
    const int e = d->bf16 ? 2 : 4, w = 16 / e;
    const Sizes z(a.K, a.V, d->bf16 ? 1 : 3);
    const Layout l = backward_layout(a, z);
    if (!workspace || workspace_bytes < l.bytes || !aligned_to(workspace, 256)) return CAWN_EWORKSPACE;
    if ((long long)a.B * a.H * l.span > 0x7fffffffLL) return CAWN_EUNSUPPORTED;
    a.q = q, a.k = k, a.v = v, a.decay = decay, a.beta = beta, a.lengths = lengths, a.dO = dO;
    a.dq = dq, a.dk = dk, a.dv = dv, a.ddecay = ddecay, a.dbeta = dbeta;
    a.vecq = a.K % w == 0 && a.qst % w == 0 && a.qsb % w == 0 && aligned_to(q, 16) && aligned_to(k, 16);
    a.veco = a.V % w == 0 && a.ost % w == 0 && a.osb % w == 0 && aligned_to(dO, 16);
    a.ws = (char *)workspace;
    a.span = l.span;
    a.s_tiles = (char *)const_cast<void *>(ckpt), a.s_chunk = (size_t)z.st * 1024, a.s_row = (size_t)(a.chunks + 1) * a.s_chunk;
    a.u_tiles = a.s_tiles + (size_t)a.B * a.H * a.s_row, a.u_chunk = (size_t)z.ut * 1024, a.u_row = (size_t)a.chunks * a.u_chunk;
    StateArgs t{};
    t.B = a.B, t.L = a.L, t.H = a.H, t.K = a.K, t.V = a.V, t.VT = a.VT, t.chunks = a.chunks, t.span = l.span, t.lengths = a.lengths;
    t.ws = a.ws, t.slot = z.bslot, t.x_at = (size_t)(z.wf + z.kf) * 1024, t.gates_at = t.x_at + (size_t)z.ut * 1024, t.y_at = t.gates_at + 3 * 1024;
    t.s_tiles = a.ws + t.y_at + (size_t)z.st * 1024, t.s_row = (size_t)l.span * z.bslot, t.s_chunk = z.bslot;
    t.x_tiles = a.ws + t.x_at, t.x_row = t.s_row, t.x_chunk = z.bslot;
    t.carry = a.ws + l.slots;
    t.begin = (const float *)dstate_out, t.end = (float *)dstate_in;
    hipStream_t s = (hipStream_t)stream;
    for (a.c1 = a.chunks;; a.c1 = a.c0) {       // from the last chunks to the first
        a.c0 = a.c1 > l.span ? a.c1 - l.span : 0;
        t.c0 = a.c0, t.c1 = a.c1, t.s_first = t.x_first = a.c0;
        t.first = a.c1 == a.chunks, t.last = a.c0 == 0;
        if (a.c1 > a.c0)
            if (int r = delta::launch_adjoint(a, d->bf16, s)) return r;
        if (int r = delta::launch_states(t, d->bf16, true, s)) return r;
        if (a.c1 > a.c0)
            if (int r = delta::launch_gradients(a, d->bf16, s)) return r;
        if (a.c0 == 0) return CAWN_OK;
    }
}

} // extern "C"
