// Gated delta rule: argument checks, sizes and the choice of a form.
#include "cawn_delta.hpp"

using namespace cawn;
using namespace cawn::ops;
using cawn::delta::Args;

using cawn::delta::Sizes;

namespace {

// How a row's chunks are cut into segments.  A segment costs each of its chunks twice (what it makes of a state, then its outputs) and
// one link of the join, so two segments gain nothing; many shorten the two passes until the chip is full or the links cost as much.
// Full are 256 CUs with the scan's workgroups that one holds; beyond that a second round would begin.
// (Whole calls, for 512, 768 and 1,024 workgroups: 8 x 8,192 tokens of 12 heads of 64, bf16, training, three to a CU: 1,594, 1,477, 1,554 us;
// 4 x 4,096 tokens of 8 heads of 128, the same, two to a CU: 722, 832, 809 us.)
// With workgroups to spare, chunks / m links of m chunks each take least where m^2 is the chunks times the ratio of a link's time to that of a chunk's
// two passes.  The ratio is not one number (a 19th to a 24th by the kernels' times, and the passes' begins and ends beside), so the rule's is the one
// that served best (us for 6, 9, 13, 19 and 26: fp32, 1,024 tokens of 8 heads of 64 53, 53, 53, 47, 47, 4,096 of 12 heads 97, 91, 91, 99, 99, 8,192 of 8
// heads 128, 123, 123, 133, 133, 16,384 of them 218, 207, 197, 195, 195; bf16 training, 8,192 of them 254, 245, 245, 256, 256).
void cut(Args *a, bool bf16)
{
    int columns;
    const long long slots = 256LL * delta::scan_held(a->K, a->VT, bf16, &columns);
    const long long groups = (long long)a->B * a->H * ceil_div(a->VT, columns);
    const long long want = groups > 0 ? slots / groups : 1;
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
    cut(a, d->bf16 != 0);
    return CAWN_OK;
}

// Byte offsets.  Kept for the backward: states and u [B H][chunks] in tiles, gates, T, A of the segments.
// Scratch of the forward: gates, A and T (unless kept), b and the begins of the segments; of the backward: dR and dS of every
// chunk, b and the ends of the segments.
struct Layout { size_t u, gates, t, a, ckpt; size_t fwd_gates, fwd_a, fwd_t, b, s, fwd; size_t ds, rb, rs, bwd; };
Layout layout_of(const Args &a)
{
    Layout l;
    const Sizes z(a.K, a.V);
    const size_t heads = (size_t)a.B * a.H, all = heads * a.chunks, segs = a.segments > 1 ? heads * a.segments : 0;
    const size_t gates = (all * delta::GATE_FLOATS * 4 + 1023) / 1024 * 1024, am = segs * z.KP * z.KP * 4, states = segs * z.st * 1024;
    l.u = all * z.st * 1024;
    l.gates = l.u + all * z.ut * 1024;
    l.t = l.gates + gates;
    l.a = l.t + all * delta::OPERAND_BYTES;
    l.ckpt = l.a + am;
    l.fwd_gates = 0;
    l.fwd_a = gates;
    l.fwd_t = l.fwd_a + am;
    l.b = l.fwd_t + all * delta::OPERAND_BYTES;
    l.s = l.b + states;
    l.fwd = l.s + states;
    l.ds = all * z.ut * 1024;
    l.rb = l.ds + all * z.st * 1024;
    l.rs = l.rb + states;
    l.bwd = l.rs + states;
    return l;
}

// the checkpoint's parts
void keep(Args *a, const Layout &l, void *ckpt)
{
    const Sizes z(a->K, a->V);
    char *p = (char *)ckpt;
    a->s_tiles = p, a->s_chunk = (size_t)z.st * 1024, a->s_row = (size_t)a->chunks * a->s_chunk;
    a->u_tiles = p + l.u, a->u_chunk = (size_t)z.ut * 1024, a->u_row = (size_t)a->chunks * a->u_chunk;
    a->gates = (float *)(p + l.gates), a->t_ops = p + l.t, a->seg_a = p + l.a;
}

// more workgroups than a grid has
bool too_many(const Args &a)
{
    const long long most = a.segments > a.chunks ? a.segments : a.chunks;
    return (long long)a.B * a.H * ceil_div(a.VT + 8, 4) > 0x7fffffffLL / (most > 0 ? most : 1);
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
    return check(d, &a) != CAWN_OK ? 0 : layout_of(a).ckpt;
}

size_t cawn_delta_workspace_bytes(const cawn_delta_desc *d)
{
    Args a;
    if (check(d, &a) != CAWN_OK) return 0;
    const Layout l = layout_of(a);
    const size_t bytes = l.fwd > l.bwd ? l.fwd : l.bwd;
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
    const int e = d->bf16 ? 2 : 4, w = 16 / e;
    a.vecq = a.K % 8 == 0 && a.qst % w == 0 && a.qsb % w == 0 && aligned_to(q, 16) && aligned_to(k, 16);
    // Token by token up to TOKEN_MAX.  (us token by token and by chunks, bf16: 12 heads of 64, 8 tokens 10.9 and 19.3, 16 tokens 19.3 and 19.2, 32 tokens
    // 35.8 and 19.6; 32 rows of 32 heads of 128, 16 tokens 105 and 86, 32 tokens 190 and 91.  Calls of up to 16 tokens need no workspace, so
    // the line is there for many rows as well.)
    if (a.L <= delta::TOKEN_MAX && !ckpt) return delta::launch_token(a, d->bf16, s);
    const Layout l = layout_of(a);
    if (!workspace || workspace_bytes < l.fwd || !aligned_to(workspace, 256)) return CAWN_EWORKSPACE;
    if (too_many(a)) return CAWN_EUNSUPPORTED;
    a.veco = a.V % 4 == 0 && a.ost % 4 == 0 && a.osb % 4 == 0 && aligned_to(o, 4 * e);
    char *ws = (char *)workspace;
    a.gates = (float *)(ws + l.fwd_gates), a.seg_a = ws + l.fwd_a, a.t_ops = ws + l.fwd_t, a.seg_b = ws + l.b, a.seg_s = ws + l.s;
    if (ckpt) keep(&a, l, ckpt);
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
    const Layout l = layout_of(a);
    if (!workspace || workspace_bytes < l.bwd || !aligned_to(workspace, 256)) return CAWN_EWORKSPACE;
    if (too_many(a)) return CAWN_EUNSUPPORTED;
    a.q = q, a.k = k, a.v = v, a.decay = decay, a.beta = beta, a.lengths = lengths, a.dO = dO, a.dstate_out = (const float *)dstate_out;
    a.dq = dq, a.dk = dk, a.dv = dv, a.ddecay = ddecay, a.dbeta = dbeta, a.dstate_in = (float *)dstate_in;
    a.vecq = a.K % w == 0 && a.qst % w == 0 && a.qsb % w == 0 && aligned_to(q, 16) && aligned_to(k, 16);
    a.veco = a.V % w == 0 && a.ost % w == 0 && a.osb % w == 0 && aligned_to(dO, 16);
    a.vecd = a.K % 4 == 0 && a.qst % 4 == 0 && a.qsb % 4 == 0 && aligned_to(dq, 4 * e) && aligned_to(dk, 4 * e);
    keep(&a, l, const_cast<void *>(ckpt));
    char *ws = (char *)workspace;
    a.dr_tiles = ws, a.ds_tiles = ws + l.ds, a.seg_b = ws + l.rb, a.seg_s = ws + l.rs;
    hipStream_t s = (hipStream_t)stream;
    if (int r = delta::launch_back(a, d->bf16, s)) return r;
    return dq || dk || dv || ddecay || dbeta ? delta::launch_gradients(a, d->bf16, s) : CAWN_OK;
}

} // extern "C"
