// Selective state space scan: argument checks, sizes and the choice of a form.
#include "cawn_select.hpp"

using namespace cawn;
using namespace cawn::ops;
using cawn::select::Args;
using cawn::select::TILE;

namespace {

// How a row's tiles are cut into segments.  Each but the last costs its tokens twice, whatever their number, and one link of the chain; more of them fill the
// chip and even out its rounds.
// One segment: where its waves fill the chip alone, or rows are so short that the passes over segments cost more than a wave's way along the row.  For each wave
// on a SIMD (1,024 in all) a pass over segments takes 0.45 us a token, backward 1.05; a wave alone takes 0.38 for its way, two on a SIMD 0.57, backward 1.0 and
// 1.6: they are even at 890 and 1,300 waves, 980 and 1,560.  What else segments cost, launches and the chain, is as long as 48 tokens, backward 24.  (us, cut and
// in one: 64 x 256 tokens of 1,024 channels 145, 102, training 463, 368; 64 x 32 43, 21, training 106, 68; 16 x 64 29, 30, training 76, 103; 64 x 1,000 of 4,096
// channels 1,577, 933; 16 x 1,024 of 2,048 channels 232, 379.)
// Else 8,192 waves in all, backward 6,144, three or four rounds of what the chip holds; beyond 64 segments, where the chain costs more than the rounds gain,
// half of that, and two tiles rather than one where that leaves 4,096 (4 x 512 tokens of 4,096 channels 88, 80).
// (us a pass for 4,096, 6,144, 8,192 and 16,384 waves, forward: 2 x 32,768 tokens of 4,096 channels 1,790, 1,720, 1,660, 1,637, training 8 x 8,192 of 768
// channels 1,326, 1,290, 1,296, 1,292; backward, 2,048, 4,096, 6,144, 8,192 and 12,288: the latter 1,326, 1,306, 1,241, 1,287, 1,251.)
void cut(Args *a, bool bwd)
{
    const long long columns = (long long)a->B * a->G * a->cbg * (a->NB > 1 ? a->NB : a->wide), waves = bwd ? 6144 : 8192;
    const long long even = columns <= 1024 && a->NB < 8 ? (bwd ? 980 : 890) : bwd ? 1560 : 1300;       // (a workgroup of eight waves has two on a SIMD)
    a->segments = 1, a->seg_tiles = a->tiles > 0 ? a->tiles : 1;
    if (a->tiles < 2 || columns >= even || (long long)a->L * (even - columns) <= even * (bwd ? 24 : 48)) return;
    long long want = columns > 0 ? waves / columns : 1;
    if (want > 64) want = waves / 2 / columns > 64 ? waves / 2 / columns : 64;
    if (want > select::SEGMENTS_MAX) want = select::SEGMENTS_MAX;
    a->seg_tiles = (int)ceil_div(a->tiles, want);
    if (a->seg_tiles == 1 && columns * (a->tiles / 2) >= 4096) a->seg_tiles = 2;
    a->segments = (int)ceil_div(a->tiles, a->seg_tiles);
}

// More bytes than are counted, or more tiles of B and C.
bool too_many(const Args &a) { return (double)a.B * (a.tiles + 1.) * a.Dp * (a.NP * a.NB) > 1e17 || (double)a.B * a.tiles * a.G > 0x7fffffff; }

// The passes of the tiled form, whose workgroups take a segment of columns each, and the launch of the other form.  (The chain has links only where the columns are
// few, and the other launches go round or are several.)
bool tiles_fit(const Args &a) { return launchable((double)a.B * a.segments * a.G * a.cbg, 64 * (a.NB > 1 ? a.NB : a.wide)); }
bool by_token(const Args &a) { return a.L <= select::TOKEN_MAX; }
bool tokens_fit(const Args &a) { return launchable((double)ceil_div((long long)a.B * a.D * select::token_lanes(a), 256), 256); }

int check(const cawn_scan_desc *d, bool bwd, Args *a)
{
    if (!d || d->B < 0 || d->L < 0 || d->D <= 0 || d->N <= 0 || d->G < 0 || (d->bf16 & ~1) || (d->dt_softplus & ~1)) return CAWN_EINVAL;
    const int G = d->G ? d->G : 1;
    if (d->D % G) return CAWN_EINVAL;
    if (d->N > select::N_MAX) return CAWN_EUNSUPPORTED;
    *a = Args{};
    a->B = d->B, a->L = d->L, a->D = d->D, a->N = d->N, a->G = G, a->cg = d->D / G, a->softplus = d->dt_softplus;
    const long long gn = (long long)G * d->N;
    a->xst = d->x_stride_t ? d->x_stride_t : d->D, a->dst = d->dt_stride_t ? d->dt_stride_t : d->D, a->bst = d->bc_stride_t ? d->bc_stride_t : gn;
    a->zst = d->z_stride_t ? d->z_stride_t : d->D, a->yst = d->y_stride_t ? d->y_stride_t : d->D;
    if (a->xst < d->D || a->dst < d->D || a->bst < gn || a->zst < d->D || a->yst < d->D) return CAWN_EINVAL;
    a->xsb = d->x_stride_b ? d->x_stride_b : a->xst * d->L, a->dsb = d->dt_stride_b ? d->dt_stride_b : a->dst * d->L;
    a->bsb = d->bc_stride_b ? d->bc_stride_b : a->bst * d->L, a->zsb = d->z_stride_b ? d->z_stride_b : a->zst * d->L;
    a->ysb = d->y_stride_b ? d->y_stride_b : a->yst * d->L;
    a->NB = d->N <= 16 ? 1 : d->N <= 32 ? 2 : d->N <= 64 ? 4 : 8;
    a->NP = (int)ceil_div(ceil_div(d->N, a->NB), 4) * 4;
    a->cpg = (int)ceil_div(a->cg, 64);
    a->wide = a->NB > 1 ? 1 : a->cpg < 4 ? a->cpg : 4;
    a->cbg = (int)ceil_div(a->cpg, a->wide);
    a->parts = a->cbg;
    // places of a channel in its row and of a token among 16 are 32 bits of bytes; tokens of a row and places of channels are counted in 32 bits
    const long long wide = 1 << 25;
    if (d->D > wide || a->xst > wide || a->dst > wide || a->zst > wide || a->yst > wide || d->L > 1 << 30 || (long long)a->cpg * G > 1 << 24) return CAWN_EUNSUPPORTED;
    a->Dp = a->cpg * G * 64;
    a->tiles = (int)ceil_div(d->L, TILE);
    cut(a, bwd);
    return too_many(*a) || !(tiles_fit(*a) || (!bwd && by_token(*a) && tokens_fit(*a))) ? CAWN_EUNSUPPORTED : CAWN_OK;
}

// Byte offsets.  Kept for the backward: B and C, states before each tile.  Scratch: forward B and C (unless kept), of segments their b, sum of delta and
// begin; backward the same of its own segments, and the partial sums.
struct Layout { size_t ck, ckpt; size_t b, g, s, fwd; size_t pbc, pa, bwd; };
Layout layout_of(const Args &f, const Args &r)
{
    const size_t npt = f.NP * f.NB, state = (size_t)f.Dp * npt * 4;
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    Layout l;
    const size_t bc = up((size_t)f.B * f.tiles * f.G * npt * 2 * TILE * 4);
    l.ck = bc;
    l.ckpt = bc + (size_t)f.B * f.tiles * state;
    const size_t fs = f.segments > 1 ? (size_t)f.B * f.segments : 0, rs = r.segments > 1 ? (size_t)r.B * r.segments : 0;
    auto parts = [&](size_t n, size_t *b, size_t *g, size_t *s) {
        *s = *b + n * state;
        *g = *s + n * state;
        return up(*g + n * f.Dp * 4);
    };
    l.b = bc;
    l.fwd = parts(fs, &l.b, &l.g, &l.s);
    size_t b = 0, g, s;
    l.pbc = parts(rs, &b, &g, &s);
    l.pa = l.pbc + up((size_t)r.B * r.tiles * TILE * r.G * r.parts * 2 * npt * 4);
    l.bwd = l.pa + (size_t)r.B * r.segments * r.Dp * (npt + 2) * 4;
    return l;
}

void segments_of(Args *a, char *ws, size_t begin)
{
    const size_t n = (size_t)a->B * a->segments, state = (size_t)a->Dp * a->NP * a->NB * 4;
    a->seg_b = (float *)(ws + begin), a->seg_s = (float *)(ws + begin + n * state), a->seg_g = (float *)(ws + begin + 2 * n * state);
}

bool misaligned(const cawn_scan_desc *d, const void *p) { return !aligned_to(p, d->bf16 ? 2 : 4); }

} // namespace

extern "C" {

size_t cawn_selective_scan_state_bytes(const cawn_scan_desc *d)
{
    Args a;
    return check(d, false, &a) != CAWN_OK ? 0 : (size_t)a.B * a.D * a.N * 4;
}

size_t cawn_selective_scan_ckpt_bytes(const cawn_scan_desc *d)
{
    Args a;
    return check(d, false, &a) != CAWN_OK || !tiles_fit(a) ? 0 : layout_of(a, a).ckpt;
}

size_t cawn_selective_scan_workspace_bytes(const cawn_scan_desc *d)
{
    Args a, r;
    if (check(d, false, &a) != CAWN_OK) return 0;
    if (check(d, true, &r) != CAWN_OK) return by_token(a) && tokens_fit(a) ? 256 : 0;         // (what uses none)
    const Layout l = layout_of(a, r);
    const size_t bytes = l.fwd > l.bwd ? l.fwd : l.bwd;
    return bytes > 256 ? bytes : 256;
}

size_t cawn_selective_scan_serve_workspace_bytes(const cawn_scan_desc *d)
{
    Args a;
    if (check(d, false, &a) != CAWN_OK || (!by_token(a) && !tiles_fit(a))) return 0;
    const size_t bytes = by_token(a) ? 0 : layout_of(a, a).fwd;
    return bytes > 256 ? bytes : 256;
}

int cawn_selective_scan_fwd(const cawn_scan_desc *d, const void *x, const void *dt, const float *A, const void *Bm, const void *Cm, const float *Dskip, const void *z,
                            const float *dt_bias, const int32_t *lengths, const void *state_in, void *y, void *state_out, void *ckpt, void *workspace,
                            size_t workspace_bytes, void *stream)
{
    Args a;
    if (int r = check(d, false, &a)) return r;
    const bool tokens = by_token(a) && !ckpt;
    if (!(tokens ? tokens_fit(a) : tiles_fit(a))) return CAWN_EUNSUPPORTED;
    if (a.B == 0) return CAWN_OK;
    if (!A || (a.L > 0 && (!x || !dt || !Bm || !Cm || !y))) return CAWN_EINVAL;
    if (misaligned(d, x) || misaligned(d, dt) || misaligned(d, Bm) || misaligned(d, Cm) || misaligned(d, z) || misaligned(d, y) || !aligned_to(A, 4) || !aligned_to(Dskip, 4) ||
        !aligned_to(dt_bias, 4) || !aligned_to(lengths, 4) || !aligned_to(state_in, 4) || !aligned_to(state_out, 4) || !aligned_to(ckpt, 16)) return CAWN_EINVAL;
    a.x = x, a.dt = dt, a.A = A, a.Bm = Bm, a.Cm = Cm, a.Dk = Dskip, a.z = z, a.bias = dt_bias, a.lengths = lengths, a.state_in = (const float *)state_in;
    a.y = y, a.state_out = (float *)state_out;
    hipStream_t s = (hipStream_t)stream;
    if (tokens) return select::launch_token(a, d->bf16, s);
    const Layout l = layout_of(a, a);
    if (!workspace || workspace_bytes < l.fwd || !aligned_to(workspace, 256)) return CAWN_EWORKSPACE;
    a.bc = (float *)(ckpt ? ckpt : workspace);
    if (ckpt) a.ck = (float *)((char *)ckpt + l.ck);
    segments_of(&a, (char *)workspace, l.b);
    return select::launch_forward(a, d->bf16, s);
}

int cawn_selective_scan_bwd(const cawn_scan_desc *d, const void *x, const void *dt, const float *A, const void *Bm, const void *Cm, const float *Dskip, const void *z,
                            const float *dt_bias, const int32_t *lengths, const void *ckpt, const void *dy, const void *dstate_out, void *dx, void *ddt, float *dA,
                            void *dBm, void *dCm, float *dDskip, void *dz, float *ddt_bias, void *dstate_in, void *workspace, size_t workspace_bytes, void *stream)
{
    Args a;
    if (int r = check(d, true, &a)) return r;
    if ((dz && !z) || (dDskip && !Dskip) || (ddt_bias && !dt_bias)) return CAWN_EINVAL;
    if (misaligned(d, x) || misaligned(d, dt) || misaligned(d, Bm) || misaligned(d, Cm) || misaligned(d, z) || misaligned(d, dy) || misaligned(d, dx) || misaligned(d, ddt) ||
        misaligned(d, dBm) || misaligned(d, dCm) || misaligned(d, dz) || !aligned_to(A, 4) || !aligned_to(Dskip, 4) || !aligned_to(dt_bias, 4) || !aligned_to(lengths, 4) ||
        !aligned_to(ckpt, 16) || !aligned_to(dstate_out, 4) || !aligned_to(dA, 4) || !aligned_to(dDskip, 4) || !aligned_to(ddt_bias, 4) || !aligned_to(dstate_in, 4))
        return CAWN_EINVAL;
    hipStream_t s = (hipStream_t)stream;
    const int NPT = a.NP * a.NB, add = d->accumulate_param_grads;
    const bool params = dA || dDskip || ddt_bias;
    const select::ParamSums sums{dA, dDskip, ddt_bias, a.N, NPT, a.Dp, a.cpg, a.cg};
    if (a.B == 0) {         // the sums over nothing
        if (params && !add) launch_sums(nullptr, 0, (long long)a.Dp * (NPT + 2), sums, 0, s);
        return launched();
    }
    if (!A || (a.L > 0 && (!x || !dt || !Bm || !Cm || !ckpt || !dy))) return CAWN_EINVAL;
    Args f;
    check(d, false, &f);
    const Layout l = layout_of(f, a);
    if (!workspace || workspace_bytes < l.bwd || !aligned_to(workspace, 256)) return CAWN_EWORKSPACE;
    a.x = x, a.dt = dt, a.A = A, a.Bm = Bm, a.Cm = Cm, a.Dk = Dskip, a.z = z, a.bias = dt_bias, a.lengths = lengths, a.dy = dy, a.dstate_out = (const float *)dstate_out;
    a.dx = dx, a.ddt = ddt, a.dB = dBm, a.dC = dCm, a.dz = dz, a.dstate_in = (float *)dstate_in;
    a.bc = (float *)const_cast<void *>(ckpt), a.ck = (float *)((char *)const_cast<void *>(ckpt) + l.ck);
    char *ws = (char *)workspace;
    segments_of(&a, ws, 0);
    a.part_bc = dBm || dCm ? (float *)(ws + l.pbc) : nullptr;
    a.part_a = params ? (float *)(ws + l.pa) : nullptr;
    if (int r = select::launch_backward(a, d->bf16, s)) return r;
    return select::launch_bc_sums(a, d->bf16, sums, add, s);
}

} // extern "C"
