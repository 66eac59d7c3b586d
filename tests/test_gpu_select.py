"""Selective state space scan, forward and backward, against 64 bits through the C ABI."""
import numpy as np
import pytest
import torch

import layer_ref as R
from layer_util import EPS, ROUND16, Scan, reference_inputs, rel_err, scan_inputs, untouched

pytestmark = pytest.mark.gpu


def tolerance(L, bf16):
    """A factor exp(delta A) is off by 2^-24 for itself and for each rounding of its exponent (three, weighed by an exponent that is below one where the
    factor counts), an update by three more; what is m tokens old has met m of them, and it counts as far as the memory goes, 256 tokens at most with
    the decays of these inputs (0.001 is the smallest, and it takes all of them rounding one way).  A sum of N products, or over a channel's neighbours, is a
    few times its root mean square in magnitude: 4.  Outputs in bf16 add their rounding."""
    return 4 * EPS * (16 + 4 * min(L, 256)) + (ROUND16 if bf16 else 0.0)


# B, L, D, N, G, z, ragged
SHAPES = [
    (1, 1, 768, 16, 1, True, False), (3, 1, 70, 16, 1, True, True), (2, 7, 96, 16, 2, False, False), (4, 16, 33, 5, 1, True, True), (2, 3, 6, 1, 3, True, False),
    (2, 5, 40, 128, 1, True, True), (3, 9, 20, 24, 4, False, True), (2, 2, 65, 64, 1, True, False),
    (2, 17, 130, 16, 1, True, False), (5, 100, 64, 16, 1, True, True), (3, 129, 200, 16, 2, False, True), (1, 1000, 64, 16, 1, True, False), (2, 333, 48, 4, 3, True, True),
    (2, 65, 70, 8, 1, True, False), (2, 50, 24, 3, 1, False, False), (2, 90, 100, 24, 2, True, True), (1, 161, 72, 64, 1, True, False), (2, 40, 130, 128, 2, False, True),
    (1, 200, 5, 16, 5, True, False), (3, 48, 320, 16, 1, True, True), (1, 33, 600, 12, 2, True, False), (1, 31, 64, 100, 1, True, False),
]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L,D,N,G,z,ragged", SHAPES)
def test_forward(B, L, D, N, G, z, ragged, bf16):
    i = scan_inputs(B, L, D, N, G, bf16, seed=L + D + N, z=z, ragged=ragged)
    s = Scan(i, bf16, ckpt=False).forward()
    torch.cuda.synchronize()
    y, state = R.scan_fwd(**reference_inputs(i))
    assert rel_err(s.y.float().cpu(), y) <= tolerance(L, bf16)
    assert rel_err(s.state_out.cpu(), state) <= tolerance(L, False)
    if ragged:
        for b, n in enumerate(i["lengths"]):
            assert bool((s.y[b, n:] == 0).all())
            if n == 0:
                assert torch.equal(s.state_out[b], s.state_in[b])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L,D,N,G,z,ragged", SHAPES)
def test_backward(B, L, D, N, G, z, ragged, bf16):
    i = scan_inputs(B, L, D, N, G, bf16, seed=2 * L + D + N, z=z, ragged=ragged)
    s = Scan(i, bf16).forward().backward()
    torch.cuda.synchronize()
    y, state = R.scan_fwd(**reference_inputs(i))
    assert rel_err(s.y.float().cpu(), y) <= tolerance(L, bf16)          # with a checkpoint, also where the call is short
    assert rel_err(s.state_out.cpu(), state) <= tolerance(L, False)
    ref = R.scan_bwd(dy=i["dy"], dstate_out=i["dstate_out"], **reference_inputs(i))
    got = s.grads()
    for n, r in ref.items():
        if n == "dz" and not z:
            continue
        assert rel_err(got[n], r) <= tolerance(L, bf16 and n in ("dx", "ddt", "dBm", "dCm", "dz")), n


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("L", [9, 120])
def test_strides_and_alignment(L, bf16):
    """Rows that are parts of wider ones, at odd places of their memory; nothing is written between them."""
    B, D, N, G, extra = 2, 70, 10, 2, (70, 27, 13, 3, 1)
    i = scan_inputs(B, L, D, N, G, bf16, seed=L, z=True)
    s = Scan(i, bf16, extra=extra, offset=3).forward().backward()
    torch.cuda.synchronize()
    y, _ = R.scan_fwd(**reference_inputs(i))
    ref, got = R.scan_bwd(dy=i["dy"], dstate_out=i["dstate_out"], **reference_inputs(i)), s.grads()
    assert rel_err(s.y.float().cpu(), y) <= tolerance(L, bf16)
    for n, r in ref.items():
        assert rel_err(got[n], r) <= tolerance(L, bf16 and n in ("dx", "ddt", "dBm", "dCm", "dz")), n
    ex, ed, eb, ez, ey = extra
    assert untouched(s.y, ey)
    for n, e in (("x", ex), ("dt", ed), ("Bm", eb), ("Cm", eb), ("z", ez)):
        assert untouched(s.g[n], e), n
    short = Scan(i, bf16, extra=extra, offset=3, ckpt=False).forward()
    assert rel_err(short.y.float().cpu(), y) <= tolerance(L, bf16) and untouched(short.y, ey)


@pytest.mark.parametrize("L", [11, 70])
def test_without_softplus_skip_bias_and_gate(L):
    i = scan_inputs(2, L, 66, 16, 1, False, seed=4, z=False, skip=False, bias=False)
    i["dt"] = np.abs(i["dt"]) * 0.1
    s = Scan(i, False, softplus=0).forward().backward()
    k = dict(reference_inputs(i), softplus=False)
    assert rel_err(s.y.cpu(), R.scan_fwd(**k)[0]) <= tolerance(L, False)
    ref = R.scan_bwd(dy=i["dy"], dstate_out=i["dstate_out"], **k)
    for n in ("dx", "ddt", "dA", "dBm", "dCm", "dstate_in"):
        assert rel_err(s.grads()[n], ref[n]) <= tolerance(L, False), n


@pytest.mark.parametrize("L", [5, 100])
def test_no_state_no_gradient_of_a_state(L):
    i = scan_inputs(2, L, 66, 16, 1, False, seed=5)
    s = Scan(i, False).forward(state_in=None, state_out=None).backward(dstate=None)
    k = dict(reference_inputs(i), state_in=None)
    assert rel_err(s.y.cpu(), R.scan_fwd(**k)[0]) <= tolerance(L, False)
    ref = R.scan_bwd(dy=i["dy"], **k)
    for n in ref:
        assert rel_err(s.grads()[n], ref[n]) <= tolerance(L, False), n


@pytest.mark.parametrize("B,L,D", [(1, 900, 64), (2, 40, 200)])
def test_gradients_one_by_one_added_and_in_place(B, L, D):
    """Each gradient asked for alone is what it is with the others; parameters' are added on request; dstate_in may be dstate_out."""
    i = scan_inputs(B, L, D, 16, 1, False, seed=6)
    all_ = Scan(i, False).forward().backward().g
    for n, v in all_.items():
        one = Scan(i, False).forward().backward(want=(n,)).g
        assert torch.equal(one[n], v), n
        for m, w in one.items():
            assert m == n or bool(torch.isnan(w).all())
    added = Scan(i, False, accumulate=1).forward().backward(fill=0.5).g
    for n in ("A", "Dskip", "dt_bias"):
        assert torch.equal(added[n], 0.5 + all_[n]), n
    assert torch.equal(Scan(i, False).forward().backward(dstate="in place").g["state_in"], all_["state_in"])


@pytest.mark.parametrize("L,ckpt", [(1, False), (16, False), (16, True), (17, False), (700, False)])
def test_state_in_place_and_unused_slots(L, ckpt):
    """state_out may be state_in; a slot without tokens keeps its state bit for bit, NaN among it; lengths are clamped."""
    B, D, N = 4, 66, 16
    i = scan_inputs(B, L, D, N, 1, True, seed=7)
    i["lengths"] = np.array([L + 5, 0, -3, (L + 1) // 2], np.int32)
    i["state_in"][1, 0, 0] = np.nan
    s = Scan(i, True, ckpt=ckpt).forward()
    held = s.state_in.clone()
    t = Scan(i, True, ckpt=ckpt)
    t.forward(state_in=held, state_out=held)
    assert torch.equal(s.y, t.y) and torch.equal(s.state_out.view(torch.int32), held.view(torch.int32))
    for b in (1, 2):
        assert torch.equal(held[b].view(torch.int32), s.state_in[b].view(torch.int32))
    k = reference_inputs(i)
    y, state = R.scan_fwd(**k)
    assert rel_err(s.y.float().cpu(), y) <= tolerance(L, True)
    assert rel_err(s.state_out[[0, 3]].cpu(), state[[0, 3]]) <= tolerance(L, False)


def test_tokens_one_by_one_and_chunks_agree_with_the_whole():
    B, L, D, N, G = 2, 150, 130, 16, 2
    i = scan_inputs(B, L, D, N, G, False, seed=8)
    whole = Scan(i, False, ckpt=False).forward()
    for cuts in ([1] * 20 + [130], [16, 17, 64, 53], [149, 1]):
        state, at, ys = whole.state_in, 0, []
        for n in cuts:
            part = {k: v[:, at:at + n] if k in ("x", "dt", "Bm", "Cm", "z", "dy") else v for k, v in i.items()}
            s = Scan(part, False, ckpt=False).forward(state_in=state)
            state, at = s.state_out, at + n
            ys.append(s.y)
        assert at == L
        assert rel_err(torch.cat(ys, 1).cpu(), whole.y.cpu()) <= 2 * tolerance(L, False)
        assert rel_err(state.cpu(), whole.state_out.cpu()) <= 2 * tolerance(L, False)


@pytest.mark.parametrize("L", [10, 300])
def test_the_same_bits_again(L):
    i = scan_inputs(3, L, 200, 16, 2, True, seed=9, ragged=True)
    a, b = (Scan(i, True).forward().backward() for _ in range(2))
    assert torch.equal(a.y, b.y) and torch.equal(a.state_out, b.state_out)
    for n in a.g:
        assert torch.equal(a.g[n], b.g[n]), n


@pytest.mark.parametrize("ckpt", [False, True])
def test_a_value_that_is_not_finite_reaches_later_tokens_of_its_channel_alone(ckpt):
    B, L, D = 2, 90, 70
    i = scan_inputs(B, L, D, 16, 1, False, seed=10)
    clean = Scan(i, False, ckpt=ckpt).forward()
    i["x"][1, 40, 7] = np.inf
    s = Scan(i, False, ckpt=ckpt).forward()
    bad = ~torch.isfinite(s.y)
    assert bool(bad[1, 40:, 7].all()) and int(bad.sum()) == L - 40
    keep = ~bad
    assert torch.equal(s.y[keep], clean.y[keep])


@pytest.mark.parametrize("L", [12, 100])
def test_strong_forgetting_and_none(L):
    """Rates of minus infinity and of zero, steps so large that nothing is left and so small that nothing comes in."""
    i = scan_inputs(2, L, 64, 16, 1, False, seed=11)
    i["A"][:, 3], i["A"][:, 5], i["A"][:, 7] = -np.inf, 0.0, -3e38
    i["bias"][:20] = 30.0
    i["bias"][20:40] = -100.0
    s = Scan(i, False).forward()
    ref = dict(reference_inputs(i))
    ref["A"] = np.where(np.isinf(ref["A"]), -1e300, ref["A"].astype(np.float64))
    y, state = R.scan_fwd(**ref)
    # steps of 30 to 32 multiply states that do not forget; their sum over the tokens is no longer of the size of the others: against each channel's own
    for c in range(64):
        assert rel_err(s.y[..., c].cpu(), y[..., c]) <= 4 * tolerance(L, False), c
        assert rel_err(s.state_out[:, c].cpu(), state[:, c]) <= 4 * tolerance(L, False), c


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L,D,N,G", [(64, 1, 2100, 16, 1), (70, 2, 3000, 10, 3), (60, 1, 1500, 24, 1), (40, 1, 500, 128, 4)])
def test_steps_of_many_rows(B, L, D, N, G, bf16):
    """States in such number that a lane takes eight of them."""
    i = scan_inputs(B, L, D, N, G, bf16, seed=N, ragged=True)
    s = Scan(i, bf16, ckpt=False).forward()
    y, state = R.scan_fwd(**reference_inputs(i))
    assert rel_err(s.y.float().cpu(), y) <= tolerance(L, bf16)
    assert rel_err(s.state_out.cpu(), state) <= tolerance(L, False)
    held = s.state_in.clone()
    t = Scan(i, bf16, ckpt=False).forward(state_in=held, state_out=held)
    assert torch.equal(t.y, s.y) and torch.equal(held, s.state_out)


@pytest.mark.parametrize("L", [12, 100])
def test_gradients_with_a_rate_of_minus_infinity(L):
    """Its factor is 0, its own gradient 0 too, and the others' are those of a rate that is finite and forgets as completely."""
    i = scan_inputs(2, L, 64, 16, 1, False, seed=21)
    i["A"][:, 3] = -np.inf
    got = Scan(i, False).forward().backward().grads()
    ref = R.scan_bwd(dy=i["dy"], dstate_out=i["dstate_out"], **{**reference_inputs(i), "A": np.where(np.isinf(i["A"]), -1e9, i["A"])})
    assert np.all(got["dA"][:, 3] == 0)
    for n, r in ref.items():
        assert rel_err(got[n], r) <= tolerance(L, False), n


def test_long_rows_in_many_segments_against_short_ones():
    """One row of 4,096 tokens is cut into many segments, eight of them in another way; with the same tokens all agree."""
    D, L = 64, 4096
    i = scan_inputs(1, L, D, 16, 1, False, seed=12)
    one = Scan(i, False).forward().backward()
    many = {k: np.repeat(v, 40, 0) if v is not None and k in ("x", "dt", "Bm", "Cm", "z", "dy", "state_in", "dstate_out") else v for k, v in i.items()}
    m = Scan(many, False).forward().backward()
    tol = 2 * tolerance(L, False)
    assert rel_err(m.y[17:18].cpu(), one.y.cpu()) <= tol and rel_err(m.state_out[39:].cpu(), one.state_out.cpu()) <= tol
    for n in ("x", "dt", "Bm", "Cm", "z", "state_in"):
        assert rel_err(m.g[n][5:6].float().cpu(), one.g[n].float().cpu()) <= tol, n
    for n in ("A", "Dskip", "dt_bias"):
        assert rel_err(m.g[n].cpu() / 40, one.g[n].cpu()) <= tol, n


def test_gradients_against_differences():
    """The kernels' own forward, moved along a direction of each input in fp32: a step of 1/64 leaves (1/64)^2 of the third derivative and rounding of
    2^-24 of the sum's terms over the step, some 1e-3 of the root mean square of such directional derivatives together."""
    i = scan_inputs(2, 40, 24, 8, 2, False, seed=13, step=(0.05, 0.5))
    s = Scan(i, False).forward().backward()
    g = dict(zip(("x", "dt", "A", "Bm", "Cm", "Dk", "z", "bias", "state_in"), (s.grads()[n] for n in ("dx", "ddt", "dA", "dBm", "dCm", "dDskip", "dz", "ddt_bias", "dstate_in"))))
    r = np.random.Generator(np.random.PCG64(14))

    def value(j):
        t = Scan(j, False, ckpt=False).forward()
        return float((t.y.double().cpu().numpy() * i["dy"]).sum() + (t.state_out.double().cpu().numpy() * i["dstate_out"]).sum())

    for n, grad in g.items():
        v = r.standard_normal(i[n].shape).astype(np.float32)
        v /= np.sqrt((v * v).sum())
        h = 1 / 64
        want = (value({**i, n: i[n] + h * v}) - value({**i, n: i[n] - h * v})) / (2 * h)
        assert abs(float((grad * v).sum()) - want) <= 4e-3 * (float(np.sqrt((grad * grad).mean())) + abs(want)) + 1e-3, n


def test_graph_and_stream():
    """Captured on a stream of its own and replayed with other inputs, the program's own work between."""
    i, j = (scan_inputs(3, 200, 130, 16, 2, True, seed=k, ragged=True) for k in (15, 16))
    j["lengths"] = i["lengths"]
    want = Scan(j, True).forward().backward()
    s = Scan(i, True).forward().backward()
    first = [s.y.clone()] + [v.clone() for v in s.g.values()]
    new = Scan(j, True)
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    g = s.g
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            s.forward()
            from paper_2604_04250_amd import binding as K
            K.check(K.cawn_selective_scan_bwd(s.d, s.x, s.dt, s.A, s.Bm, s.Cm, s.Dk, s.z, s.bias, s.lengths, s.ckpt, s.dy, s.dstate_out, g["x"], g["dt"], g["A"], g["Bm"],
                                              g["Cm"], g["Dskip"], g["z"], g["dt_bias"], g["state_in"], s.ws))
    for k in range(3):
        for v in g.values():
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip([s.y] + list(g.values()), first):
            assert torch.equal(a, b)
        torch.ones(1000, device="cuda").sum()
    for n in ("x", "dt", "Bm", "Cm", "z", "dy", "A", "Dk", "bias", "state_in", "dstate_out"):
        getattr(s, n).copy_(getattr(new, n))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(s.y, want.y)
    for n in g:
        assert torch.equal(g[n], want.g[n]), n


@pytest.mark.parametrize("ckpt", [False, True])
def test_no_tokens_pass_the_state_and_its_gradient(ckpt):
    i = scan_inputs(2, 0, 70, 16, 1, False, seed=17)
    s = Scan(i, False, ckpt=ckpt).forward().backward()
    assert torch.equal(s.state_out, s.state_in) and torch.equal(s.g["state_in"], s.dstate_out)
    for n in ("A", "Dskip", "dt_bias"):
        assert bool((s.g[n] == 0).all()), n


def test_rows_far_apart():
    """A batch whose rows lie more than 2^31 elements from each other."""
    L, D, N, far = 40, 64, 16, (1 << 31) + 64
    i = scan_inputs(2, L, D, N, 1, True, seed=18)
    base = Scan(i, True).forward().backward()
    s = Scan(i, True)
    big = torch.empty(far + L * D, device="cuda", dtype=torch.bfloat16)
    out = torch.empty(far + L * D, device="cuda", dtype=torch.bfloat16)
    s.x = big.as_strided((2, L, D), (far, D, 1))
    s.x.copy_(base.x)
    s.y = out.as_strided((2, L, D), (far, D, 1))
    s.dy = s.y                                           # (gradients have the stride of what they belong to: a call without y's comes behind)
    s.d.x_stride_b = s.d.y_stride_b = far
    s.forward()
    torch.cuda.synchronize()
    assert torch.equal(s.y, base.y) and torch.equal(s.state_out, base.state_out)
    s.dy.copy_(base.dy)
    from paper_2604_04250_amd import binding as K
    dx = torch.empty(far + L * D, device="cuda", dtype=torch.bfloat16).as_strided((2, L, D), (far, D, 1))
    K.check(K.cawn_selective_scan_bwd(s.d, s.x, s.dt, s.A, s.Bm, s.Cm, s.Dk, s.z, s.bias, None, s.ckpt, s.dy, s.dstate_out, dx, None, None, None, None, None, None, None, None,
                                      s.ws))
    assert torch.equal(dx, base.g["x"])


@pytest.mark.parametrize("bf16", [False, True])
def test_rows_of_a_batch_that_fills_the_chip_are_the_rows_by_themselves(bf16):
    """60 rows of 16 columns of channels go along their rows at once, a row by itself is cut into segments."""
    B, L, D, N = 60, 75, 1024, 16
    i = scan_inputs(B, L, D, N, 1, bf16, seed=77, ragged=True)
    s = Scan(i, bf16).forward().backward()
    torch.cuda.synchronize()
    whole, sums = s.grads(), {}
    tol, tol32 = 2 * tolerance(L, bf16), 2 * tolerance(L, False)        # (both are off)
    for b in range(B):
        row = {k: v if v is None or k in ("A", "Dk", "bias") else v[b:b + 1] for k, v in i.items()}
        t = Scan(row, bf16).forward().backward()
        torch.cuda.synchronize()
        if i["lengths"][b]:
            assert rel_err(s.y[b].float().cpu(), t.y[0].float().cpu()) <= tol and rel_err(s.state_out[b].cpu(), t.state_out[0].cpu()) <= tol32
        else:
            assert torch.equal(s.y[b], t.y[0]) and torch.equal(s.state_out[b], t.state_out[0])
        for n, g in t.grads().items():
            if n in ("dA", "dDskip", "ddt_bias"):
                sums[n] = sums.get(n, 0) + g.astype(np.float64)
            elif i["lengths"][b]:
                assert rel_err(whole[n][b], g[0]) <= (tol32 if n == "dstate_in" else tol), (n, b)
    for n, g in sums.items():
        assert rel_err(whole[n], g) <= tol32, n


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("N", [9, 11, 12, 17, 20, 24, 33, 40, 48, 65, 70, 96])
def test_states_that_waves_share_in_twelves(N, bf16):
    B, L, D, G = 2, 150, 74, 2
    i = scan_inputs(B, L, D, N, G, bf16, seed=N, ragged=True)
    s = Scan(i, bf16).forward().backward()
    torch.cuda.synchronize()
    y, state = R.scan_fwd(**reference_inputs(i))
    assert rel_err(s.y.float().cpu(), y) <= tolerance(L, bf16) and rel_err(s.state_out.cpu(), state) <= tolerance(L, False)
    ref, got = R.scan_bwd(dy=i["dy"], dstate_out=i["dstate_out"], **reference_inputs(i)), s.grads()
    for n, r in ref.items():
        assert rel_err(got[n], r) <= tolerance(L, bf16 and n in ("dx", "ddt", "dBm", "dCm", "dz")), n
