"""Short causal convolution with an activation, forward and backward, against 64 bits through the C ABI."""
import numpy as np
import pytest
import torch

import layer_ref as R
from layer_util import DEV, EPS, ROUND16, dev, host, like, rel_err, rng, rounded, scratch, strided, untouched
from paper_2604_04250_amd import binding as K

pytestmark = pytest.mark.gpu

# a sum of k + 1 terms, and an activation whose exponential is good to 2^-23 and 2^-24 of its exponent (up to 8 here), over a root mean square that may be a
# third of the terms'
TOL = EPS * 64
TOL16 = ROUND16 + TOL
# column sums: a term is of the size of the root of the sum's, so rounding adds up to 2^-24 times a few roots of the rows
TOLSUM = 2e-5


def _inputs(B, L, C, k, bf16, seed, ragged=False, bias=True):
    r = rng(seed)
    i = dict(x=rounded(r.standard_normal((B, L, C)), bf16), w=(r.standard_normal((C, k)) / np.sqrt(k)).astype(np.float32),
             bias=(0.1 * r.standard_normal(C)).astype(np.float32) if bias else None, state_in=rounded(r.standard_normal((B, k - 1, C)), bf16),
             dy=rounded(r.standard_normal((B, L, C)), bf16), dstate_out=r.standard_normal((B, k - 1, C)).astype(np.float32), lengths=None)
    if ragged:
        n = r.integers(0, L + 1, B)
        n[0], n[-1] = L, 0
        n[1:-1][:3] = np.minimum([1, 2, 3], L)[: max(0, B - 2)]
        i["lengths"] = n.astype(np.int32)
    return i


class Conv:
    def __init__(self, i, act, bf16, extra=(0, 0), offset=0, accumulate=0):
        self.i, self.extra = i, extra
        dt = torch.bfloat16 if bf16 else torch.float32
        B, L, C = i["x"].shape
        k = i["w"].shape[1]
        a = {n: i[n].copy() for n in ("x", "dy")}
        if i["lengths"] is not None:
            for b in range(B):
                for v in a.values():
                    v[b, max(0, int(i["lengths"][b])):] = np.nan
        ex, ey = extra
        self.d = K.make_conv_desc(B, L, C, k, act=act, bf16=int(bf16), accumulate_param_grads=accumulate, x_stride_t=C + ex if ex else 0, y_stride_t=C + ey if ey else 0)
        self.x, self.dy = strided(a["x"], dt, ex, offset), strided(a["dy"], dt, ey, offset)
        self.w, self.bias, self.state_in, self.dstate_out = (dev(i[n]) for n in ("w", "bias", "state_in", "dstate_out"))
        self.lengths = None if i["lengths"] is None else torch.from_numpy(i["lengths"]).to(DEV)
        self.y, self.state_out = like(self.x, ey), torch.full((B, k - 1, C), float("nan"), device=DEV)
        self.ws = scratch(K.cawn_causal_conv_workspace_bytes(self.d))

    def forward(self, state_in="own", state_out="own", stream=None):
        K.check(K.cawn_causal_conv_fwd(self.d, self.x, self.w, self.bias, self.lengths, self.state_in if state_in == "own" else state_in, self.y,
                                       self.state_out if state_out == "own" else state_out, stream))
        return self

    def backward(self, want=("x", "w", "bias", "state_in"), state_in="own", dstate="own", fill=float("nan")):
        self.g = dict(x=like(self.x, self.extra[0]), w=torch.full_like(self.w, fill), bias=torch.full((self.x.shape[2],), fill, device=DEV),
                      state_in=torch.full_like(self.state_in, float("nan")))
        if dstate == "in place":
            self.g["state_in"] = self.dstate_out
        g = {n: v if n in want else None for n, v in self.g.items()}
        K.check(K.cawn_causal_conv_bwd(self.d, self.x, self.w, self.bias, self.lengths, self.state_in if state_in == "own" else state_in, self.dy,
                                       None if dstate is None else self.dstate_out, g["x"], g["w"], g["bias"], g["state_in"], self.ws))
        return self


def _compare(c, i, act, bf16, state=True, dstate=True):
    k = dict(bias=i["bias"], act=act, lengths=i["lengths"], state_in=i["state_in"] if state else None)
    y, last, _, _ = R.conv_fwd(i["x"], i["w"], **k)
    ref = R.conv_bwd(i["x"], i["w"], i["dy"], i["dstate_out"] if dstate else None, **k)
    assert rel_err(host(c.y), y) <= (TOL16 if bf16 else TOL)
    assert np.array_equal(host(c.state_out), last.astype(np.float32))
    assert rel_err(host(c.g["x"]), ref["dx"]) <= (TOL16 if bf16 else TOL)
    assert rel_err(host(c.g["w"]), ref["dw"]) <= TOLSUM and rel_err(host(c.g["bias"]), ref["dbias"]) <= TOLSUM
    if c.state_in.numel():
        assert rel_err(host(c.g["state_in"]), ref["dstate_in"]) <= TOL


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L,C,k,act,ragged", [
    (1, 1, 768, 4, 1, False), (5, 1, 64, 4, 1, True), (2, 2, 24, 4, 0, False), (3, 3, 40, 3, 1, True), (6, 5, 8, 4, 1, True), (2, 31, 100, 2, 1, False),
    (2, 32, 33, 4, 1, False), (3, 33, 264, 4, 1, True), (2, 200, 768, 4, 1, False), (1, 1000, 7, 3, 0, False), (4, 65, 520, 1, 1, True), (70, 40, 16, 4, 1, True),
    (1, 3000, 2056, 4, 1, False)])
def test_forward_and_backward(B, L, C, k, act, ragged, bf16):
    i = _inputs(B, L, C, k, bf16, seed=B + L + C, ragged=ragged)
    c = Conv(i, act, bf16).forward().backward()
    torch.cuda.synchronize()
    _compare(c, i, act, bf16)
    if ragged:
        for b, n in enumerate(i["lengths"]):
            assert bool((c.y[b, n:] == 0).all()) and bool((c.g["x"][b, n:] == 0).all())


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("extra,offset", [((8, 16), 0), ((3, 5), 0), ((0, 0), 1)])
def test_strides_and_alignment(extra, offset, bf16):
    i = _inputs(2, 50, 40, 4, bf16, seed=3)
    c = Conv(i, 1, bf16, extra, offset).forward().backward()
    torch.cuda.synchronize()
    _compare(c, i, 1, bf16)
    assert untouched(c.y, extra[1]) and untouched(c.g["x"], extra[0])


def test_without_states_and_bias():
    i = _inputs(2, 40, 24, 4, False, seed=4, bias=False)
    c = Conv(i, 1, False).forward(state_in=None).backward(state_in=None, dstate=None)
    _compare(c, i, 1, False, state=False, dstate=False)
    c.forward(state_in=None, state_out=None)


def test_gradients_one_by_one_added_and_in_place():
    i = _inputs(4, 70, 24, 4, False, seed=5, ragged=True)
    all_ = Conv(i, 1, False).forward().backward().g
    for n, v in all_.items():
        one = Conv(i, 1, False).backward(want=(n,)).g
        assert torch.equal(one[n], v), n
        for m, w in one.items():
            assert m == n or bool(torch.isnan(w).all())
    added = Conv(i, 1, False, accumulate=1).backward(fill=0.5).g
    for n in ("w", "bias"):
        assert torch.equal(added[n], 0.5 + all_[n]), n
    assert torch.equal(Conv(i, 1, False).backward(dstate="in place").g["state_in"], all_["state_in"])


@pytest.mark.parametrize("L", [1, 2, 40])
def test_state_in_place_and_unused_slots(L):
    i = _inputs(4, L, 24, 4, True, seed=6)
    i["lengths"] = np.array([L + 9, 0, -1, 1], np.int32)
    i["state_in"][1, 0, 0] = np.nan
    c = Conv(i, 1, True).forward()
    d = Conv(i, 1, True)
    d.forward(state_in=d.state_in, state_out=d.state_in)
    assert torch.equal(c.y, d.y) and torch.equal(c.state_out.view(torch.int32), d.state_in.view(torch.int32))
    for b in (1, 2):
        assert torch.equal(c.state_out[b].view(torch.int32), c.state_in[b].view(torch.int32))


def test_no_tokens_pass_the_state():
    i = _inputs(2, 0, 24, 4, False, seed=7)
    c = Conv(i, 1, False).forward().backward()
    assert torch.equal(c.state_out, c.state_in) and torch.equal(c.g["state_in"], c.dstate_out)
    assert bool((c.g["w"] == 0).all()) and bool((c.g["bias"] == 0).all())


def test_tokens_one_by_one_are_the_whole_to_the_bit():
    i = _inputs(2, 37, 40, 4, True, seed=8)
    whole = Conv(i, 1, True).forward()
    state, ys = whole.state_in, []
    for t in range(37):
        c = Conv({**i, "x": i["x"][:, t:t + 1], "dy": i["dy"][:, t:t + 1]}, 1, True).forward(state_in=state)
        state = c.state_out
        ys.append(c.y)
    assert torch.equal(torch.cat(ys, 1), whole.y) and torch.equal(state, whole.state_out)


def test_gradients_against_differences():
    """A step of 1/64 along a direction of length one, the forward in fp32: as far off as its square of the third derivative, and 2^-24 of the sums over it."""
    i = _inputs(2, 40, 16, 4, False, seed=9)
    g = Conv(i, 1, False).backward().g
    r = rng(10)

    def value(j):
        c = Conv(j, 1, False).forward()
        return float((c.y.double().cpu().numpy() * i["dy"]).sum() + (c.state_out.double().cpu().numpy() * i["dstate_out"]).sum())

    for n in ("x", "w", "bias", "state_in"):
        v = r.standard_normal(i[n].shape).astype(np.float32)
        v /= np.sqrt((v * v).sum())
        want = (value({**i, n: i[n] + v / 64}) - value({**i, n: i[n] - v / 64})) * 32
        got = float((host(g[n]) * v).sum())
        assert abs(got - want) <= 4e-3 * (float(np.sqrt((host(g[n]) ** 2).mean())) + abs(want)) + 1e-3, n


def test_rows_far_apart():
    """A batch whose rows lie more than 2^31 elements from each other."""
    L, C, far = 70, 64, (1 << 31) + 64
    i = _inputs(2, L, C, 4, True, seed=11)
    base = Conv(i, 1, True).forward().backward()
    c = Conv(i, 1, True)
    new = lambda: torch.empty(far + L * C, device=DEV, dtype=torch.bfloat16).as_strided((2, L, C), (far, C, 1))  # noqa: E731
    c.x, c.y, dx = new(), new(), new()
    c.x.copy_(base.x)
    c.d.x_stride_b = c.d.y_stride_b = far
    c.forward()
    assert torch.equal(c.y, base.y)
    c.y.copy_(base.dy)
    K.check(K.cawn_causal_conv_bwd(c.d, c.x, c.w, c.bias, None, c.state_in, c.y, c.dstate_out, dx, None, None, None, c.ws))
    assert torch.equal(dx, base.g["x"])


def test_captured_and_replayed():
    i, j = (_inputs(3, 70, 40, 4, True, seed=k, ragged=True) for k in (12, 13))
    j["lengths"] = i["lengths"]
    want, c = Conv(j, 1, True).forward().backward(), Conv(i, 1, True).forward().backward()
    new, g = Conv(j, 1, True), c.g
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward()
        K.check(K.cawn_causal_conv_bwd(c.d, c.x, c.w, c.bias, c.lengths, c.state_in, c.dy, c.dstate_out, g["x"], g["w"], g["bias"], g["state_in"], c.ws))
    for n in ("x", "dy", "w", "bias", "state_in", "dstate_out"):
        getattr(c, n).copy_(getattr(new, n))
    for _ in range(3):
        for v in g.values():
            v.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.y, want.y) and torch.equal(c.state_out, want.state_out)
        assert all(torch.equal(g[n], want.g[n]) for n in g)
        torch.ones(1000, device=DEV).sum()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("k", [1, 2, 3, 4])
def test_every_end_of_a_row(k, bf16):
    """Widths one after the other: units of one to four channels at the end, rows of fewer than four."""
    for C in [*range(1, 14), 129, 130, 131]:
        i = _inputs(5, 37, C, k, bf16, seed=C, ragged=True)
        c = Conv(i, 1, bf16, (0, 3), offset=1).forward().backward()
        torch.cuda.synchronize()
        _compare(c, i, 1, bf16)
        assert untouched(c.y, 3)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L,C", [(70, 1, 1027), (9, 40, 769), (33, 2, 258), (5, 0, 7)])
def test_state_in_place_at_widths_that_end_inside_a_unit(B, L, C, bf16):
    """The last channels of a row are read together with some that stand before them, whose state another thread replaces."""
    i = _inputs(B, L, C, 4, bf16, seed=8)
    i["lengths"] = np.asarray([(b * 7) % (L + 2) for b in range(B)], np.int32)
    c, d = (Conv(i, 1, bf16) for _ in range(2))
    c.forward().backward()
    d.forward(state_in=d.state_in, state_out=d.state_in)
    assert torch.equal(c.y, d.y) and torch.equal(c.state_out, d.state_in)
    d.state_in.copy_(c.state_in)
    d.backward(dstate="in place")
    for n, g in c.g.items():
        assert torch.equal(g, d.g[n]), n
