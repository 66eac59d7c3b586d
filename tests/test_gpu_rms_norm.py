"""Root-mean-square norm joined with the residual addition, its output in 8 bits among them, against 64 bits through the C ABI."""
import numpy as np
import pytest
import torch

import layer_ref as R
from layer_util import DEV, EPS, ROUND16, dev, host, like, rel_err, rng, rounded, scratch, strided, untouched
from paper_2604_04250_amd import binding as K

pytestmark = pytest.mark.gpu

# the mean of squares has a relative error of 2^-24 times the length of its longest chain of sums (8 x 32 values a thread, and the levels of the join), a
# half of it counts, and a few roundings more; gradients subtract a projection of the same size
TOL = EPS * 200
TOL16 = ROUND16 + TOL
TOLSUM = 2e-5
E4M3 = torch.float8_e4m3fn


class Rms:
    def __init__(self, rows, C, bf16, res_bf16, seed, block=0, extra=(0, 0, 0), offset=0, residual=True, weight=True, accumulate=0, scale=1.0):
        r = rng(seed)
        X, Rt = (torch.bfloat16 if b else torch.float32 for b in (bf16, res_bf16))
        ex, er, ey = self.extra = extra
        self.bf16, self.res_bf16, self.rows, self.C = bf16, res_bf16, rows, C
        self.x = strided(scale * r.standard_normal((rows, C)), X, ex, offset)
        self.res = strided(3 * scale * r.standard_normal((rows, C)), Rt, er, offset) if residual else None
        self.w = dev(1 + 0.2 * r.standard_normal(C)) if weight else None
        self.dy, self.dh = strided(r.standard_normal((rows, C)), X, ey, offset), strided(r.standard_normal((rows, C)), Rt, er, offset)
        self.d = K.make_rms_desc(rows, C, bf16=int(bf16), residual_bf16=int(res_bf16), block=block, accumulate_param_grads=accumulate, x_stride=C + ex if ex else 0,
                                 residual_stride=C + er if er else 0, y_stride=C + ey if ey else 0)
        self.block, self.nb = block, -(-C // block) if block else 1
        self.h, self.y = like(self.dh, er), like(self.dy, ey)
        self.q = torch.full((rows * (C + ey) + offset,), 0x55, dtype=torch.uint8, device=DEV)
        self.qv = self.q[offset:].view(rows, C + ey)[:, :C]
        self.scales, self.rstd = torch.full((rows, self.nb), float("nan"), device=DEV), torch.full((rows,), float("nan"), device=DEV)
        self.ws = scratch(K.cawn_rms_norm_add_workspace_bytes(self.d))

    def forward(self, y=True, q=False, h=True, rstd=True):
        K.check(K.cawn_rms_norm_add_fwd(self.d, self.x, self.res, self.w, self.h if h else None, self.y if y else None, self.qv if q else None, self.scales if q else None,
                                        self.rstd if rstd else None))
        return self

    def backward(self, want=("x", "res", "w"), dh=True, fill=float("nan")):
        self.g = dict(x=like(self.x, self.extra[0]), res=like(self.dh, self.extra[1]), w=torch.full((self.C,), fill, device=DEV))
        g = {n: v if n in want else None for n, v in self.g.items()}
        K.check(K.cawn_rms_norm_add_bwd(self.d, self.h, self.w, self.rstd, self.dy, self.dh if dh else None, g["x"], g["res"], g["w"], self.ws))
        return self

    def held(self):
        """h as it should be kept."""
        s = host(self.x) + (0 if self.res is None else host(self.res))      # (fp32, one rounding)
        return rounded(s, self.res_bf16)


SHAPES = [(1, 1), (4, 768), (3, 16), (1021, 97), (17, 1001), (5, 2048), (300, 1536), (3, 1544), (2, 4096), (3, 5000), (2, 8192), (2, 16384), (2, 16392), (2, 32768), (1, 8191), (2, 20001),
          (70, 24)]


@pytest.mark.parametrize("bf16,res_bf16", [(False, False), (True, False), (True, True), (False, True)])
@pytest.mark.parametrize("rows,C", SHAPES)
def test_forward_and_backward(rows, C, bf16, res_bf16):
    s = Rms(rows, C, bf16, res_bf16, seed=rows + C).forward().backward()
    torch.cuda.synchronize()
    h = s.held()
    assert np.array_equal(host(s.h), h)
    y, r = R.rms_fwd(h, host(s.w))
    assert rel_err(host(s.y), y) <= (TOL16 if bf16 else TOL) and rel_err(host(s.rstd), r) <= TOL
    d, dw = R.rms_bwd(h, host(s.dy), host(s.w), host(s.dh))
    assert rel_err(host(s.g["x"]), d) <= (TOL16 if bf16 else TOL) and rel_err(host(s.g["res"]), d) <= (TOL16 if res_bf16 else TOL)
    assert rel_err(host(s.g["w"]), dw) <= TOLSUM


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("C,extra,offset", [(768, (8, 16, 32), 0), (768, (1, 2, 3), 0), (768, (0, 0, 0), 1), (100, (4, 0, 4), 0), (9000, (8, 8, 8), 3)])
def test_strides_and_alignment(C, extra, offset, bf16):
    s = Rms(7, C, bf16, bf16, seed=C, block=32, extra=extra, offset=offset).forward(q=True).backward()
    torch.cuda.synchronize()
    h = s.held()
    assert np.array_equal(host(s.h), h)
    assert rel_err(host(s.y), R.rms_fwd(h, host(s.w))[0]) <= (TOL16 if bf16 else TOL)
    d, dw = R.rms_bwd(h, host(s.dy), host(s.w), host(s.dh))
    assert rel_err(host(s.g["x"]), d) <= (TOL16 if bf16 else TOL) and rel_err(host(s.g["w"]), dw) <= TOLSUM
    ex, er, ey = extra
    assert untouched(s.y, ey) and untouched(s.h, er) and untouched(s.g["x"], ex) and untouched(s.g["res"], er)
    if ey:
        assert bool((s.q[offset:].view(7, C + ey)[:, C:] == 0x55).all())
    _check_q(s, h)


def _check_q(s, h):
    """The scale is that of the block's largest value; a value stands at the e4m3 value next to its quotient: 2^-4 of it off at most (below 2^-6, where steps
    are even, 2^-10), and 2^-24 times what the norm's own roundings are."""
    y = R.rms_fwd(h, host(s.w))[0]
    most, at = R.blocks_of(y, s.block)
    scales = host(s.scales).astype(np.float64)
    assert rel_err(scales, most / 448) <= TOL
    v = s.qv.contiguous().view(E4M3).float().cpu().numpy().astype(np.float64)
    want = y / np.where(scales == 0, 1, scales)[:, at]
    off = np.abs(v - want)
    assert np.all(off <= np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10) * (1 + 16 * TOL) + TOL * np.abs(want))
    assert np.abs(v).max() <= 448


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,C,block", [(4, 768, 0), (4, 768, 128), (33, 4096, 128), (5, 100, 16), (3, 97, 32), (2, 1001, 128), (3, 8192, 32), (2, 16384, 0), (2, 20000, 128), (2, 20000, 0),
                                          (2, 32768, 16), (9, 48, 48), (9, 96, 48), (1000, 16, 16), (6, 768, 1024), (2, 9001, 64), (2, 9001, 0)])
def test_eight_bits(rows, C, block, bf16):
    s = Rms(rows, C, bf16, bf16, seed=C + block, block=block).forward(y=False, q=True, h=False, rstd=False)
    torch.cuda.synchronize()
    assert bool(torch.isnan(s.h).all()) and bool(torch.isnan(s.rstd).all())
    _check_q(s, s.held())
    t = Rms(rows, C, bf16, bf16, seed=C + block, block=block).forward(y=True, q=True)
    assert torch.equal(s.q, t.q) and torch.equal(s.scales, t.scales)


@pytest.mark.parametrize("C,block", [(64, 0), (64, 16), (97, 16), (4096, 128), (20000, 128), (20000, 0)])
def test_eight_bits_of_zeros_infinities_and_nan(C, block):
    s = Rms(4, C, False, False, seed=3, block=block, residual=False, weight=False)
    s.x[0] = 0.0                    # a row of zeros: scale 0, zeros
    s.x[1, :16] = 0.0               # a block of zeros where 16 channels share a scale
    s.x[2, 5] = float("nan")        # the norm's sum is NaN, and with it the whole row
    s.x[3] *= 1e-42 / s.x[3].abs().max()
    s.forward(y=True, q=True)
    torch.cuda.synchronize()
    v = s.qv.contiguous().view(E4M3).float()
    assert bool((s.scales[0] == 0).all()) and bool((v[0] == 0).all())
    assert bool((v[1, :16] == 0).all()) and bool((v[1, 16:].abs() <= 448).all())
    assert bool(torch.isnan(s.scales[2]).all()) and bool(torch.isnan(v[2]).all()) and bool(torch.isnan(s.y[2]).all())
    assert bool((s.scales[3] == 0).all()) and bool((v[3] == 0).all())       # below 448 x 2^-126


def test_without_residual_weight_and_what_is_not_asked_for():
    s = Rms(9, 200, True, False, seed=4, residual=False, weight=False).forward()
    assert torch.equal(s.h, s.x.float())
    assert rel_err(host(s.y), R.rms_fwd(host(s.x))[0]) <= TOL16
    s.backward(dh=False)
    d, dw = R.rms_bwd(host(s.x), host(s.dy))
    assert rel_err(host(s.g["res"]), d) <= TOL and rel_err(host(s.g["w"]), dw) <= TOLSUM
    all_ = s.g
    for n in all_:
        one = s.backward(want=(n,), dh=False).g
        assert torch.equal(one[n], all_[n])
        for m in one:
            assert m == n or bool(torch.isnan(one[m]).all())
    t = Rms(9, 200, True, False, seed=4, residual=False, weight=False, accumulate=1).forward().backward(dh=False, fill=0.5)
    assert torch.equal(t.g["w"], 0.5 + all_["w"])


@pytest.mark.parametrize("C", [96, 768, 4096, 20000])
def test_in_place(C):
    """The residual stream where it was, the output where x was; gradients where those from above were."""
    s = Rms(6, C, True, True, seed=5).forward().backward()
    t = Rms(6, C, True, True, seed=5)
    K.check(K.cawn_rms_norm_add_fwd(t.d, t.x, t.res, t.w, t.res, t.x, None, None, t.rstd))
    assert torch.equal(t.res, s.h) and torch.equal(t.x, s.y)
    dw = torch.empty(C, device=DEV)
    K.check(K.cawn_rms_norm_add_bwd(t.d, t.res, t.w, t.rstd, t.dy, t.dh, t.dy, t.dh, dw, t.ws))
    assert torch.equal(t.dy, s.g["x"]) and torch.equal(t.dh, s.g["res"]) and torch.equal(dw, s.g["w"])
    u = Rms(6, C, True, True, seed=5)
    K.check(K.cawn_rms_norm_add_fwd(u.d, u.x, u.res, u.w, u.x, None, u.qv, u.scales, u.rstd))
    assert torch.equal(u.x, s.h)


def test_no_rows():
    s = Rms(3, 40, False, False, seed=6)
    d = K.make_rms_desc(0, 40)
    dw = torch.full((40,), 3.0, device=DEV)
    K.check(K.cawn_rms_norm_add_fwd(d, s.x, s.res, s.w, s.h, s.y, None, None, None))
    K.check(K.cawn_rms_norm_add_bwd(d, s.h, s.w, s.rstd, s.dy, s.dh, s.h, s.h, dw, s.ws))
    assert bool(torch.isnan(s.h).all()) and bool(torch.isnan(s.y).all()) and bool((dw == 0).all())


def test_many_rows_of_few_channels_and_the_same_bits_again():
    a, b = (Rms(100003, 24, False, False, seed=7).forward().backward() for _ in range(2))
    for n in a.g:
        assert torch.equal(a.g[n], b.g[n])
    d, dw = R.rms_bwd(a.held(), host(a.dy), host(a.w), host(a.dh))
    assert rel_err(host(a.g["x"]), d) <= TOL and rel_err(host(a.g["w"]), dw) <= 4 * TOLSUM        # (a column of 100,003 terms)


def test_rows_far_apart():
    """Rows more than 2^31 elements from each other."""
    C, far = 768, (1 << 31) + 768
    a = Rms(2, C, True, True, seed=8).forward().backward()
    new = lambda: torch.empty(far + C, device=DEV, dtype=torch.bfloat16).as_strided((2, C), (far, 1))  # noqa: E731
    x, h, y = new(), new(), new()
    x.copy_(a.x)
    d = K.make_rms_desc(2, C, bf16=1, residual_bf16=1, x_stride=far, residual_stride=far, y_stride=far)
    h.copy_(a.res)
    rstd = torch.empty(2, device=DEV)
    K.check(K.cawn_rms_norm_add_fwd(d, x, h, a.w, h, y, None, None, rstd))
    assert torch.equal(h, a.h) and torch.equal(y, a.y)
    y.copy_(a.dy)
    dw = torch.empty(C, device=DEV)
    K.check(K.cawn_rms_norm_add_bwd(d, h, a.w, rstd, y, None, x, None, dw, a.ws))
    b = Rms(2, C, True, True, seed=8).forward().backward(dh=False)
    assert torch.equal(x, b.g["x"]) and torch.equal(dw, b.g["w"])


@pytest.mark.parametrize("bf16,res_bf16", [(False, False), (True, False), (True, True), (False, True)])
@pytest.mark.parametrize("C", [3, 7, 13, 97, 1001, 1541, 4093, 8190, 9001, 16385, 20001])
def test_in_place_at_widths_that_end_inside_a_unit(C, bf16, res_bf16):
    """The last channels of a row are read together with some that stand before them, which another thread replaces."""
    s = Rms(37, C, bf16, res_bf16, seed=9).forward().backward()
    t = Rms(37, C, bf16, res_bf16, seed=9)
    K.check(K.cawn_rms_norm_add_fwd(t.d, t.x, t.res, t.w, t.res, t.x, None, None, t.rstd))
    assert torch.equal(t.res, s.h) and torch.equal(t.x, s.y) and torch.equal(t.rstd, s.rstd)
    dw = torch.empty(C, device=DEV)
    K.check(K.cawn_rms_norm_add_bwd(t.d, t.res, t.w, t.rstd, t.dy, t.dh, t.dy, t.dh, dw, t.ws))
    assert torch.equal(t.dy, s.g["x"]) and torch.equal(t.dh, s.g["res"]) and torch.equal(dw, s.g["w"])


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("block", [0, 16, 32])
def test_every_end_of_a_row(block, bf16):
    """Widths one after the other: units of all lengths at the end, blocks of one channel and of sixteen."""
    for C in [*range(1, 50), *range(1530, 1546)]:
        s = Rms(5, C, bf16, bf16, seed=C, block=block, extra=(0, 0, 3), offset=1).forward(q=True).backward()
        torch.cuda.synchronize()
        h = s.held()
        assert np.array_equal(host(s.h), h)
        assert rel_err(host(s.y), R.rms_fwd(h, host(s.w))[0]) <= (TOL16 if bf16 else TOL)
        d, dw = R.rms_bwd(h, host(s.dy), host(s.w), host(s.dh))
        assert rel_err(host(s.g["x"]), d) <= (TOL16 if bf16 else TOL) and rel_err(host(s.g["w"]), dw) <= TOLSUM
        assert untouched(s.y, 3) and bool((s.q[1:].view(5, C + 3)[:, C:] == 0x55).all())
        _check_q(s, h)


@pytest.mark.parametrize("C", [21, 1001, 20001])
def test_an_infinite_weight_stays_in_its_channel(C):
    s = Rms(3, C, False, False, seed=11, block=16)
    s.w[C - 6] = float("inf")       # read by the thread of the last channels too
    s.forward(q=True)
    t = Rms(3, C, False, False, seed=11, block=16).forward(q=True)
    torch.cuda.synchronize()
    there = torch.arange(C, device=DEV) != C - 6
    assert bool(torch.isinf(s.y[:, C - 6]).all()) and torch.equal(s.y[:, there], t.y[:, there])
    blocks = torch.arange(s.nb, device=DEV) != (C - 6) // 16
    assert torch.equal(s.scales[:, blocks], t.scales[:, blocks]) and bool(torch.isinf(s.scales[:, (C - 6) // 16]).all())
