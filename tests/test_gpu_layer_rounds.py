"""The norm and the short convolution with more rows than their workgroups take at once, so that each goes on to another."""
import numpy as np
import pytest
import torch

import layer_ref as R
from layer_util import DEV, dev, host, rel_err, rng, rounded, scratch
from paper_2604_04250_amd import binding as K
from test_gpu_causal_conv import TOL as CONV_TOL
from test_gpu_causal_conv import TOL16 as CONV_TOL16
from test_gpu_rms_norm import E4M3, TOL, TOL16, TOLSUM, Rms, _check_q

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16,res_bf16", [(False, False), (True, False), (True, True), (False, True)])
@pytest.mark.parametrize("rows,C", [(1600, 1537), (1600, 2048), (800, 9001)])
def test_norm_backward_of_more_rows_than_workgroups(rows, C, bf16, res_bf16):
    """Rows that are a workgroup's: 768 take two rounds and three."""
    _norm(rows, C, bf16, res_bf16)


@pytest.mark.parametrize("bf16,res_bf16", [(False, False), (True, False), (True, True)])
@pytest.mark.parametrize("rows,C", [(1600, 16392), (800, 20001)])
def test_norm_backward_of_more_rows_than_workgroups_that_no_registers_hold(rows, C, bf16, res_bf16):
    """The sums of dweight go on from what the row before left of them in the workspace."""
    _norm(rows, C, bf16, res_bf16)


def _norm(rows, C, bf16, res_bf16):
    s = Rms(rows, C, bf16, res_bf16, seed=rows + C).forward().backward()
    torch.cuda.synchronize()
    h = host(s.h)
    d, dw = R.rms_bwd(h, host(s.dy), host(s.w), host(s.dh))
    assert rel_err(host(s.g["x"]), d) <= (TOL16 if bf16 else TOL) and rel_err(host(s.g["res"]), d) <= (TOL16 if res_bf16 else TOL)
    assert rel_err(host(s.g["w"]), dw) <= TOLSUM
    alone = s.g["w"].clone()
    assert torch.equal(s.backward(want=("w",)).g["w"], alone)


@pytest.mark.parametrize("rows,C,block", [(16500, 784, 48), (65600, 256, 48), (131300, 128, 96)])
def test_maxima_of_blocks_by_way_of_lds_row_after_row(rows, C, block):
    """Blocks whose lanes are no power of two: 16,384 workgroups of one, four and eight rows each."""
    s = Rms(rows, C, False, False, seed=C, block=block, residual=False).forward(q=True, h=False)
    torch.cuda.synchronize()
    _check_q(s, host(s.x))


@pytest.mark.parametrize("block", [0, 48])
def test_norm_forward_of_long_rows_row_after_row(block):
    """16,400 rows beyond what registers hold on 16,384 workgroups; the first and last of them against 64 bits."""
    rows, C = 16400, 16392
    gen = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn((rows, C), generator=gen, device=DEV, dtype=torch.bfloat16)
    x[-16:] *= 0.25             # smaller than what the workgroup's first row left
    w = 1 + 0.2 * torch.randn(C, generator=gen, device=DEV)
    d = K.make_rms_desc(rows, C, bf16=1, residual_bf16=1, block=block)
    y, q, scales = torch.empty_like(x), torch.empty((rows, C), dtype=torch.uint8, device=DEV), torch.empty((rows, -(-C // block) if block else 1), device=DEV)
    K.check(K.cawn_rms_norm_add_fwd(d, x, None, w, None, y, q, scales, None))
    torch.cuda.synchronize()
    part = Rms.__new__(Rms)
    for some in (slice(0, 16), slice(rows - 16, rows)):
        h = host(x[some])
        part.w, part.block, part.scales, part.qv = w, block, scales[some], q[some]
        assert rel_err(host(y[some]), R.rms_fwd(h, host(w))[0]) <= TOL16
        _check_q(part, h)
    assert bool(torch.isfinite(q.view(E4M3)[:: 1024].float()).all())


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L,C,k", [(600000, 3, 4, 3), (20000, 1, 128, 4), (21000, 2, 130, 2)])
def test_convolution_backward_of_more_runs_than_workgroups_take_at_once(B, L, C, k, bf16):
    """2,048 workgroups of 256 and of 8 runs each go on to other rows; the sums of dw and dbias go with them."""
    r = rng(B)
    x, dy, state = (rounded(r.standard_normal(s), bf16) for s in ((B, L, C), (B, L, C), (B, k - 1, C)))
    w, bias = (r.standard_normal((C, k)) / np.sqrt(k)).astype(np.float32), (0.1 * r.standard_normal(C)).astype(np.float32)
    lengths = r.integers(0, L + 1, B).astype(np.int32)

    def reference(rows):
        line = np.concatenate([state[rows], x[rows]], 1).astype(np.float64)
        z = sum(w[:, i].astype(np.float64) * line[:, i:i + L] for i in range(k)) + bias
        dz = dy[rows] * R.silu_slope(z) * (np.arange(L) < lengths[rows][:, None])[..., None]
        dline = np.zeros_like(line)
        for i in range(k):
            dline[:, i:i + L] += dz * w[:, i]
        return dict(dx=dline[:, k - 1:], dw=np.stack([(dz * line[:, i:i + L]).sum((0, 1)) for i in range(k)], 1), dbias=dz.sum((0, 1)), dstate_in=dline[:, :k - 1])

    few = slice(0, 5)           # (all rows at once: the same as one by one)
    for n, v in R.conv_bwd(x[few], w, dy[few], None, bias=bias, act=1, lengths=lengths[few], state_in=state[few]).items():
        assert np.allclose(reference(few)[n], v, rtol=1e-12, atol=1e-12), n
    ref = reference(slice(None))
    dt = torch.bfloat16 if bf16 else torch.float32
    d = K.make_conv_desc(B, L, C, k, act=1, bf16=int(bf16))
    gx, gdy, gw, gb, gs = (dev(a) for a in (x, dy, w, bias, state))
    gx, gdy = gx.to(dt), gdy.to(dt)
    dx, dw, db, ds = (torch.full_like(t, float("nan")) for t in (gx, gw, gb, gs))
    K.check(K.cawn_causal_conv_bwd(d, gx, gw, gb, torch.from_numpy(lengths).to(DEV), gs, gdy, None, dx, dw, db, ds, scratch(K.cawn_causal_conv_workspace_bytes(d))))
    torch.cuda.synchronize()
    assert rel_err(host(dx), ref["dx"]) <= (CONV_TOL16 if bf16 else CONV_TOL) and rel_err(host(ds), ref["dstate_in"]) <= CONV_TOL
    assert rel_err(host(dw), ref["dw"]) <= TOLSUM and rel_err(host(db), ref["dbias"]) <= TOLSUM
