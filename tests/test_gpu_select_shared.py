"""Selective scan with more than 16 states, which waves share, over rows of several tiles a workgroup; and bounds on long rows that follow how roundings add up."""
import numpy as np
import pytest
import torch

import layer_ref as R
from layer_util import EPS, ROUND16, Scan, host, reference_inputs, rel_err, scan_inputs
from test_gpu_select import tolerance

pytestmark = pytest.mark.gpu
STREAMS = ("dx", "ddt", "dBm", "dCm", "dz")


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L,D,N,G", [
    # two tiles in one segment: rows too short to be cut
    (3, 24, 70, 24, 1), (3, 24, 70, 64, 1), (3, 24, 70, 128, 1), (2, 32, 130, 100, 2),
    # five tiles in one segment: the batch fills the chip (1,560 and 1,600 waves)
    (13, 75, 60, 24, 60), (10, 75, 80, 64, 40), (25, 80, 40, 128, 8), (13, 75, 1980, 24, 30),
    # two and three tiles in each of 47 and 44 segments
    (4, 1500, 24, 24, 12), (4, 1500, 12, 64, 6), (4, 2100, 6, 128, 3)])
def test_several_tiles_a_workgroup(B, L, D, N, G, bf16):
    i = scan_inputs(B, L, D, N, G, bf16, seed=L + D + N, ragged=True)
    s = Scan(i, bf16).forward().backward()
    torch.cuda.synchronize()
    y, state = R.scan_fwd(**reference_inputs(i))
    assert rel_err(host(s.y), y) <= tolerance(L, bf16) and rel_err(host(s.state_out), state) <= tolerance(L, False)
    ref, got = R.scan_bwd(dy=i["dy"], dstate_out=i["dstate_out"], **reference_inputs(i)), s.grads()
    for n, r in ref.items():
        assert rel_err(got[n], r) <= tolerance(L, bf16 and n in STREAMS), n
    # in another workspace, without a checkpoint, and again
    t = Scan(i, bf16, ckpt=False).forward()
    assert torch.equal(t.y, s.y) and torch.equal(t.state_out, s.state_out)
    u = Scan(i, bf16).forward().backward()
    for n, g in s.g.items():
        assert torch.equal(u.g[n], g), n


def _off(got, want):
    """|| got - want || / || want ||"""
    got, want = (np.asarray(v, np.float64) for v in (got, want))
    return float(np.sqrt(((got - want) ** 2).sum() / (want ** 2).sum()))


# A rounding's root mean square is 0.5 x 2^-24 of the value.  A factor exp(delta A) is off by some 1.3 x 2^-24 (its exponential, the update's sum), and a state by
# the root of half the tokens that it remembers times that; steps are spread over their logarithm from 0.001 to 0.1, and with states that count as their squares do,
# delta / A, the mean of 1 / (delta A) is 0.099 / (0.0215 x 0.21) = 22: 1.3 x 11^1/2 = 4.3 x 2^-24 of the outputs' norm.  Four times that is left for what is
# not independent: the rates' own rounding, which is one for all tokens, softplus, the gate.
OUT = 16 * EPS
# Gradients are products of such states with gradients that come the same way, 6 x 2^-24, and the two parts of delta's, A p and x du, take from each other.  A sum
# over n tokens in their order is off by 0.35 n^1/2 x 2^-24 of its own size: 14 for 1,500.  Four times that, too.
GRAD = 64 * EPS


def _coherent(L):
    """What a state (or a gradient that reaches it from behind, and with them a parameter's) held before the call weighs more than what the call adds where steps are small, and its errors do not average out: the exponential's instruction,
    good to 2^-24 near 1, is 0.11 x 2^-24 low in the mean there (over exponents of -0.001 to -0.0003, and 0.02 over -0.1 to -0.03).  A state is L of them off, or as
    many as it remembers, 1,000."""
    return 0.125 * min(L, 1000) * EPS


def _compare_norms(s, L, y, state, ref, bf16):
    off = dict(y=(_off(host(s.y), y), OUT + (ROUND16 if bf16 else 0)), state_out=(_off(host(s.state_out), state), OUT + _coherent(L)))
    got = s.grads()
    off.update({n: (_off(got[n], r), GRAD + (_coherent(L) if n not in STREAMS else ROUND16 if bf16 else 0)) for n, r in ref.items()})
    assert all(a <= b for a, b in off.values()), {n: f"{a / EPS:.1f} of {b / EPS:.0f}" for n, (a, b) in off.items()}


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L,D,N,G", [(16, 500, 60, 16, 60), (2, 1500, 70, 16, 1), (13, 700, 60, 24, 60), (2, 1500, 24, 64, 12)])
def test_how_far_long_rows_are_off(B, L, D, N, G, bf16):
    """Rows in one segment and in many, of up to 16 states and of more."""
    i = scan_inputs(B, L, D, N, G, bf16, seed=L + N)
    s = Scan(i, bf16).forward().backward()
    torch.cuda.synchronize()
    y, state = R.scan_fwd(**reference_inputs(i))
    _compare_norms(s, L, y, state, R.scan_bwd(dy=i["dy"], dstate_out=i["dstate_out"], **reference_inputs(i)), bf16)


def test_parameter_gradients_of_long_rows_in_one_segment():
    """1,024 waves of 1,500 tokens each, one running sum a parameter and row; against the recurrence in 64 bits, all rows at once, and autograd."""
    B, L, D, N, G = 64, 1500, 64, 16, 16
    i = scan_inputs(B, L, D, N, G, False, seed=3)
    s = Scan(i, False).forward().backward()
    v = {n: torch.from_numpy(np.asarray(i[n], np.float64)).cuda().requires_grad_() for n in ("x", "dt", "A", "Bm", "Cm", "Dk", "z", "bias", "state_in")}
    delta = torch.nn.functional.softplus(v["dt"] + v["bias"], threshold=1000)
    Bm, Cm = (v[n].repeat_interleave(D // G, 2) for n in ("Bm", "Cm"))
    S, ys = v["state_in"], []
    for t in range(L):
        S = torch.exp(delta[:, t, :, None] * v["A"]) * S + (delta[:, t] * v["x"][:, t])[..., None] * Bm[:, t]
        ys.append((Cm[:, t] * S).sum(-1))
    y = (torch.stack(ys, 1) + v["Dk"] * v["x"]) * torch.nn.functional.silu(v["z"])
    torch.autograd.backward([y, S], [torch.from_numpy(np.asarray(i[n], np.float64)).cuda() for n in ("dy", "dstate_out")])
    names = dict(dx="x", ddt="dt", dA="A", dBm="Bm", dCm="Cm", dDskip="Dk", dz="z", ddt_bias="bias", dstate_in="state_in")
    _compare_norms(s, L, y.detach().cpu(), S.detach().cpu(), {g: v[n].grad.cpu() for g, n in names.items()}, False)


@pytest.mark.parametrize("B,L,D,N,G", [(2, 1500, 70, 16, 1), (3, 100, 130, 64, 2), (64, 40, 1024, 8, 1), (2, 16, 70, 16, 1), (2, 1, 70, 128, 1)])
def test_a_forward_in_the_scratch_of_serving(B, L, D, N, G):
    """The same bits as in the larger one, and nothing written behind it."""
    from paper_2604_04250_amd import binding as K
    i = scan_inputs(B, L, D, N, G, True, seed=L, ragged=True)
    a, b = (Scan(i, True, ckpt=False) for _ in range(2))
    n = K.cawn_selective_scan_serve_workspace_bytes(b.d)
    guarded = torch.full((n + 4096,), 0xa5, dtype=torch.uint8, device="cuda")
    b.ws = guarded[:n]
    a.forward()
    b.forward()
    torch.cuda.synchronize()
    assert torch.equal(a.y, b.y) and torch.equal(a.state_out, b.state_out)
    assert bool((guarded[n:] == 0xa5).all())
