"""The selective scan, the short convolution and the norm at sizes whose launches go round: more work than the workgroups of one take at once."""
import pytest
import torch

import layer_ref as R
from layer_util import DEV, EPS, ROUND16, Scan, reference_inputs, rel_err, scan_inputs, scratch
from paper_2604_04250_amd import binding as K

pytestmark = pytest.mark.gpu


def test_parameter_sums_over_more_columns_than_a_launch_counts_threads_for():
    """Column sums of 5 x 33,554,435 columns: 5.2 million workgroups of 1,024 threads would be more than 2^32.  One token: each gradient is a product."""
    C, k = (1 << 25) + 3, 4
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, dy, state = (torch.randn(s, generator=gen, device=DEV) for s in ((1, 1, C), (1, 1, C), (1, k - 1, C)))
    w = torch.randn((C, k), generator=gen, device=DEV)
    d = K.make_conv_desc(1, 1, C, k)
    dw, db = torch.full_like(w, float("nan")), torch.full((C,), float("nan"), device=DEV)
    K.check(K.cawn_causal_conv_bwd(d, x, w, None, None, state, dy, None, None, dw, db, None, scratch(K.cawn_causal_conv_workspace_bytes(d))))
    assert torch.equal(db, dy[0, 0])
    for i in range(k):
        assert torch.equal(dw[:, i], dy[0, 0] * (state[0, i] if i < k - 1 else x[0, 0])), i
    K.check(K.cawn_causal_conv_bwd(K.make_conv_desc(0, 1, C, k), x, w, None, None, state, dy, None, None, dw, db, None, None))        # sums over nothing
    assert not bool(dw.any()) and not bool(db.any())


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L,D,N,G,ragged", [
    (3, 720, 500, 8, 500, True),            # 67,500 tiles of B and C, 4,219 workgroups of their gradients: both go round
    (1, 18, 1 << 18, 2, 4, False),          # 1,572,864 columns of parameter sums
])
def test_scan_whose_launches_go_round(B, L, D, N, G, ragged, bf16):
    i = scan_inputs(B, L, D, N, G, bf16, seed=D, ragged=ragged)
    s = Scan(i, bf16).forward().backward()
    torch.cuda.synchronize()
    # as in the scan's own tests: 256 tokens of memory at most, four roundings a token
    tol = 4 * EPS * (16 + 4 * min(L, 256))
    y, state = R.scan_fwd(**reference_inputs(i))
    assert rel_err(s.y.float().cpu(), y) <= tol + (ROUND16 if bf16 else 0) and rel_err(s.state_out.cpu(), state) <= tol
    ref, got = R.scan_bwd(dy=i["dy"], dstate_out=i["dstate_out"], **reference_inputs(i)), s.grads()
    for n, r in ref.items():
        assert rel_err(got[n], r) <= tol + (ROUND16 if bf16 and n in ("dx", "ddt", "dBm", "dCm", "dz") else 0), n


def test_state_gradients_in_place_of_more_rows_than_a_launch_takes_at_once():
    """18 million threads on 16.8 million; one token of two taps: the state's gradient is that token's share of the older tap, or, of a row without it, what was there."""
    B, C = 6000003, 3
    gen = torch.Generator(device=DEV).manual_seed(2)
    x, dy, state, dstate = (torch.randn((B, 1, C), generator=gen, device=DEV) for _ in range(4))
    w = torch.randn((C, 2), generator=gen, device=DEV)
    lengths = (torch.arange(B, device=DEV) % 3 > 0).int()
    there = lengths.bool()[:, None, None]
    want, wx = torch.where(there, w[:, 0] * dy, dstate), torch.where(there, w[:, 1] * dy + dstate, 0)
    d, dx = K.make_conv_desc(B, 1, C, 2), torch.empty_like(x)
    K.check(K.cawn_causal_conv_bwd(d, x, w, None, lengths, state, dy, dstate, dx, None, None, dstate, None))
    assert torch.equal(dstate, want)
    assert float((dx - wx).abs().max()) <= 2 * 2.0 ** -24 * float(wx.abs().max())        # (a product and a sum, rounded once or twice)
