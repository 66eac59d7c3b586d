"""Decoding steps of the gated delta rule as a server makes them: one token, some slots without a request, the state in place."""
import pytest
import torch

from gpu_util import rel_err
from paper_2604_04250_amd import binding as K
from test_gpu_delta import TOL, TOL16, desc, fwd, host, make, num, ref_fwd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L,H,Hk,Kd,V", [(9, 1, 4, 2, 64, 64), (3, 1, 2, 1, 128, 40), (40, 1, 32, 32, 128, 128), (5, 7, 3, 3, 24, 65)])
def test_steps_in_place_with_unused_slots(B, L, H, Hk, Kd, V, bf16):
    lengths = [L if b % 3 != 1 else 0 for b in range(B)]
    x = make(B, L, H, Hk, Kd, V, bf16, 1, B + V, lengths)
    d = desc(x, 1)
    ref_o, ref_s = ref_fwd(host(x), 1)
    x["state_in"][1::3, ..., ::5] = float("nan")            # what a slot holds that nobody uses
    o, so, _ = fwd(x, d, ckpt=False)
    state, o_ = x["state_in"].clone(), torch.full_like(x["v"], float("nan"))
    K.check(K.cawn_delta_rule_fwd(d, x["q"], x["k"], x["v"], x["decay"], x["beta"], x["lengths"], state, o_, state, None, None))
    none = torch.full_like(x["v"], float("nan"))
    K.check(K.cawn_delta_rule_fwd(d, x["q"], x["k"], x["v"], x["decay"], x["beta"], x["lengths"], x["state_in"], none, None, None, None))
    torch.cuda.synchronize()
    assert torch.equal(o, o_) and torch.equal(o, none) and torch.equal(so.view(torch.int32), state.view(torch.int32))
    assert torch.equal(state.view(torch.int32)[1::3], x["state_in"].view(torch.int32)[1::3]) and not o[1::3].any()
    used = [b for b in range(B) if lengths[b]]
    assert rel_err(num(o)[used], ref_o[used]) <= (TOL16 if bf16 else TOL)
    assert rel_err(num(state)[used], ref_s[used]) <= TOL
