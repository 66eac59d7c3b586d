"""Gated delta rule on calls long enough to be cut into segments (six chunks of 64 tokens and more): states in place, rows that end before the
last segment, every width of a key, against 64 bits and against the same call laid out otherwise."""
import pytest
import torch

from gpu_util import rel_err
from paper_2604_04250_amd import binding as K
from test_gpu_delta import TOL, buffers, desc, fwd, host, make, num, ref_fwd
from test_gpu_delta_bwd import NAMES, ref
from test_gpu_delta_bwd import check as check_gradients
from test_gpu_delta_bwd import run as run_bwd

pytestmark = pytest.mark.gpu


def _in_place(x, d, ckpt):
    """The forward with the state carried in one buffer -> o, state, checkpoint."""
    ck, ws = buffers(d)
    o, state = torch.full_like(x["v"], float("nan")), x["state_in"].clone()
    K.check(K.cawn_delta_rule_fwd(d, x["q"], x["k"], x["v"], x["decay"], x["beta"], x["lengths"], state, o, state, ck if ckpt else None, ws))
    torch.cuda.synchronize()
    return o, state, ck


# the last segments of rows that end early begin and end with the state the first ones made: nothing but their launch orders them
IN_PLACE = [(4, 400, 8, 4, 64, 64, [400, 1, 0, 70]), (2, 1030, 3, 3, 64, 72, None), (3, 450, 2, 1, 128, 40, [449, 64, 65]), (5, 390, 4, 4, 24, 130, [2, 390, 0, 200, 63])]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L,H,Hk,Kd,V,lengths", IN_PLACE)
def test_a_state_in_place_is_a_state_passed_on(B, L, H, Hk, Kd, V, lengths, bf16):
    x = make(B, L, H, Hk, Kd, V, bf16, 1, L + V, lengths)
    d = desc(x, 1)
    ref_s = ref_fwd(host(x), 1)[1]
    for ckpt in (False, True):
        o, so, _ = fwd(x, d, ckpt)
        o_, state, _ = _in_place(x, d, ckpt)
        assert torch.equal(o_, o) and torch.equal(state, so)
        assert rel_err(num(state), ref_s) <= TOL


@pytest.mark.parametrize("B,L,H,Hk,Kd,V,lengths", IN_PLACE)
def test_gradients_behind_a_state_in_place_and_in_place_themselves(B, L, H, Hk, Kd, V, lengths):
    x = make(B, L, H, Hk, Kd, V, False, 1, L + V + 1, lengths)
    d = desc(x, 1)
    apart = run_bwd(x, d)
    check_gradients(apart, ref(host(x), 1), False)
    ck = _in_place(x, d, True)[2]
    ws = buffers(d)[1]
    like = dict(dq=x["q"], dk=x["k"], dv=x["v"], ddecay=x["decay"], dbeta=x["beta"])
    got = {n: torch.full_like(t, float("nan")) for n, t in like.items()} | dict(dstate_in=x["dstate_out"].clone())
    K.check(K.cawn_delta_rule_bwd(d, x["q"], x["k"], x["v"], x["decay"], x["beta"], x["lengths"], ck, x["do"], got["dstate_in"], *[got[n] for n in NAMES], ws))
    torch.cuda.synchronize()
    for n in NAMES:
        assert torch.equal(got[n], apart[n]), n
