"""Gated delta rule on calls long enough to be cut into segments (six chunks of 64 tokens and more): states in place, rows that end before the
last segment, every width of a key, against 64 bits and against the same call laid out otherwise."""
import pytest
import torch

from gpu_util import rel_err
from paper_2604_04250_amd import binding as K
from test_gpu_delta import TOL, TOL16, buffers, desc, fwd, host, make, num, ref_fwd
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


@pytest.mark.parametrize("Kd,V", [(64, 64), (128, 40), (20, 24)])
def test_the_state_of_an_unused_slot_is_passed_through_bit_by_bit(Kd, V):
    """Whatever it holds, and the rows beside it are what they are without it."""
    x = make(3, 450, 2, 1, Kd, V, False, 1, 51, [450, 0, 65])
    d = desc(x, 1)
    clean_o, clean_s, _ = fwd(x, d)
    clean = run_bwd(x, d)
    for t in (x["state_in"], x["dstate_out"]):
        flat = t[1].view(-1)
        flat[::7], flat[1::7], flat[2::7], flat[3::7] = float("nan"), float("inf"), -3.3e38, 1.2345678e-36
        flat[4::7], flat[5::7] = 1e-45, -0.0
    for o, so in (fwd(x, d)[:2], _in_place(x, d, True)[:2]):
        assert torch.equal(so[1].view(torch.int32), x["state_in"][1].view(torch.int32))
        assert not o[1].any() and all(torch.equal(o[b], clean_o[b]) and torch.equal(so[b], clean_s[b]) for b in (0, 2))
    got = run_bwd(x, d)
    assert torch.equal(got["dstate_in"][1].view(torch.int32), x["dstate_out"][1].view(torch.int32))
    for n in NAMES:
        assert all(torch.equal(got[n][b], clean[n][b]) for b in (0, 2)), n
        assert n == "dstate_in" or not got[n][1].any(), n


# six chunks and more: MODE 1 of both passes and the join at every padded width of a key (32, 64, 128), on value tiles that fill eight waves, leave half
# of them empty or end inside one; heads that share keys; rows without tokens, of one, ending in the first segment, inside a chunk and on its edge
SEGMENTED = [(1, 400, 2, 2, 16, 40, 0, None), (2, 390, 4, 2, 33, 256, 1, [390, 0]), (3, 450, 2, 1, 128, 40, 1, [449, 0, 65]), (2, 520, 3, 3, 128, 256, 0, [1, 512]),
             (1, 1100, 2, 1, 127, 72, 1, None), (4, 385, 2, 2, 5, 7, 1, [385, 384, 64, -2]), (2, 700, 6, 2, 64, 128, 1, [700, 130]), (1, 2500, 1, 1, 32, 200, 1, None),
             (2, 640, 2, 1, 96, 16, 0, [640, 321]), (1, 390, 12, 4, 64, 33, 1, [999]), (1, 5000, 1, 1, 24, 64, 1, [4801])]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L,H,Hk,Kd,V,norm,lengths", SEGMENTED)
def test_forward_in_segments(B, L, H, Hk, Kd, V, norm, lengths, bf16):
    x = make(B, L, H, Hk, Kd, V, bf16, norm, 3 * L + V, lengths)
    ref_o, ref_s = ref_fwd(host(x), norm)
    for ckpt in (False, True):
        o, so, _ = fwd(x, desc(x, norm), ckpt)
        assert rel_err(num(o), ref_o) <= (TOL16 if bf16 else TOL)
        assert rel_err(num(so), ref_s) <= TOL
        for b, n in enumerate(lengths or ()):
            assert not o[b, max(n, 0):].any()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L,H,Hk,Kd,V,norm,lengths", SEGMENTED)
def test_gradients_in_segments(B, L, H, Hk, Kd, V, norm, lengths, bf16):
    x = make(B, L, H, Hk, Kd, V, bf16, norm, 5 * L + V, lengths)
    got = run_bwd(x, desc(x, norm))
    check_gradients(got, ref(host(x), norm), bf16)
    for b, n in enumerate(lengths or ()):
        for m in NAMES[:5]:
            assert not got[m][b, max(n, 0):].any(), m


@pytest.mark.parametrize("Kd,V", [(64, 72), (128, 40)])
def test_what_lies_beyond_a_row_is_not_read_in_segments(Kd, V):
    x = make(3, 450, 2, 1, Kd, V, False, 1, 61, [449, 0, 70])
    clean_o, clean_s, _ = fwd(x, desc(x, 1))
    clean = run_bwd(x, desc(x, 1))
    for n in ("q", "k", "v", "decay", "beta", "do"):
        x[n][0, 449:], x[n][1], x[n][2, 70:] = float("nan"), float("nan"), float("inf")
    o, so, _ = fwd(x, desc(x, 1))
    assert torch.equal(o, clean_o) and torch.equal(so, clean_s)
    got = run_bwd(x, desc(x, 1))
    assert all(torch.equal(got[n], clean[n]) for n in NAMES)


@pytest.mark.parametrize("cut", [300, 384, 449])
def test_forgetting_completely_in_segments(cut):
    """Across a segment's edge, and on it."""
    x = make(1, 500, 2, 2, 64, 64, False, 1, 62)
    x["decay"][0, cut] = float("-inf")
    o, so, _ = fwd(x, desc(x, 1))
    ref_o, ref_s = ref_fwd(host(x), 1)
    assert rel_err(num(o), ref_o) <= TOL and rel_err(num(so), ref_s) <= TOL
    check_gradients(run_bwd(x, desc(x, 1)), ref(host(x), 1), False)


def test_a_long_sequence_passed_in_long_pieces_in_place():
    """Pieces that are cut into segments, the state carried in one buffer from each to the next, single tokens between them."""
    x = make(2, 1800, 3, 3, 64, 64, False, 1, 63)
    ref_o, ref_s = ref_fwd(host(x), 1)
    state, at, parts = x["state_in"].clone(), 0, []
    for n in (449, 1, 640, 16, 694):
        piece = [x[m][:, at:at + n].contiguous() for m in ("q", "k", "v", "decay", "beta")]
        d = K.make_delta_desc(2, n, 3, 64, 64, scale=0.6, qk_norm=1)
        o = torch.empty(2, n, 3, 64, device=x["v"].device)
        K.check(K.cawn_delta_rule_fwd(d, *piece, None, state, o, state, None, buffers(d)[1]))
        parts.append(o)
        at += n
    torch.cuda.synchronize()
    assert at == 1800
    assert rel_err(num(torch.cat(parts, 1)), ref_o) <= TOL and rel_err(num(state), ref_s) <= TOL
