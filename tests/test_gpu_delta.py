"""Gated delta rule against 64 bits through the C ABI: single tokens, short and long calls, both types, shared heads, ragged rows."""
import numpy as np
import pytest
import torch

import ops_ref as R
from gpu_util import DEV, rel_err
from paper_2604_04250_amd import binding as K

pytestmark = pytest.mark.gpu

# fp32: products over up to 128 keys and 64 tokens, each sum within some 100 roundings of 2^-24 of its terms' size; what a row holds of
# earlier tokens shrinks, so errors do not pile up.  bf16 outputs add one rounding to 8 significant bits, 2^-8 at most.
TOL = 2e-5
TOL16 = 2.0 ** -8 + TOL


def make(B, L, H, Hk, Kd, V, bf16, norm, seed, lengths=None, low=1e-3):
    r = np.random.Generator(np.random.PCG64(seed))
    dt = torch.bfloat16 if bf16 else torch.float32
    q, k, v, do = (r.standard_normal(s) for s in ((B, L, Hk, Kd), (B, L, Hk, Kd), (B, L, H, V), (B, L, H, V)))
    if not norm:
        q, k = (t / np.sqrt((t * t).sum(-1, keepdims=True)) for t in (q, k))
    act = lambda a: torch.from_numpy(a.astype(np.float32)).to(DEV).to(dt)  # noqa: E731
    f32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEV)  # noqa: E731
    x = dict(q=act(q), k=act(k), v=act(v), do=act(do), decay=f32(-low ** r.uniform(0, 1, (B, L, H))), beta=f32(r.uniform(0.02, 0.98, (B, L, H))),
             state_in=f32(0.5 * r.standard_normal((B, H, Kd, V))), dstate_out=f32(0.3 * r.standard_normal((B, H, Kd, V))))
    x["lengths"] = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    return x


def host(x):
    return {n: None if t is None else t.cpu().numpy() if t.dtype == torch.int32 else t.double().cpu().numpy() for n, t in x.items()}


def desc(x, norm, scale=0.6, **strides):
    B, L, Hk, Kd = x["q"].shape
    H, V = x["v"].shape[2:]
    return K.make_delta_desc(B, L, H, Kd, V, Hk=Hk, scale=scale, qk_norm=norm, bf16=int(x["q"].dtype == torch.bfloat16), **strides)


def buffers(d):
    return tuple(torch.full((max(256, n(d)),), 0xff, dtype=torch.uint8, device=DEV) for n in (K.cawn_delta_ckpt_bytes, K.cawn_delta_workspace_bytes))


def fwd(x, d, ckpt=True):
    ck, ws = buffers(d)
    o = torch.full_like(x["v"], float("nan"))
    so = torch.full((d.B, d.H, d.K, d.V), float("nan"), device=DEV)
    K.check(K.cawn_delta_rule_fwd(d, x["q"], x["k"], x["v"], x["decay"], x["beta"], x["lengths"], x["state_in"], o, so, ck if ckpt else None, ws))
    torch.cuda.synchronize()
    return o, so, ck


def ref_fwd(h, norm, scale=0.6):
    return R.delta_fwd(h["q"], h["k"], h["v"], h["decay"], h["beta"], scale, norm, 1e-6, h["lengths"], h["state_in"])


def num(t):
    return t.float().cpu().numpy()


SHAPES = [  # B, L, H, Hk, K, V, norm, lengths
    (1, 1, 1, 1, 1, 1, 0, None), (3, 1, 4, 2, 64, 64, 1, None), (5, 1, 12, 12, 64, 64, 1, [1, 0, 1, 1, 0]), (2, 1, 3, 1, 128, 256, 0, None),
    (2, 3, 2, 1, 16, 40, 1, None), (1, 16, 2, 2, 96, 128, 0, None), (2, 17, 2, 2, 64, 64, 1, [17, 3]), (1, 63, 2, 1, 32, 16, 1, None),
    (2, 64, 2, 2, 64, 64, 0, None), (1, 65, 2, 2, 64, 72, 1, None), (3, 150, 4, 2, 64, 128, 1, [150, 0, 65]), (2, 200, 2, 2, 128, 128, 1, None),
    (1, 257, 3, 3, 5, 7, 1, None), (2, 130, 2, 1, 33, 65, 0, [1, 128]), (4, 70, 8, 2, 16, 16, 1, [64, 70, 0, -3]), (1, 1030, 1, 1, 64, 64, 1, None),
    (1, 300, 2, 2, 127, 33, 1, [999])]


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("B,L,H,Hk,Kd,V,norm,lengths", SHAPES)
def test_forward(B, L, H, Hk, Kd, V, norm, lengths, bf16):
    x = make(B, L, H, Hk, Kd, V, bf16, norm, 100 * L + V, lengths)
    h = host(x)
    ref_o, ref_s = ref_fwd(h, norm)
    for ckpt in (False, True):
        o, so, _ = fwd(x, desc(x, norm), ckpt)
        assert rel_err(num(o), ref_o) <= (TOL16 if bf16 else TOL)
        assert rel_err(num(so), ref_s) <= TOL
        if lengths is not None:
            for b, n in enumerate(lengths):
                assert not o[b, max(n, 0):].any()
                if n <= 0:
                    assert torch.equal(so[b], x["state_in"][b])


def test_what_lies_beyond_a_row_is_not_read():
    x = make(3, 140, 2, 1, 64, 64, False, 1, 5, [140, 0, 70])
    clean = fwd(x, desc(x, 1))[:2]
    for n in ("q", "k", "v", "decay", "beta"):
        x[n][1] = float("nan")
        x[n][2, 70:] = float("inf")
    got = fwd(x, desc(x, 1))[:2]
    assert all(torch.equal(a, b) for a, b in zip(clean, got))


@pytest.mark.parametrize("L", [6, 200])
def test_forgetting_completely(L):
    """A decay of minus infinity (or of the type's lowest value) begins anew: what came before cannot be told from nothing."""
    x = make(2, L, 2, 2, 64, 64, False, 1, 6)
    cut = L // 2 + 1
    x["decay"][0, cut] = float("-inf")
    x["decay"][1, cut] = torch.finfo(torch.float32).min
    x["decay"][1, cut + 1] = float("-inf")
    o, so, _ = fwd(x, desc(x, 1))
    h = host(x)
    ref_o, ref_s = ref_fwd(h, 1)
    assert rel_err(num(o), ref_o) <= TOL and rel_err(num(so), ref_s) <= TOL


@pytest.mark.parametrize("L", [5, 130])
def test_beta_of_zero_writes_nothing_and_of_two_reflects(L):
    x = make(2, L, 2, 1, 32, 32, False, 1, 7)
    x["beta"][0] = 0
    x["beta"][1, ::3] = 2
    x["beta"][1, 1] = -0.5
    o, so, _ = fwd(x, desc(x, 1))
    ref_o, ref_s = ref_fwd(host(x), 1)
    assert rel_err(num(o), ref_o) <= TOL and rel_err(num(so), ref_s) <= TOL


def test_keys_all_alike():
    """The triangular system at its worst: every key the same, every beta near one, nothing forgotten."""
    x = make(1, 128, 1, 1, 64, 64, False, 1, 8)
    x["k"][:] = x["k"][:, :1]
    x["beta"][:] = 0.999
    x["decay"][:] = -1e-4
    o, so, _ = fwd(x, desc(x, 1))
    ref_o, ref_s = ref_fwd(host(x), 1)
    assert rel_err(num(o), ref_o) <= TOL and rel_err(num(so), ref_s) <= TOL


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("pad", [0, 3])
def test_rows_of_a_packed_projection(bf16, pad):
    """q, k and v as column blocks of one tensor, o with rows of its own length; nothing between them is written."""
    B, L, H, Hk, Kd, V = 2, 90, 4, 2, 24, 20
    x = make(B, L, H, Hk, Kd, V, bf16, 1, 9)
    ref_o, ref_s = ref_fwd(host(x), 1)
    wq, wv = Hk * Kd, H * V
    row = 2 * wq + wv + pad
    packed = torch.full((B, L, row), float("nan"), device=DEV, dtype=x["q"].dtype)
    for at, n in ((0, "q"), (wq, "k"), (2 * wq, "v")):
        packed[..., at:at + x[n][0, 0].numel()] = x[n].reshape(B, L, -1)
    o = torch.full((B, L + 1, wv + 2 * pad), float("nan"), device=DEV, dtype=x["q"].dtype)
    d = K.make_delta_desc(B, L, H, Kd, V, Hk=Hk, scale=0.6, qk_norm=1, bf16=int(bf16), qk_stride_t=row, v_stride_t=row,
                          o_stride_b=(L + 1) * (wv + 2 * pad), o_stride_t=wv + 2 * pad)
    so = torch.empty(B, H, Kd, V, device=DEV)
    ck, ws = buffers(d)
    K.check(K.cawn_delta_rule_fwd(d, packed, packed[..., wq:], packed[..., 2 * wq:], x["decay"], x["beta"], None, x["state_in"], o, so, None, ws))
    torch.cuda.synchronize()
    assert rel_err(num(o[:, :L, :wv]).reshape(ref_o.shape), ref_o) <= (TOL16 if bf16 else TOL)
    assert rel_err(num(so), ref_s) <= TOL
    assert bool(torch.isnan(o[:, L:]).all()) and bool(torch.isnan(o[..., wv:]).all())


def test_passing_a_sequence_in_pieces():
    """Chunks of any length with the state carried in place, single tokens among them, agree with one call to rounding."""
    x = make(2, 333, 3, 3, 64, 64, False, 1, 10)
    whole_o, whole_s, _ = fwd(x, desc(x, 1))
    state, at, parts = x["state_in"].clone(), 0, []
    for n in (1, 128, 63, 1, 0, 16, 124):
        piece = {m: (t[:, at:at + n].contiguous() if m in ("q", "k", "v", "decay", "beta") else t) for m, t in x.items()}
        d = K.make_delta_desc(2, n, 3, 64, 64, scale=0.6, qk_norm=1)
        o = torch.empty(2, n, 3, 64, device=DEV)
        K.check(K.cawn_delta_rule_fwd(d, piece["q"], piece["k"], piece["v"], piece["decay"], piece["beta"], None, state, o, state, None, buffers(d)[1]))
        parts.append(o)
        at += n
    torch.cuda.synchronize()
    assert at == 333
    assert rel_err(num(torch.cat(parts, 1)), num(whole_o)) <= TOL and rel_err(num(state), num(whole_s)) <= TOL


def test_no_state_in_and_none_out():
    x = make(2, 100, 2, 2, 64, 64, False, 1, 11)
    x["state_in"] = None
    d = desc(x, 1)
    o = torch.empty_like(x["v"])
    K.check(K.cawn_delta_rule_fwd(d, x["q"], x["k"], x["v"], x["decay"], x["beta"], None, None, o, None, None, buffers(d)[1]))
    torch.cuda.synchronize()
    assert rel_err(num(o), ref_fwd(host(x), 1)[0]) <= TOL


def test_another_stream_than_the_current_one():
    x = make(2, 150, 2, 2, 64, 64, True, 1, 12)
    want = fwd(x, desc(x, 1))[:2]
    s = torch.cuda.Stream()
    d = desc(x, 1)
    ck, ws = buffers(d)
    o, so = torch.empty_like(x["v"]), torch.empty_like(x["state_in"])
    torch.cuda.synchronize()
    K.check(K.cawn_delta_rule_fwd(d, x["q"], x["k"], x["v"], x["decay"], x["beta"], None, x["state_in"], o, so, ck, ws, stream=s))
    s.synchronize()
    assert torch.equal(o, want[0]) and torch.equal(so, want[1])
