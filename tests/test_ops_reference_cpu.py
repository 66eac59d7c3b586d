"""The 64-bit references of the operators beside the scan, and the refusals of their entry points (CPU only, nothing is launched)."""
import ctypes as C

import numpy as np
import pytest

import ops_ref as R
from paper_2604_04250_amd import binding as K


def _delta_inputs(seed, B=2, L=5, H=4, Hk=2, Kd=3, V=2):
    r = np.random.Generator(np.random.PCG64(seed))
    return dict(q=r.standard_normal((B, L, Hk, Kd)), k=r.standard_normal((B, L, Hk, Kd)), v=r.standard_normal((B, L, H, V)),
                decay=-r.uniform(0.01, 1, (B, L, H)), beta=r.uniform(0.1, 0.9, (B, L, H)), state_in=r.standard_normal((B, H, Kd, V)))


def test_delta_rule_is_its_matrix_form():
    """S[t] = a (I - beta k k^T) S[t-1] + beta k v^T, o = scale S^T q, one head at a time."""
    x = _delta_inputs(1)
    o, S = R.delta_fwd(**x, scale=0.7)
    for b in range(2):
        for h in range(4):
            s = x["state_in"][b, h]
            for t in range(5):
                k, be = x["k"][b, t, h // 2], x["beta"][b, t, h]
                s = np.exp(x["decay"][b, t, h]) * (np.eye(3) - be * np.outer(k, k)) @ s + be * np.outer(k, x["v"][b, t, h])
                assert np.allclose(o[b, t, h], 0.7 * s.T @ x["q"][b, t, h // 2], atol=1e-12)
            assert np.allclose(S[b, h], s, atol=1e-12)


@pytest.mark.parametrize("norm,lengths", [(0, None), (1, None), (1, [3, 0]), (0, [1, 5])])
def test_delta_rule_gradients_are_its_differences(norm, lengths):
    x = _delta_inputs(2)
    r = np.random.Generator(np.random.PCG64(3))
    do, dS = r.standard_normal(x["v"].shape), r.standard_normal(x["state_in"].shape)

    def loss(y):
        o, S = R.delta_fwd(**y, scale=0.7, qk_norm=norm, lengths=lengths)
        return (o * do).sum() + (S * dS).sum()

    g = R.delta_bwd(**{n: t for n, t in x.items()}, do=do, dstate_out=dS, scale=0.7, qk_norm=norm, lengths=lengths)
    for name in x:
        way = r.standard_normal(x[name].shape)
        h = 1e-5
        num = (loss({**x, name: x[name] + h * way}) - loss({**x, name: x[name] - h * way})) / (2 * h)
        # truncation h^2 |f'''| and rounding 1e-16 |f| / h are both near 1e-10
        assert abs(num - (g["d" + name] * way).sum()) <= 1e-7 * (1 + abs(num)), name


@pytest.mark.parametrize("kind", [0, 1, 2])
def test_group_norm_gradients_are_its_differences(kind):
    r = np.random.Generator(np.random.PCG64(4))
    x, w, b, dy = r.standard_normal((2, 3, 8)), 1 + 0.2 * r.standard_normal(8), r.standard_normal(8), r.standard_normal((2, 3, 8))
    g = R.norm_bwd(x, w, b, dy, 4, kind)
    for i, name in ((0, "dx"), (1, "dweight"), (2, "dbias")):
        args = [x, w, b]
        way = r.standard_normal(args[i].shape)
        f = lambda s: (R.norm_fwd(*[a + s * way if j == i else a for j, a in enumerate(args)], 4, kind)[0] * dy).sum()  # noqa: E731
        num = (f(1e-5) - f(-1e-5)) / 2e-5
        assert abs(num - (g[name] * way).sum()) <= 1e-7 * (1 + abs(num)), name


def test_philox_words_are_the_published_ones():
    """Known answers of the generator's authors for the zero counter and key."""
    assert R.philox(0, 0) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]


def test_operators_refuse_what_they_cannot_do():
    L_, null, fake = K.lib(), C.c_void_p(None), C.c_void_p(0x1000)
    odd = C.c_void_p(0x1001)

    def fwd(d, *a):
        a = list(a) or [fake] * 11
        return L_.cawn_delta_rule_fwd(C.byref(d), *a, 1 << 40, null)

    def bwd(d, *a):
        a = list(a) or [fake] * 16
        return L_.cawn_delta_rule_bwd(C.byref(d), *a, 1 << 40, null)

    for call in (fwd, bwd):
        for bad in (K.make_delta_desc(-1, 4, 2, 8, 8), K.make_delta_desc(1, -4, 2, 8, 8), K.make_delta_desc(1, 4, 0, 8, 8),
                    K.make_delta_desc(1, 4, 2, 0, 8), K.make_delta_desc(1, 4, 2, 8, 0), K.make_delta_desc(1, 4, 3, 8, 8, Hk=2),
                    K.make_delta_desc(1, 4, 2, 8, 8, bf16=2), K.make_delta_desc(1, 4, 2, 8, 8, qk_norm=3),
                    K.make_delta_desc(1, 4, 2, 8, 8, qk_stride_t=15), K.make_delta_desc(1, 4, 2, 8, 8, v_stride_t=15),
                    K.make_delta_desc(1, 4, 2, 8, 8, o_stride_t=15)):
            assert call(bad) == K.CAWN_EINVAL
            assert K.cawn_delta_state_bytes(bad) == K.cawn_delta_ckpt_bytes(bad) == K.cawn_delta_workspace_bytes(bad) == 0
        assert call(K.make_delta_desc(1, 4, 2, 129, 8)) == K.CAWN_EUNSUPPORTED
    ok = K.make_delta_desc(1, 4, 2, 8, 8)
    assert L_.cawn_delta_rule_fwd(None, *([fake] * 11), 0, null) == K.CAWN_EINVAL
    for i in (0, 1, 2, 3, 4, 7):                                     # required pointers, then misaligned ones
        assert fwd(ok, *[null if j == i else fake for j in range(11)]) == K.CAWN_EINVAL, i
        assert fwd(ok, *[odd if j == i else fake for j in range(11)]) == K.CAWN_EINVAL, i
    long_ = K.make_delta_desc(1, 400, 2, 8, 8)
    assert L_.cawn_delta_rule_fwd(C.byref(long_), *([fake] * 11), 16, null) == K.CAWN_EWORKSPACE
    assert L_.cawn_delta_rule_fwd(C.byref(long_), *([fake] * 10), C.c_void_p(0x1010), 1 << 40, null) == K.CAWN_EWORKSPACE
    for i in (0, 1, 2, 3, 4, 6, 7):
        assert bwd(ok, *[null if j == i else fake for j in range(16)]) == K.CAWN_EINVAL, i
    assert L_.cawn_delta_rule_bwd(C.byref(ok), *([fake] * 16), 16, null) == K.CAWN_EWORKSPACE
    assert K.cawn_delta_state_bytes(K.make_delta_desc(3, 4, 2, 8, 5)) == 3 * 2 * 8 * 5 * 4

    def nfwd(d, *a):
        a = list(a) or [fake] * 6
        return L_.cawn_group_norm_fwd(C.byref(d), *a, 1 << 40, null)

    for bad in (K.make_norm_desc(-1, 1, 8, 2), K.make_norm_desc(1, -1, 8, 2), K.make_norm_desc(1, 1, 0, 1), K.make_norm_desc(1, 1, 8, 3),
                K.make_norm_desc(1, 1, 8, 0), K.make_norm_desc(1, 1, 8, 2, act=3), K.make_norm_desc(1, 1, 8, 2, act=-1),
                K.make_norm_desc(1, 1, 8, 2, bf16=2), K.make_norm_desc(1, 1, 8, 2, x_stride_t=7), K.make_norm_desc(1, 1, 8, 2, y_stride_t=7)):
        assert nfwd(bad) == K.CAWN_EINVAL
        assert L_.cawn_group_norm_bwd(C.byref(bad), *([fake] * 9), 1 << 40, null) == K.CAWN_EINVAL
        assert K.cawn_group_norm_workspace_bytes(bad) == 0
    nd = K.make_norm_desc(2, 3, 8, 2)
    for i in (0, 3):
        assert nfwd(nd, *[null if j == i else fake for j in range(6)]) == K.CAWN_EINVAL
        assert nfwd(nd, *[odd if j == i else fake for j in range(6)]) == K.CAWN_EINVAL
    assert L_.cawn_group_norm_fwd(C.byref(nd), *([fake] * 6), 8, null) == K.CAWN_EWORKSPACE
    for i in (0, 3, 4):
        assert L_.cawn_group_norm_bwd(C.byref(nd), *[null if j == i else fake for j in range(9)], 1 << 40, null) == K.CAWN_EINVAL
    assert L_.cawn_group_norm_bwd(C.byref(nd), *([fake] * 9), 8, null) == K.CAWN_EWORKSPACE

    for bad in (K.make_dropout_desc(-1, 4), K.make_dropout_desc(4, -1), K.make_dropout_desc(4, 4, p=-0.1), K.make_dropout_desc(4, 4, p=1.5),
                K.make_dropout_desc(4, 4, p=float("nan")), K.make_dropout_desc(4, 4, bf16=2), K.make_dropout_desc(4, 4, x_stride=3),
                K.make_dropout_desc(4, 4, y_stride=3), K.make_dropout_desc(4, 4, residual_stride=3)):
        assert L_.cawn_dropout_add_fwd(C.byref(bad), fake, fake, fake, fake, null) == K.CAWN_EINVAL
    dd = K.make_dropout_desc(4, 4)
    for i in (0, 2, 3):
        assert L_.cawn_dropout_add_fwd(C.byref(dd), *[null if j == i else fake for j in range(4)], null) == K.CAWN_EINVAL
        assert L_.cawn_dropout_add_fwd(C.byref(dd), *[odd if j == i else fake for j in range(4)], null) == K.CAWN_EINVAL
    for i in range(3):
        assert L_.cawn_dropout_add_bwd(C.byref(dd), *[null if j == i else fake for j in range(3)], null) == K.CAWN_EINVAL
    # nothing to do is no error
    assert L_.cawn_dropout_add_fwd(C.byref(K.make_dropout_desc(0, 4)), null, null, null, null, null) == K.CAWN_OK
    assert fwd(K.make_delta_desc(0, 4, 2, 8, 8), *([null] * 11)) == K.CAWN_OK


def test_operator_descriptors_match_the_header():
    import os
    import re
    hdr = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "cawn.h")).read()
    for ty in (K.cawn_delta_desc, K.cawn_norm_desc, K.cawn_dropout_desc):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (ty.__name__, ty.__name__), hdr, re.S).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        names = [n.strip() for decl in body.split(";") if decl.strip() for n in decl.strip().split(None, 1)[1].split(",")]
        assert names == [f[0] for f in ty._fields_]


def test_marshalling_of_operators_refuses_what_it_cannot_pass():
    import torch
    d = K.make_dropout_desc(-1, 4)
    assert K.cawn_dropout_add_bwd(d, None, None, None, stream=0) == K.CAWN_EINVAL
    assert K.cawn_delta_rule_bwd(K.make_delta_desc(-1, 1, 1, 1, 1), *([None] * 16), stream=0) == K.CAWN_EINVAL
    assert K.cawn_delta_rule_fwd(K.make_delta_desc(-1, 1, 1, 1, 1), *([None] * 11), stream=0) == K.CAWN_EINVAL
    assert K.cawn_group_norm_fwd(K.make_norm_desc(-1, 1, 1, 1), *([None] * 6), stream=0) == K.CAWN_EINVAL
    assert K.cawn_group_norm_bwd(K.make_norm_desc(-1, 1, 1, 1), *([None] * 9), stream=0) == K.CAWN_EINVAL
    with pytest.raises(AssertionError, match="device pointers"):
        K.cawn_dropout_add_bwd(d, torch.zeros(4), None, None, stream=0)
    with pytest.raises(TypeError, match="cawn_dropout_desc"):
        K.cawn_dropout_add_bwd(K.make_norm_desc(1, 1, 1, 1), None, None, None, stream=0)
    with pytest.raises(TypeError, match="cawn_delta_desc"):
        K.cawn_delta_rule_fwd(K.make_desc(1, 1, 1, 1), *([None] * 11), stream=0)
