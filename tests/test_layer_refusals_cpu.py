"""Refusals of the selective scan, the short convolution and the norm (CPU only, nothing is launched)."""
import ctypes as C

import pytest

from paper_2604_04250_amd import binding as K

FAKE, ODD = C.c_void_p(0x1000), C.c_void_p(0x1001)
BIG = 1 << 40


def _args(n, bad=None, what=ODD):
    return [what if j == bad else FAKE for j in range(n)]


def test_scan_refusals():
    L = K.lib()
    fwd, bwd = L.cawn_selective_scan_fwd, L.cawn_selective_scan_bwd

    def both(d, want):
        r = C.byref(d) if d is not None else None
        assert fwd(r, *_args(14), BIG, None) == want
        assert bwd(r, *_args(22), BIG, None) == want

    both(None, K.CAWN_EINVAL)
    for k in (dict(B=-1), dict(L=-1), dict(D=0), dict(N=0), dict(G=-1), dict(G=3), dict(bf16=2), dict(dt_softplus=2), dict(x_stride_t=31), dict(dt_stride_t=31),
              dict(bc_stride_t=31, G=2), dict(z_stride_t=5), dict(y_stride_t=31)):
        d = K.make_scan_desc(**{**dict(B=2, L=100, D=32, N=16), **k})
        both(d, K.CAWN_EINVAL)
        assert K.cawn_selective_scan_workspace_bytes(d) == K.cawn_selective_scan_ckpt_bytes(d) == K.cawn_selective_scan_state_bytes(d) == 0
    both(K.make_scan_desc(2, 100, 32, 129), K.CAWN_EUNSUPPORTED)
    both(K.make_scan_desc(1 << 30, 1 << 30, 32, 16), K.CAWN_EUNSUPPORTED)      # sizes beyond what is counted
    d = K.make_scan_desc(2, 100, 32, 16)
    for i in range(13):
        assert fwd(C.byref(d), *_args(14, i), BIG, None) == K.CAWN_EINVAL, i
    for i in range(21):
        assert bwd(C.byref(d), *_args(22, i), BIG, None) == K.CAWN_EINVAL, i
    for i in (0, 1, 2, 3, 4, 10):
        assert fwd(C.byref(d), *_args(14, i, None), BIG, None) == K.CAWN_EINVAL, i
    for i in (0, 1, 2, 3, 4, 9, 10):
        assert bwd(C.byref(d), *_args(22, i, None), BIG, None) == K.CAWN_EINVAL, i
    for i in (5, 6, 7):                 # a gradient of what is not there: Dskip, z, dt_bias
        assert bwd(C.byref(d), *_args(22, i, None), BIG, None) == K.CAWN_EINVAL, i
    for f, n in ((fwd, 14), (bwd, 22)):
        assert f(C.byref(d), *_args(n), 16, None) == K.CAWN_EWORKSPACE
        assert f(C.byref(d), *_args(n, n - 1, None), BIG, None) == K.CAWN_EWORKSPACE
        assert f(C.byref(d), *_args(n, n - 1, C.c_void_p(0x1010)), BIG, None) == K.CAWN_EWORKSPACE
    assert fwd(C.byref(K.make_scan_desc(0, 100, 32, 16)), *([None] * 14), 0, None) == K.CAWN_OK


@pytest.mark.parametrize("bf16", [0, 1])
def test_conv_refusals(bf16):
    L = K.lib()
    fwd, bwd = L.cawn_causal_conv_fwd, L.cawn_causal_conv_bwd

    def both(d, want):
        r = C.byref(d) if d is not None else None
        assert fwd(r, *_args(7), None) == want
        assert bwd(r, *_args(12), BIG, None) == want

    both(None, K.CAWN_EINVAL)
    for k in (dict(B=-1), dict(L=-1), dict(C=0), dict(k=0), dict(act=2), dict(act=-1), dict(bf16=2), dict(x_stride_t=23), dict(y_stride_t=23)):
        d = K.make_conv_desc(**{**dict(B=2, L=10, C=24, k=4, bf16=bf16), **k})
        both(d, K.CAWN_EINVAL)
        assert K.cawn_causal_conv_workspace_bytes(d) == K.cawn_causal_conv_state_bytes(d) == 0
    both(K.make_conv_desc(2, 10, 24, 5, bf16=bf16), K.CAWN_EUNSUPPORTED)
    reserved = K.make_conv_desc(2, 10, 24, 4, bf16=bf16)
    reserved.reserved = 1
    both(reserved, K.CAWN_EINVAL)
    d = K.make_conv_desc(2, 10, 24, 4, bf16=bf16)
    for i in range(7):
        assert fwd(C.byref(d), *_args(7, i), None) == K.CAWN_EINVAL, i
    for i in range(11):
        assert bwd(C.byref(d), *_args(12, i), BIG, None) == K.CAWN_EINVAL, i
    for i in (0, 1, 5):
        assert fwd(C.byref(d), *_args(7, i, None), None) == K.CAWN_EINVAL, i
    for i in (0, 1, 5):
        assert bwd(C.byref(d), *_args(12, i, None), BIG, None) == K.CAWN_EINVAL, i
    assert bwd(C.byref(d), *_args(12), 16, None) == K.CAWN_EWORKSPACE
    assert bwd(C.byref(d), *_args(12, 11, None), BIG, None) == K.CAWN_EWORKSPACE
    assert bwd(C.byref(d), *_args(12, 11, C.c_void_p(0x1010)), BIG, None) == K.CAWN_EWORKSPACE
    assert fwd(C.byref(K.make_conv_desc(0, 10, 24, 4)), *([None] * 7), None) == K.CAWN_OK


@pytest.mark.parametrize("bf16,res", [(0, 0), (1, 0), (1, 1), (0, 1)])
def test_norm_refusals(bf16, res):
    L = K.lib()
    fwd, bwd = L.cawn_rms_norm_add_fwd, L.cawn_rms_norm_add_bwd

    def both(d, want):
        r = C.byref(d) if d is not None else None
        assert fwd(r, *_args(8), None) == want
        assert bwd(r, *_args(9), BIG, None) == want

    both(None, K.CAWN_EINVAL)
    for k in (dict(rows=-1), dict(C=0), dict(bf16=2), dict(residual_bf16=-1), dict(block=-16), dict(block=24), dict(x_stride=63), dict(residual_stride=63), dict(y_stride=63)):
        d = K.make_rms_desc(**{**dict(rows=4, C=64, bf16=bf16, residual_bf16=res), **k})
        both(d, K.CAWN_EINVAL)
        assert K.cawn_rms_norm_add_workspace_bytes(d) == 0
    both(K.make_rms_desc(4, 32769, bf16=bf16, residual_bf16=res), K.CAWN_EUNSUPPORTED)
    d = K.make_rms_desc(4, 64, bf16=bf16, residual_bf16=res)
    for i in (0, 1, 2, 3, 4, 6, 7):
        assert fwd(C.byref(d), *_args(8, i), None) == K.CAWN_EINVAL, i
    for i in range(8):
        assert bwd(C.byref(d), *_args(9, i), BIG, None) == K.CAWN_EINVAL, i
    assert fwd(C.byref(d), *_args(8, 0, None), None) == K.CAWN_EINVAL
    assert fwd(C.byref(d), FAKE, FAKE, FAKE, FAKE, None, None, None, None, None) == K.CAWN_EINVAL        # neither y nor q
    assert fwd(C.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, None, None) == K.CAWN_EINVAL        # q without scales
    assert fwd(C.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, None, None) == K.CAWN_EINVAL        # scales without q
    for i in (0, 2, 3):
        assert bwd(C.byref(d), *_args(9, i, None), BIG, None) == K.CAWN_EINVAL, i
    assert bwd(C.byref(d), *_args(9), 16, None) == K.CAWN_EWORKSPACE
    assert bwd(C.byref(d), *_args(9, 8, None), BIG, None) == K.CAWN_EWORKSPACE
    assert fwd(C.byref(K.make_rms_desc(0, 64)), *_args(8, 0, None)[:5], None, None, None, None) == K.CAWN_OK


def test_the_bindings_wrappers_pass_as_many_arguments_as_their_entry_points_take():
    import inspect
    for name, d in (("cawn_selective_scan_fwd", K.make_scan_desc(-1, 1, 1, 1)), ("cawn_selective_scan_bwd", K.make_scan_desc(-1, 1, 1, 1)),
                    ("cawn_causal_conv_fwd", K.make_conv_desc(-1, 1, 1, 1)), ("cawn_causal_conv_bwd", K.make_conv_desc(-1, 1, 1, 1)),
                    ("cawn_rms_norm_add_fwd", K.make_rms_desc(-1, 1)), ("cawn_rms_norm_add_bwd", K.make_rms_desc(-1, 1))):
        f = getattr(K, name)
        n = len(inspect.signature(f).parameters) - 2
        assert f(d, *([None] * n), stream=0) == K.CAWN_EINVAL, name
        with pytest.raises(TypeError):
            f(K.make_dropout_desc(1, 1), *([None] * n), stream=0)


def test_sizes_whose_places_32_bits_do_not_count_are_refused():
    most = (1 << 31) - 1

    def scan(d):
        return d, "cawn_selective_scan_fwd", [*_args(14), BIG], K.cawn_selective_scan_workspace_bytes

    def conv(d):
        return d, "cawn_causal_conv_fwd", _args(7), K.cawn_causal_conv_workspace_bytes

    for d, name, args, size in (scan(K.make_scan_desc(1, most, 4, 1)), scan(K.make_scan_desc(1, (1 << 30) + 1, 4, 1)),
                             scan(K.make_scan_desc(1, 100, 1 << 25, 1, G=1 << 25)),        # 64 places a group
                             scan(K.make_scan_desc(1, 100, 1 << 26, 1)), scan(K.make_scan_desc(1, 100, 4, 1, dt_stride_t=1 << 26)),
                             conv(K.make_conv_desc(1, most, 1, 4)), conv(K.make_conv_desc(1, 1, most, 4))):
        assert size(d) == 0
        assert getattr(K.lib(), name)(C.byref(d), *args, None) == K.CAWN_EUNSUPPORTED
    assert K.cawn_selective_scan_workspace_bytes(K.make_scan_desc(1, 1 << 30, 4, 1)) > 0
    assert K.cawn_causal_conv_workspace_bytes(K.make_conv_desc(1, 1 << 30, 1, 4)) > 0
