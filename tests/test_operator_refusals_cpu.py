"""Refusals of the operators beside the scan that their entry points owe every pointer (CPU only, nothing is launched)."""
import ctypes as C

import pytest

from paper_2604_04250_amd import binding as K

FAKE, ODD = C.c_void_p(0x1000), C.c_void_p(0x1001)


def _with(n, i):
    return [ODD if j == i else FAKE for j in range(n)]


@pytest.mark.parametrize("rows", [2, 0])
@pytest.mark.parametrize("bf16", [0, 1])
def test_group_norm_refuses_every_misaligned_pointer(bf16, rows):
    """Statistics and gradients of parameters among them, also where there is nothing to normalise and only the latter are written."""
    L_ = K.lib()
    d = K.make_norm_desc(rows, 3, 8, 2, bf16=bf16)
    for i in (0, 1, 2, 3, 4) if rows else (4,):
        assert L_.cawn_group_norm_fwd(C.byref(d), *_with(6, i), 1 << 40, None) == K.CAWN_EINVAL, i
    for i in (0, 1, 2, 3, 4, 5, 6, 7) if rows else (6, 7):
        assert L_.cawn_group_norm_bwd(C.byref(d), *_with(9, i), 1 << 40, None) == K.CAWN_EINVAL, i


def test_delta_rule_refuses_every_misaligned_pointer():
    L_ = K.lib()
    d = K.make_delta_desc(1, 400, 2, 8, 8)
    for i in range(10):
        assert L_.cawn_delta_rule_fwd(C.byref(d), *_with(11, i), 1 << 40, None) == K.CAWN_EINVAL, i
    for i in range(15):
        assert L_.cawn_delta_rule_bwd(C.byref(d), *_with(16, i), 1 << 40, None) == K.CAWN_EINVAL, i
