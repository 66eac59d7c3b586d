"""Scratch of a program that only serves (CPU only, nothing is launched)."""
import ctypes as C

import pytest

from paper_2604_04250_amd import binding as K

FAKE, BIG = C.c_void_p(0x1000), 1 << 50


def _forward(d, nbytes):
    return K.lib().cawn_selective_scan_fwd(C.byref(d), *([FAKE] * 12), None, FAKE, nbytes, None)


def test_a_forward_without_a_checkpoint_needs_none_of_the_partial_sums():
    d = K.make_scan_desc(2, 32768, 4096, 128, bf16=1)
    serve, both = K.cawn_selective_scan_serve_workspace_bytes(d), K.cawn_selective_scan_workspace_bytes(d)
    # B and C in fp32, and of eight segments a row what they make of zero, their begin and their sum of delta
    assert serve == 2 * 32768 * 2 * 128 * 4 + 2 * 8 * (2 * 4096 * 128 + 4096) * 4 and both > 30 * serve
    assert _forward(d, serve - 1) == K.CAWN_EWORKSPACE
    step = K.make_scan_desc(128, 1, 4096, 16, bf16=1)
    assert K.cawn_selective_scan_serve_workspace_bytes(step) == 256 and K.cawn_selective_scan_workspace_bytes(step) > 10 << 20


@pytest.mark.parametrize("B,L,D,N,G", [(1, 17, 64, 16, 1), (3, 1000, 768, 16, 1), (2, 333, 48, 100, 3), (64, 200, 1024, 8, 2)])
def test_it_is_what_the_forward_asks_for(B, L, D, N, G):
    d = K.make_scan_desc(B, L, D, N, G=G)
    serve = K.cawn_selective_scan_serve_workspace_bytes(d)
    assert 256 < serve <= K.cawn_selective_scan_workspace_bytes(d)
    assert _forward(d, serve - 1) == K.CAWN_EWORKSPACE


def test_none_for_what_is_refused():
    for d in (K.make_scan_desc(-1, 100, 32, 16), K.make_scan_desc(2, 100, 32, 129), K.make_scan_desc(1 << 26, 17, 64, 1), K.make_scan_desc(1 << 26, 1, 64, 1)):
        assert K.cawn_selective_scan_serve_workspace_bytes(d) == 0
    assert K.cawn_selective_scan_serve_workspace_bytes(K.make_scan_desc(0, 100, 32, 16)) == 256
