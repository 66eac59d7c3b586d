"""Where the launches of the selective scan and the short convolution end: 2^32 threads (CPU only, nothing is launched)."""
import ctypes as C

import pytest

from paper_2604_04250_amd import binding as K

FAKE, BIG = C.c_void_p(0x1000), 1 << 50


def _scan(d, form):
    """What a call of the form says before anything is launched; nothing is if it is not refused for its size."""
    L = K.lib()
    ckpt = None if form == "tokens" else FAKE
    if form == "back":
        return L.cawn_selective_scan_bwd(C.byref(d), *([FAKE] * 21), C.c_void_p(0x1010), BIG, None)
    return L.cawn_selective_scan_fwd(C.byref(d), *([FAKE] * 10), C.c_void_p(0x1001), FAKE, ckpt, FAKE, BIG, None)


# the last number of rows that a launch has threads for: threads of a row in the tiled form
@pytest.mark.parametrize("L", [17, 100])
@pytest.mark.parametrize("D,N,G,threads", [(64, 1, 1, 64), (65, 4, 1, 128), (256, 1, 1, 256), (320, 1, 1, 512), (3, 1, 3, 192), (64, 20, 1, 128), (64, 64, 1, 256), (64, 128, 1, 512)])
def test_rows_of_the_scan_by_tiles(D, N, G, threads, L):
    most = ((1 << 32) - 1) // threads
    held, beyond = (K.make_scan_desc(B, L, D, N, G=G) for B in (most, most + 1))
    assert K.cawn_selective_scan_state_bytes(held) == most * D * N * 4
    assert K.cawn_selective_scan_ckpt_bytes(held) > 0 and K.cawn_selective_scan_workspace_bytes(held) > 0
    assert _scan(held, "tiles") == K.CAWN_EINVAL and _scan(held, "back") == K.CAWN_EWORKSPACE           # (a misaligned y, a misaligned workspace)
    for f in (K.cawn_selective_scan_state_bytes, K.cawn_selective_scan_ckpt_bytes, K.cawn_selective_scan_workspace_bytes):
        assert f(beyond) == 0
    for form in ("tokens", "tiles", "back"):
        assert _scan(beyond, form) == K.CAWN_EUNSUPPORTED


@pytest.mark.parametrize("D,N,threads", [(64, 1, 64), (64, 4, 64), (1000, 8, 1000), (128, 16, 256), (64, 128, 1024)])
def test_rows_of_the_scan_by_tokens(D, N, threads):
    """The state of up to 16 tokens without a checkpoint; with one, and backward, the tiled form has its own end."""
    most = ((1 << 32) - 256) // threads
    held, beyond = (K.make_scan_desc(B, 1, D, N) for B in (most, most + 1))
    assert K.cawn_selective_scan_state_bytes(held) == most * D * N * 4 and K.cawn_selective_scan_workspace_bytes(held) >= 256
    assert _scan(held, "tokens") == K.CAWN_EINVAL
    assert _scan(beyond, "tokens") == K.CAWN_EUNSUPPORTED


def test_more_rows_by_tokens_than_by_tiles():
    d = K.make_scan_desc(1 << 27, 1, 1, 1)
    assert K.cawn_selective_scan_state_bytes(d) == 4 << 27 and K.cawn_selective_scan_workspace_bytes(d) == 256 and K.cawn_selective_scan_ckpt_bytes(d) == 0
    assert _scan(d, "tokens") == K.CAWN_EINVAL
    assert _scan(d, "tiles") == _scan(d, "back") == K.CAWN_EUNSUPPORTED


def test_tokens_and_groups_that_the_launches_go_round_for():
    for d in (K.make_scan_desc(1, 1 << 30, 4, 1), K.make_scan_desc(64, 1 << 20, 64, 1, G=64)):
        assert K.cawn_selective_scan_ckpt_bytes(d) > 0 and K.cawn_selective_scan_workspace_bytes(d) > 0
        assert _scan(d, "tiles") == K.CAWN_EINVAL and _scan(d, "back") == K.CAWN_EWORKSPACE


@pytest.mark.parametrize("L,channels,k,threads", [(1, 64, 4, 16), (8, 13, 2, 4), (33, 3, 1, 6), (65, 1024, 4, 768)])
def test_rows_of_the_convolution(L, channels, k, threads):
    """Threads of a row: runs of 32 tokens, four channels each or, of fewer than four, one."""
    most = ((1 << 32) - 256) // threads
    held, beyond = (K.make_conv_desc(B, L, channels, k) for B in (most, most + 256 // threads + 1))
    fwd = lambda d: K.lib().cawn_causal_conv_fwd(C.byref(d), *([FAKE] * 5), C.c_void_p(0x1001), FAKE, None)  # noqa: E731
    assert K.cawn_causal_conv_state_bytes(held) == most * (k - 1) * channels * 4
    assert fwd(held) == K.CAWN_EINVAL           # (a misaligned y)
    assert K.cawn_causal_conv_state_bytes(beyond) == 0
    assert fwd(beyond) == K.CAWN_EUNSUPPORTED
