"""How the gated delta rule cuts a row into segments, as the checkpoint's size shows it (CPU only)."""
import pytest

from paper_2604_04250_amd import binding as K


def _segments(B, L, H, Kd, V, bf16):
    """From the checkpoint: per head and chunk a state, u, 9 x 64 gates (all of them to the next KiB) and 18 KiB of T; per head and segment a matrix."""
    KP, VT, heads, chunks = 32 if Kd <= 32 else 64 if Kd <= 64 else 128, -(-V // 16), B * H, -(-L // 64)
    fixed = heads * chunks * 1024 * ((KP // 16) * VT + 4 * VT + 18) + -(-heads * chunks * 9 * 64 * 4 // 1024) * 1024
    rest = K.cawn_delta_ckpt_bytes(K.make_delta_desc(B, L, H, Kd, V, bf16=bf16)) - fixed
    assert rest >= 0 and rest % (heads * KP * KP * 4) == 0
    return max(1, rest // (heads * KP * KP * 4))


# workgroups of the outputs' pass that are there at once: 256 compute units, each holding what registers and LDS leave room for
@pytest.mark.parametrize("bf16,Kd,held", [(0, 64, 2), (1, 64, 3), (1, 128, 2), (0, 32, 3)])
def test_no_call_is_cut_into_more_workgroups_than_are_there_at_once(bf16, Kd, held):
    cut = 0
    for B in (1, 2, 3, 5, 7, 10, 16, 33):
        for H, V in ((4, 128), (12, 64), (3, 40)):
            groups = B * H * -(-V // 64)
            for L in range(1, 2600, 64):
                n = _segments(B, L, H, Kd, V, bf16)
                assert n <= -(-L // 64)
                if n > 1:
                    assert n >= 3 and n * groups <= 256 * held, (B, L, H, V, n)
                    cut += 1
    assert cut > 100
