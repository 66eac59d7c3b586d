"""bf16 calls of the gated delta rule hold the arithmetic of fp32: what a large state leaves where it has just been overwritten."""
import pytest

from gpu_util import rel_err
from test_gpu_delta import desc, fwd, host, make, num, ref_fwd

pytestmark = pytest.mark.gpu

# The state is SIZE times the values.  A query of the key just written, with beta = 1, finds the value alone: products of SIZE that cancel
# to one.  Each is held to some 100 roundings of 2^-24; a bf16 output adds 2^-8 of itself.
SIZE = 1000.0
TERMS = SIZE * 100 * 2.0 ** -24
TOL16 = 2.0 ** -8 + TERMS


def _overwritten(L, Kd, V, seed):
    x = make(1, L, 2, 2, Kd, V, True, 1, seed)
    x["state_in"] *= SIZE
    x["beta"][:] = 1
    x["decay"][:] = -1e-3
    x["q"] = x["k"].clone()
    return x


@pytest.mark.parametrize("L,Kd,V", [(17, 64, 64), (64, 64, 72), (130, 128, 64), (100, 32, 40), (450, 64, 64)])
def test_values_written_over_a_large_state(L, Kd, V):
    x = _overwritten(L, Kd, V, L)
    want = ref_fwd(host(x), 1)[0]
    o = num(fwd(x, desc(x, 1))[0])
    assert rel_err(o, want) <= TOL16
    # token by token the same
    for t in range(0, 16):
        assert rel_err(o[:, t], want[:, t]) <= TOL16
