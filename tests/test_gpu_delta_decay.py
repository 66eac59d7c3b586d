"""Gradient of the decays where much is forgotten: it shrinks with e^decay, and is judged on its own scale.

Every term of it carries the factor by which a state shrinks across the token, so its error is that of the other fp32 gradients (4e-5 of their
root mean square), whatever the factor."""
import numpy as np
import pytest

from gpu_util import rel_err
from test_gpu_delta import desc, host, make, num
from test_gpu_delta_bwd import TOL, ref, run

pytestmark = pytest.mark.gpu


def _own_scale(got, want):
    """Largest error in units of a value or of the root mean square, scaled so that neither underflows."""
    size = np.sqrt(np.mean((want / np.abs(want).max()) ** 2)) * np.abs(want).max()
    return rel_err(got.astype(np.float64) / size, want / size)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("decay", [-1.0, -4.0, -8.0, -12.0, -20.0, -60.0])
@pytest.mark.parametrize("B,L,H,Hk,Kd,V,norm", [(1, 150, 2, 2, 64, 64, 1), (2, 450, 2, 1, 128, 40, 0), (1, 97, 4, 2, 24, 72, 1)])
def test_the_same_decay_everywhere(B, L, H, Hk, Kd, V, norm, decay, bf16):
    x = make(B, L, H, Hk, Kd, V, bf16, norm, int(L - 3 * decay))
    x["decay"][:] = decay
    got = run(x, desc(x, norm), want=("ddecay",))
    assert _own_scale(num(got["ddecay"]), ref(host(x), norm)["ddecay"]) <= TOL


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("decay", [-8.0, -15.0, -40.0])
def test_a_few_tokens_that_forget_almost_everything(decay, bf16):
    """Those tokens' gradients by themselves, and the others'."""
    x = make(2, 200, 2, 1, 64, 72, bf16, 1, 31, [200, 133])
    x["decay"][:] = -0.05
    x["decay"][:, 3::5] = decay
    some = np.zeros(x["decay"].shape, bool)
    some[0, 3::5] = some[1, 3:133:5] = True
    got, want = num(run(x, desc(x, 1), want=("ddecay",))["ddecay"]), ref(host(x), 1)["ddecay"]
    assert _own_scale(got[some], want[some]) <= TOL
    rest = ~some
    rest[1, 133:] = False
    assert _own_scale(got[rest], want[rest]) <= TOL
