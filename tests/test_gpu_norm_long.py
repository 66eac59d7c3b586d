"""Group norm over clips of very many tokens."""
import pytest
import torch

from gpu_util import DEV
from paper_2604_04250_amd import binding as K

pytestmark = pytest.mark.gpu

PART = 1 << 27


def _filled(T, gen):
    t = torch.empty(1, T, 1, device=DEV, dtype=torch.bfloat16)
    for at in range(0, T, PART):
        n = min(PART, T - at)
        t[0, at:at + n, 0] = (torch.randn(n, generator=gen, device=DEV) * 1.5 + 0.25).bfloat16()
    return t


def _parts(T):
    return [slice(at, min(at + PART, T)) for at in range(0, T, PART)]


def _moments(x):
    total = lambda f: sum(float(f(x[0, s].double())) for s in _parts(x.shape[1]))  # noqa: E731
    mean = total(torch.sum) / x.shape[1]
    return mean, (total(lambda v: (v - mean).square().sum()) / x.shape[1] + 1e-5) ** -0.5


def test_the_variance_of_a_billion_values():
    """Sums of any length hold what sums of some 64 values do: 4e-6, as over short clips."""
    T = 1 << 30
    x = _filled(T, torch.Generator(device=DEV).manual_seed(2))
    y, stats = torch.empty_like(x), torch.empty(1, 1, 2, device=DEV)
    d = K.make_norm_desc(1, T, 1, 1, bf16=1)
    ws = torch.empty(max(256, K.cawn_group_norm_workspace_bytes(d)), dtype=torch.uint8, device=DEV)
    K.check(K.cawn_group_norm_fwd(d, x, None, None, y, stats, ws))
    torch.cuda.synchronize()
    mean, rstd = _moments(x)
    assert abs(float(stats[0, 0, 0]) - mean) <= 4e-6
    assert abs(float(stats[0, 0, 1]) / rstd - 1) <= 4e-6
