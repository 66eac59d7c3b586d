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


def test_a_clip_of_the_longest_length():
    """One channel, 2^31 - 1 tokens in bf16.  A value is some ten roundings of 2^-24 from its inputs, then one of 2^-8; a column sum of 2^31 terms that 2^17 threads
    add up, 2^14 each, holds 2^-24 of a thread's own sum in each addition: 2^7 roundings of random sign, 1e-5 of the sum's usual size."""
    T = 2 ** 31 - 1
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, dy = _filled(T, gen), _filled(T, gen)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    w, b = torch.full((1,), 1.25, device=DEV), torch.full((1,), -0.5, device=DEV)
    stats, dw, db = torch.empty(1, 1, 2, device=DEV), torch.empty(1, device=DEV), torch.empty(1, device=DEV)
    d = K.make_norm_desc(1, T, 1, 1, bf16=1)
    ws = torch.empty(max(256, K.cawn_group_norm_workspace_bytes(d)), dtype=torch.uint8, device=DEV)
    K.check(K.cawn_group_norm_fwd(d, x, w, b, y, stats, ws))
    K.check(K.cawn_group_norm_bwd(d, x, w, b, stats, dy, dx, dw, db, ws))
    torch.cuda.synchronize()
    mean, rstd = _moments(x)
    assert abs(float(stats[0, 0, 0]) - mean) <= 4e-6 and abs(float(stats[0, 0, 1]) / rstd - 1) <= 4e-6
    total = lambda f: sum(float(f(s)) for s in _parts(T))  # noqa: E731
    xh = lambda s: (x[0, s].double() - mean) * rstd  # noqa: E731
    sum_b, sum_w = total(lambda s: dy[0, s].double().sum()), total(lambda s: (dy[0, s].double() * xh(s)).sum())
    assert abs(float(db) - sum_b) <= 2e-5 * max(abs(sum_b), T ** 0.5) and abs(float(dw) - sum_w) <= 2e-5 * max(abs(sum_w), T ** 0.5)
    for s in _parts(T):
        for got, want in ((y, 1.25 * xh(s) - 0.5), (dx, 1.25 * rstd * (dy[0, s].double() - sum_b / T - xh(s) * (sum_w / T)))):
            err = (got[0, s].double() - want).abs()
            assert bool((err <= (2.0 ** -8 + 4e-6) * want.abs().clamp_min(1.0)).all())


def test_many_rows_of_more_tokens_than_a_plain_sum_takes():
    """More rows than workgroups, so that one takes rows one after the other, each of 150 tokens a thread: sums are folded within a row and begin anew with the next."""
    B, T, C = 2049, 150, 2048
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.empty(B, T, C, device=DEV, dtype=torch.bfloat16)
    for b in range(0, B, 512):
        x[b:b + 512] = torch.randn(x[b:b + 512].shape, generator=gen, device=DEV).bfloat16() * 1.5 + 0.25
    x[2048] = x[2048] * 3 - 7
    x[0] += 5
    y, stats = torch.empty_like(x), torch.empty(B, 2, 2, device=DEV)
    d = K.make_norm_desc(B, T, C, 2, act=1, bf16=1)
    ws = torch.empty(max(256, K.cawn_group_norm_workspace_bytes(d)), dtype=torch.uint8, device=DEV)
    K.check(K.cawn_group_norm_fwd(d, x, None, None, y, stats, ws))
    torch.cuda.synchronize()
    for b in (0, 1, 1024, 2047, 2048):
        v = x[b].double().view(T, 2, C // 2)
        mean, var = v.mean((0, 2)), v.var((0, 2), correction=0)
        rstd = (var + 1e-5) ** -0.5
        assert bool(((stats[b, :, 0].double() - mean).abs() <= 4e-6 * mean.abs().clamp_min(1.0)).all()) and bool(((stats[b, :, 1].double() / rstd - 1).abs() <= 4e-6).all())
        z = (v - mean[None, :, None]) * rstd[None, :, None]
        want = (z * torch.sigmoid(z)).view(T, C)
        assert bool(((y[b].double() - want).abs() <= (2.0 ** -8 + 1e-5) * want.abs().clamp_min(1.0)).all())
