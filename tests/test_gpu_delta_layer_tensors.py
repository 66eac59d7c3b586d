"""The example's functions on tensors as programs have them: strided."""
import pytest
import torch

from gpu_util import DEV
from test_gpu_delta_layer import E

pytestmark = pytest.mark.gpu


def _inputs(B=2, L=70, H=2, Kw=32, V=40):
    gen = torch.Generator(device=DEV).manual_seed(3)
    new = lambda *s: torch.randn(s, generator=gen, device=DEV)  # noqa: E731
    return [new(B, L, H, Kw), new(B, L, H, Kw), new(B, L, H, V), -new(B, L, H).abs(), torch.sigmoid(new(B, L, H)), new(B, H, Kw, V)]


def _strided(t):
    """The same values, every second element of a row twice as long."""
    return torch.stack([t, torch.full_like(t, float("nan"))], -1)[..., 0]


def _gradients(f, inputs, weights):
    inputs = [t.detach().requires_grad_() for t in inputs]
    outs = f(*inputs)
    outs = outs if isinstance(outs, tuple) else (outs,)
    return [t.detach() for t in outs] + list(torch.autograd.grad(outs, inputs, weights))


def test_strided_tensors_are_what_their_values_are():
    x = _inputs()
    wo, ws = torch.randn_like(x[2]), torch.randn_like(x[5])
    rule = lambda *a: E.DeltaRule.apply(*a, None)  # noqa: E731
    for got, want in zip(_gradients(rule, [_strided(t) for t in x], [_strided(wo), ws.transpose(2, 3).contiguous().transpose(2, 3)]), _gradients(rule, x, [wo, ws])):
        assert torch.equal(got, want)
    t, w, b = torch.randn(33, 96, device=DEV), torch.randn(96, device=DEV), torch.randn(96, device=DEV)
    norm = lambda *a: E.HeadNorm.apply(*a, 4)  # noqa: E731
    dy = torch.randn_like(t)
    for got, want in zip(_gradients(norm, [_strided(t), _strided(w), _strided(b)], [_strided(dy)]), _gradients(norm, [t, w, b], [dy])):
        assert torch.equal(got, want)
    state = torch.randn(2, 2, 40, 32, device=DEV).transpose(2, 3)
    assert torch.equal(E.DeltaRule.apply(*x[:5], state, None)[1], E.DeltaRule.apply(*x[:5], state.contiguous(), None)[1])
