"""The example's functions on tensors as programs have them: strided, of other types, differentiated twice."""
import pytest
import torch

from gpu_util import DEV, rel_err
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


def test_a_layer_in_bfloat16():
    """Against the same weights and inputs in fp32: five roundings of 2^-8 on the way, five deviations of them, and a norm between; 0.1 of the root
    mean square is far from wrong."""
    torch.manual_seed(9)
    low = E.DeltaLayer(64, 2, 2, 32, 32, p=0.0).to(DEV).to(torch.bfloat16)
    high = E.DeltaLayer(64, 2, 2, 32, 32, p=0.0).to(DEV)
    high.load_state_dict({n: t.float() if t.is_floating_point() else t for n, t in low.state_dict().items()})
    x = torch.randn(3, 90, 64, device=DEV).bfloat16()
    dy = torch.randn_like(x)
    a, b = x.clone().requires_grad_(), x.float().requires_grad_()
    y, want = low(a)[0], high(b)[0]
    y.backward(dy)
    want.backward(dy.float())
    assert rel_err(y.detach().float().cpu(), want.detach().cpu()) <= 0.1 and rel_err(a.grad.float().cpu(), b.grad.cpu()) <= 0.1
    for n in ("norm_w", "norm_b"):
        got, ref = getattr(low, n).grad, getattr(high, n).grad
        assert got.dtype == torch.bfloat16 and rel_err(got.float().cpu(), ref.cpu()) <= 0.1


def test_types_that_would_be_misread_are_refused():
    x = _inputs()
    for i in range(6):
        y = list(x)
        y[i] = y[i].double() if i == 2 else y[i].bfloat16()
        with pytest.raises(TypeError):
            E.DeltaRule.apply(*y, None)
    with pytest.raises(TypeError, match="lengths"):
        E.DeltaRule.apply(*x, torch.tensor([70, 3], device=DEV))
    t = torch.randn(8, 32, device=DEV)
    with pytest.raises(TypeError):
        E.HeadNorm.apply(t.half(), t[0], t[0], 2)
    with pytest.raises(TypeError, match="residual"):
        E.DropoutAdd.apply(t, t.bfloat16(), torch.tensor([1, 0], device=DEV), 0.1)
    with pytest.raises(TypeError, match="rng"):
        E.DropoutAdd.apply(t, t, torch.tensor([1, 0], device=DEV, dtype=torch.int32), 0.1)


def test_a_second_derivative_is_an_error():
    x = [t.requires_grad_() for t in _inputs()]
    t, w = torch.randn(8, 32, device=DEV, requires_grad=True), torch.randn(32, device=DEV, requires_grad=True)
    for out, at in ((E.DeltaRule.apply(*x, None)[0], x[0]), (E.HeadNorm.apply(t, w, w, 2), t), (E.DropoutAdd.apply(t, t, torch.tensor([1, 0], device=DEV), 0.1), t)):
        g, = torch.autograd.grad(out.square().sum(), at, create_graph=True)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            g.square().sum().backward()
