"""The example's layer: the new operators together, as a program uses them."""
import importlib.util
import os

import numpy as np
import pytest
import torch
import torch.nn.functional as F

import ops_ref as R
from gpu_util import DEV, rel_err

pytestmark = pytest.mark.gpu

_spec = importlib.util.spec_from_file_location("delta_layer", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                                                                           "delta_layer.py"))
E = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(E)


def _plain(layer, x):
    """The same layer token by token in float64, without dropout."""
    H, Hk, Kw, V = layer.heads, layer.key_heads, layer.key, layer.value
    B, L, width = x.shape
    q, k = F.linear(x, layer.qk.weight).view(B, L, 2, Hk, Kw).unbind(2)
    v = F.linear(x, layer.v.weight).view(B, L, H, V)
    forget, beta = F.linear(x, layer.gates.weight, layer.gates.bias).view(B, L, 2, H).unbind(2)
    q, k = (t / (t.square().sum(-1, keepdim=True) + 1e-6).sqrt() for t in (q, k))
    q, k = (t.repeat_interleave(H // Hk, 2) for t in (q, k))
    S, out = x.new_zeros(B, H, Kw, V), []
    for t in range(L):
        r = S * torch.exp(-F.softplus(forget[:, t]))[..., None, None]
        u = torch.sigmoid(beta[:, t])[..., None] * (v[:, t] - (r * k[:, t][..., None]).sum(2))
        S = r + k[:, t][..., None] * u[:, :, None]
        out.append(Kw ** -0.5 * (S * q[:, t][..., None]).sum(2))
    o = torch.stack(out, 1)
    o = (o - o.mean(-1, keepdim=True)) / (o.var(-1, unbiased=False, keepdim=True) + 1e-5).sqrt()
    z = o.reshape(B, L, H * V) * layer.norm_w + layer.norm_b
    return F.linear(F.silu(z), layer.out.weight) + x


def test_gradients_of_the_layer():
    """Two fp32 matrix products, the mixer, the norm and two more stand between a weight and the loss: each holds 2^-22 or so of its own
    size, and the norm divides by deviations of a tenth, so that 2e-4 of a gradient's root mean square is left to a long way from wrong."""
    torch.manual_seed(5)
    layer = E.DeltaLayer(48, 4, 2, 24, 40, p=0.0).to(DEV)
    x = torch.randn(3, 90, 48, device=DEV, requires_grad=True)
    dy = torch.randn(3, 90, 48, device=DEV)
    y, _ = layer(x)
    y.backward(dy)
    twin = E.DeltaLayer(48, 4, 2, 24, 40, p=0.0).double()
    twin.load_state_dict({n: t.cpu() for n, t in layer.state_dict().items()})
    x64 = x.detach().cpu().double().requires_grad_()
    y64 = _plain(twin, x64)
    y64.backward(dy.cpu().double())
    assert rel_err(y.detach().cpu(), y64.detach()) <= 2e-4
    assert rel_err(x.grad.cpu(), x64.grad) <= 2e-4
    for (n, p), (_, p64) in zip(layer.named_parameters(), twin.named_parameters()):
        assert rel_err(p.grad.cpu(), p64.grad) <= 2e-4, n


def test_dropout_of_the_layer_scales_what_it_keeps():
    torch.manual_seed(6)
    layer = E.DeltaLayer(64, 2, 2, 32, 32, p=0.25).to(DEV)
    x = torch.randn(2, 70, 64, device=DEV)
    with torch.no_grad():
        seed, offset = layer.rng.tolist()
        some = layer(x)[0] - x
        assert layer.rng.tolist() == [seed, offset + 2 * 70 * 64 // 4]
        every = layer.eval()(x)[0] - x
    kept = torch.from_numpy(R.keep_mask(140, 64, seed, offset, 0.25)).to(DEV).view(2, 70, 64)
    want = torch.where(kept, every / 0.75, torch.zeros_like(every))
    assert (some - want).abs().max().item() <= 2e-6 * (1 + x.abs().max().item())


@pytest.mark.parametrize("cut", [1, 20, 37])
def test_served_token_by_token_from_any_cut(cut):
    """Chunks and single tokens are two ways through the recurrence; each holds its values to some 2^-20 of their size."""
    torch.manual_seed(7)
    model = E.Recall(24).to(DEV)
    first, second, _ = E.pairs(5, 24, 20, torch.Generator().manual_seed(1), DEV)
    answers = E.serve(model, first, second, cut)
    with torch.no_grad():
        whole = model(first, second)[0][:, cut:]
    assert rel_err(answers.cpu(), whole.cpu()) <= 2e-5


def test_it_learns():
    torch.manual_seed(8)
    model = E.Recall(8).to(DEV)
    losses = E.train(model, 120, 8, 6)
    assert np.isfinite(losses).all() and np.mean(losses[-10:]) < 0.5 * losses[0]


@pytest.mark.parametrize("bf16", [False, True])
def test_captured_and_replayed(bf16):
    """The calls of a training step in a graph: every replay, with other work and new inputs between, gives what the calls give by themselves."""
    K = E.K
    dt = torch.bfloat16 if bf16 else torch.float32
    B, L, H, Kw, V = 2, 300, 3, 64, 72
    gen = torch.Generator(device=DEV).manual_seed(4)
    new = lambda *s, t=dt: torch.randn(s, generator=gen, device=DEV).to(t)  # noqa: E731
    d = K.make_delta_desc(B, L, H, Kw, V, qk_norm=1, bf16=int(bf16))
    n = K.make_norm_desc(B * L, 1, H * V, H, act=1, bf16=int(bf16))
    p = K.make_dropout_desc(B * L, H * V, p=0.2, bf16=int(bf16))
    q, k, v, do = new(B, L, H, Kw), new(B, L, H, Kw), new(B, L, H, V), new(B, L, H, V)
    decay, beta, w, b = -new(B, L, H, t=torch.float32).abs(), new(B, L, H, t=torch.float32), new(H * V, t=torch.float32), new(H * V, t=torch.float32)
    state, rng = new(B, H, Kw, V, t=torch.float32), torch.tensor([5, 6], device=DEV)
    ck, ws = E._scratch(K.cawn_delta_ckpt_bytes(d), DEV), E._scratch(K.cawn_delta_workspace_bytes(d), DEV)
    nws = E._scratch(K.cawn_group_norm_workspace_bytes(n), DEV)

    def step(out):
        K.check(K.cawn_delta_rule_fwd(d, q, k, v, decay, beta, None, state, out["o"], out["s"], ck, ws))
        K.check(K.cawn_group_norm_fwd(n, out["o"], w, b, out["y"], out["stats"], nws))
        K.check(K.cawn_dropout_add_fwd(p, out["y"], v, rng, out["z"]))
        K.check(K.cawn_dropout_add_bwd(p, do, rng, out["dy"]))
        K.check(K.cawn_group_norm_bwd(n, out["o"], w, b, out["stats"], out["dy"], out["do"], out["dw"], out["db"], nws))
        K.check(K.cawn_delta_rule_bwd(d, q, k, v, decay, beta, None, ck, out["do"], None, out["dq"], out["dk"], out["dv"], out["da"], out["dbeta"],
                                      out["ds"], ws))

    def outputs():
        e = torch.empty_like
        return dict(o=e(v), s=e(state), y=e(v), z=e(v), dy=e(v), do=e(v), stats=torch.empty(B * L, H, 2, device=DEV), dw=e(w), db=e(b), dq=e(q), dk=e(k), dv=e(v),
                    da=e(decay), dbeta=e(beta), ds=e(state))

    kept = outputs()
    step(kept)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(kept)
    for i in range(4):
        q.copy_(new(B, L, H, Kw)), state.mul_(0.5), rng.add_(torch.tensor([0, 1000], device=DEV))
        want = outputs()
        step(want)
        for t in kept.values():
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(kept[x], want[x]) for x in want), (i, [x for x in want if not torch.equal(kept[x], want[x])])
