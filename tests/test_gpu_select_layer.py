"""The example's layer: the norm with the residual addition, the short convolution and the selective scan together, as a program uses them."""
import importlib.util
import os

import numpy as np
import pytest
import torch
import torch.nn.functional as F

from gpu_util import DEV, rel_err

pytestmark = pytest.mark.gpu

_spec = importlib.util.spec_from_file_location("select_layer", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples",
                                                                            "select_layer.py"))
E = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(E)


def _plain(layer, x, residual):
    """The same layer token by token in the type of x."""
    B, L, _ = x.shape
    D, N, G, k = layer.channels, layer.states, layer.groups, layer.taps
    h = x + residual
    y = layer.norm * h / (h.square().mean(-1, keepdim=True) + 1e-5).sqrt()
    u, z = F.linear(y, layer.into.weight).view(B, L, 2, D).unbind(2)
    line = torch.cat([u.new_zeros(B, k - 1, D), u], 1)
    u = F.silu(sum(layer.conv_w[:, i] * line[:, i:i + L] for i in range(k)) + layer.conv_b)
    dt, Bm, Cm = F.linear(u, layer.select.weight).split([layer.rank, G * N, G * N], -1)
    Bm, Cm = (t.reshape(B, L, G, N).repeat_interleave(D // G, 2) for t in (Bm, Cm))
    delta, A = F.softplus(F.linear(dt, layer.steps.weight) + layer.dt_bias), -torch.exp(layer.log_rate)
    S, out = u.new_zeros(B, D, N), []
    for t in range(L):
        S = torch.exp(delta[:, t][..., None] * A) * S + (delta[:, t] * u[:, t])[..., None] * Bm[:, t]
        out.append((Cm[:, t] * S).sum(-1) + layer.skip * u[:, t])
    return F.linear(torch.stack(out, 1) * F.silu(z), layer.out.weight), h


def _layer(seed=5):
    torch.manual_seed(seed)
    return E.SelectLayer(48, 136, 12, groups=2, rank=5)


def test_gradients_of_the_layer():
    """Three fp32 matrix products, the norm, the convolution and the scan stand between a weight and the loss, each good to some 2^-21 of its own size; the
    projections' sums over 136 channels cancel to a tenth of their terms: 2e-4 of a gradient's root mean square is left to a long way from wrong."""
    layer = _layer().to(DEV)
    x, residual = (torch.randn(3, 90, 48, device=DEV, requires_grad=True) for _ in range(2))
    dy, dh = torch.randn(3, 90, 48, device=DEV), torch.randn(3, 90, 48, device=DEV)
    y, h, _ = layer(x, residual)
    torch.autograd.backward([y, h], [dy, dh])
    twin = _layer().double()
    twin.load_state_dict({n: t.cpu() for n, t in layer.state_dict().items()})
    x64, r64 = (t.detach().cpu().double().requires_grad_() for t in (x, residual))
    y64, h64 = _plain(twin, x64, r64)
    torch.autograd.backward([y64, h64], [dy.cpu().double(), dh.cpu().double()])
    for got, want in ((y, y64), (h, h64)):
        assert rel_err(got.detach().cpu(), want.detach()) <= 2e-4
    for got, want in ((x, x64), (residual, r64)):
        assert rel_err(got.grad.cpu(), want.grad) <= 2e-4
    for (n, p), (_, p64) in zip(layer.named_parameters(), twin.named_parameters()):
        assert rel_err(p.grad.cpu(), p64.grad) <= 2e-4, n


def test_a_padded_batch_is_its_rows_by_themselves():
    layer = _layer(6).to(DEV)
    lengths = torch.tensor([70, 0, 1, 33], dtype=torch.int32, device=DEV)
    x, residual = torch.randn(4, 70, 48, device=DEV), torch.randn(4, 70, 48, device=DEV)
    with torch.no_grad():
        y, _, (conv, ssm) = layer(x, residual, lengths=lengths)
        for b, n in enumerate(lengths.tolist()):
            if n == 0:
                assert bool((conv[b] == 0).all()) and bool((ssm[b] == 0).all())
                continue
            one, _, (c1, s1) = layer(x[b:b + 1, :n], residual[b:b + 1, :n])
            assert rel_err(y[b, :n].cpu(), one[0].cpu()) <= 2e-5
            assert rel_err(conv[b].cpu(), c1[0].cpu()) <= 2e-5 and rel_err(ssm[b].cpu(), s1[0].cpu()) <= 2e-5


@pytest.mark.parametrize("cut", [1, 10, 19])
def test_served_token_by_token_from_any_cut(cut):
    """Tiles and single tokens are two ways through the recurrence; each holds its values to some 2^-20 of their size, through two layers."""
    torch.manual_seed(7)
    model = E.Repeat(12).to(DEV)
    ids, _ = E.shown(5, 12, 10, torch.Generator().manual_seed(1), DEV)
    answers = E.serve(model, ids, cut)
    with torch.no_grad():
        whole = model(ids)[0][:, cut:]
    assert rel_err(answers.cpu(), whole.cpu()) <= 4e-5


def test_it_trains():
    torch.manual_seed(8)
    model = E.Repeat(6, layers=1).to(DEV)
    losses = E.train(model, 4, 6, 5, rows=8)
    assert len(losses) == 4 and np.isfinite(losses).all()
    assert all(p.grad is not None and bool(torch.isfinite(p.grad).all()) for p in model.parameters())


def test_other_types_are_refused():
    layer = _layer(9).to(DEV)
    with pytest.raises(TypeError, match="float16"):
        E.AddNorm.apply(torch.ones(4, 48, device=DEV, dtype=torch.float16), torch.ones(4, 48, device=DEV), layer.norm, 1e-5)
    with pytest.raises(TypeError, match="int64"):
        E.ShortConv.apply(torch.ones(1, 4, 8, device=DEV), torch.ones(8, 4, device=DEV), torch.ones(8, device=DEV), torch.ones(1, 3, 8, device=DEV),
                          torch.tensor([4], device=DEV))


@pytest.mark.parametrize("bf16", [False, True])
def test_captured_and_replayed(bf16):
    """The calls of a training step in a graph, with workspaces that they share in their order: every replay, with other work and new inputs between, gives
    what the calls give by themselves."""
    K = E.K
    dt = torch.bfloat16 if bf16 else torch.float32
    B, L, C, N, G = 2, 300, 136, 16, 2
    gen = torch.Generator(device=DEV).manual_seed(4)
    f32 = torch.float32
    new = lambda *s, t=dt: torch.randn(s, generator=gen, device=DEV).to(t)  # noqa: E731
    n = K.make_rms_desc(B * L, C, bf16=int(bf16), residual_bf16=0)
    q = K.make_rms_desc(B * L, C, bf16=int(bf16), residual_bf16=0, block=32)
    c = K.make_conv_desc(B, L, C, 4, act=1, bf16=int(bf16))
    s = K.make_scan_desc(B, L, C, N, G=G, bf16=int(bf16))
    x, z, step, dy, Bm, Cm = new(B, L, C), new(B, L, C), new(B, L, C), new(B, L, C), new(B, L, G, N), new(B, L, G, N)
    res, nw, w, bias, A, skip, dtb = new(B, L, C, t=f32), new(C, t=f32), new(C, 4, t=f32), new(C, t=f32), -new(C, N, t=f32).abs(), new(C, t=f32), new(C, t=f32)
    cs, ss = new(B, 3, C, t=f32), new(B, C, N, t=f32)
    lengths = torch.tensor([300, 171], dtype=torch.int32, device=DEV)
    ck = E._scratch(K.cawn_selective_scan_ckpt_bytes(s), DEV)
    ws = E._scratch(max(K.cawn_selective_scan_workspace_bytes(s), K.cawn_causal_conv_workspace_bytes(c), K.cawn_rms_norm_add_workspace_bytes(n)), DEV)

    def outputs():
        e = torch.empty_like
        o = dict(h=e(res), y=e(x), rstd=torch.empty(B * L, device=DEV), u=e(x), cs=e(cs), v=e(x), ss=e(ss), dv=e(x), dstep=e(x), dA=e(A), dB=e(Bm), dC=e(Cm), dskip=e(skip),
                 dz=e(x), ddtb=e(dtb), dss=e(ss), du=e(x), dw=e(w), dbias=e(bias), dcs=e(cs), dx=e(x), dres=e(res), dnw=e(nw),
                 q8=torch.empty(B * L, C, dtype=torch.float8_e4m3fn, device=DEV), scales=torch.empty(B * L, 5, device=DEV))
        return o

    def run(o):
        K.check(K.cawn_rms_norm_add_fwd(n, x, res, nw, o["h"], o["y"], None, None, o["rstd"]))
        K.check(K.cawn_causal_conv_fwd(c, o["y"], w, bias, lengths, cs, o["u"], o["cs"]))
        K.check(K.cawn_selective_scan_fwd(s, o["u"], step, A, Bm, Cm, skip, z, dtb, lengths, ss, o["v"], o["ss"], ck, ws))
        K.check(K.cawn_rms_norm_add_fwd(q, o["v"], o["h"], nw, None, None, o["q8"], o["scales"], None))
        K.check(K.cawn_selective_scan_bwd(s, o["u"], step, A, Bm, Cm, skip, z, dtb, lengths, ck, dy, None, o["dv"], o["dstep"], o["dA"], o["dB"], o["dC"], o["dskip"],
                                          o["dz"], o["ddtb"], o["dss"], ws))
        K.check(K.cawn_causal_conv_bwd(c, o["y"], w, bias, lengths, cs, o["dv"], None, o["du"], o["dw"], o["dbias"], o["dcs"], ws))
        K.check(K.cawn_rms_norm_add_bwd(n, o["h"], nw, o["rstd"], o["du"], None, o["dx"], o["dres"], o["dnw"], ws))

    def same(a, b):
        return torch.equal(a.view(torch.uint8) if a.dtype == torch.float8_e4m3fn else a, b.view(torch.uint8) if b.dtype == torch.float8_e4m3fn else b)

    kept = outputs()
    run(kept)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(kept)
    for i in range(4):
        x.copy_(new(B, L, C)), ss.mul_(0.5), lengths.copy_(torch.tensor([300 - 40 * i, 31 * i], dtype=torch.int32))
        want = outputs()
        run(want)
        for t in kept.values():
            t.view(torch.uint8).fill_(0xff)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(same(kept[k], want[k]) for k in want), (i, [k for k in want if not same(kept[k], want[k])])
