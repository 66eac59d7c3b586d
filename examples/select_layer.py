"""A layer of the selective state space scan, trained and served through the library's entry points.

The layer: the norm of the residual stream with the last layer's output added to it; a projection gives x and the gate z; x goes through the short causal
convolution; projections of it give the steps dt, B and C; the scan mixes along the tokens; a projection.  The norm, the convolution and the scan are the
library's, forward and backward; the projections are torch's.

    python examples/select_layer.py          # on an MI355X: learns to repeat what was shown, then answers token by token

The task: a sequence shows symbols and then asks for them again, in their order.
"""
from __future__ import annotations

import math
import os
import sys

import torch
import torch.nn.functional as F
from torch.autograd.function import once_differentiable

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2604_04250_amd import binding as K  # noqa: E402


def _scratch(nbytes, device):
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def _types(wanted, **tensors):
    """The entry points take pointers: what a tensor holds has to be checked before."""
    for name, t in tensors.items():
        if t is not None and t.dtype != wanted:
            raise TypeError(f"{name} is {t.dtype}, not {wanted}")


def _shapes(**wanted):
    """... and how much of it there is: name = (tensor, shape)."""
    for name, (t, shape) in wanted.items():
        if t is not None and tuple(t.shape) != shape:
            raise ValueError(f"{name} is {list(t.shape)}, not {list(shape)}")


def _activation(t):
    return torch.bfloat16 if t.dtype == torch.bfloat16 else torch.float32


class AddNorm(torch.autograd.Function):
    """x [rows,C], residual [rows,C] -> the residual stream h = x + residual, and weight h / rms(h)."""

    @staticmethod
    def forward(ctx, x, residual, weight, eps):
        _types(_activation(x), x=x)
        _types(_activation(residual), residual=residual)
        _types(torch.float32, weight=weight)
        _shapes(residual=(residual, tuple(x.shape)), weight=(weight, (x.shape[-1],)))
        x, residual, weight = x.contiguous(), residual.contiguous(), weight.contiguous()
        d = K.make_rms_desc(*x.shape, eps=eps, bf16=int(x.dtype == torch.bfloat16), residual_bf16=int(residual.dtype == torch.bfloat16))
        h, y, rstd = torch.empty_like(residual), torch.empty_like(x), torch.empty(x.shape[0], device=x.device)
        K.check(K.cawn_rms_norm_add_fwd(d, x, residual, weight, h, y, None, None, rstd))
        ctx.d = d
        ctx.save_for_backward(h, weight, rstd)
        return h, y

    @staticmethod
    @once_differentiable
    def backward(ctx, dh, dy):
        h, weight, rstd = ctx.saved_tensors
        dx, dres, dw = torch.empty_like(dy, memory_format=torch.contiguous_format), torch.empty_like(h), torch.empty_like(weight)
        K.check(K.cawn_rms_norm_add_bwd(ctx.d, h, weight, rstd, dy.contiguous(), dh.contiguous(), dx, dres, dw,
                                        _scratch(K.cawn_rms_norm_add_workspace_bytes(ctx.d), h.device)))
        return dx, dres, dw, None


class ShortConv(torch.autograd.Function):
    """x [B,L,C], w [C,k], bias [C], state [B,k-1,C] fp32 -> SiLU of the convolution, the state behind the last token."""

    @staticmethod
    def forward(ctx, x, w, bias, state, lengths):
        _types(_activation(x), x=x)
        _types(torch.float32, w=w, bias=bias, state=state)
        _types(torch.int32, lengths=lengths)
        (B, _, C), k = x.shape, w.shape[1]
        _shapes(w=(w, (C, k)), bias=(bias, (C,)), state=(state, (B, k - 1, C)), lengths=(lengths, (B,)))
        x, w, bias, state = (t.contiguous() for t in (x, w, bias, state))
        lengths = None if lengths is None else lengths.contiguous()
        d = K.make_conv_desc(*x.shape, k, act=1, bf16=int(x.dtype == torch.bfloat16))
        y, out = torch.empty_like(x), torch.empty_like(state)
        K.check(K.cawn_causal_conv_fwd(d, x, w, bias, lengths, state, y, out))
        ctx.d = d
        ctx.save_for_backward(x, w, bias, state, lengths)
        return y, out

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dout):
        x, w, bias, state, lengths = ctx.saved_tensors
        dx, dw, db, dstate = (torch.empty_like(t) for t in (x, w, bias, state))
        K.check(K.cawn_causal_conv_bwd(ctx.d, x, w, bias, lengths, state, dy.contiguous(), dout.contiguous(), dx, dw, db, dstate,
                                       _scratch(K.cawn_causal_conv_workspace_bytes(ctx.d), x.device)))
        return dx, dw, db, dstate, None


class SelectiveScan(torch.autograd.Function):
    """x, dt, z [B,L,D], A [D,N], Bm, Cm [B,L,G,N], skip, dt_bias [D], state [B,D,N] fp32 -> y [B,L,D], the state behind the last token.

    grad: the caller's torch.is_grad_enabled(), which is off inside; a parameter needs its gradient whether or not.  Without a backward to come there is
    no checkpoint, and calls of a few tokens go token by token."""

    @staticmethod
    def forward(ctx, x, dt, A, Bm, Cm, skip, z, dt_bias, state, lengths, grad=True):
        _types(_activation(x), x=x, dt=dt, Bm=Bm, Cm=Cm, z=z)
        _types(torch.float32, A=A, skip=skip, dt_bias=dt_bias, state=state)
        _types(torch.int32, lengths=lengths)
        (B, L, D), N, G = x.shape, A.shape[1], Bm.shape[2]
        _shapes(dt=(dt, (B, L, D)), z=(z, (B, L, D)), A=(A, (D, N)), Bm=(Bm, (B, L, G, N)), Cm=(Cm, (B, L, G, N)), skip=(skip, (D,)),
                dt_bias=(dt_bias, (D,)), state=(state, (B, D, N)), lengths=(lengths, (B,)))
        x, dt, A, Bm, Cm, skip, z, dt_bias, state = (t.contiguous() for t in (x, dt, A, Bm, Cm, skip, z, dt_bias, state))
        lengths = None if lengths is None else lengths.contiguous()
        d = K.make_scan_desc(B, L, D, N, G=G, dt_softplus=1, bf16=int(x.dtype == torch.bfloat16))
        ckpt = _scratch(K.cawn_selective_scan_ckpt_bytes(d), x.device) if grad and any(ctx.needs_input_grad) else None
        size = K.cawn_selective_scan_serve_workspace_bytes if ckpt is None else K.cawn_selective_scan_workspace_bytes
        y, out = torch.empty_like(x), torch.empty_like(state)
        K.check(K.cawn_selective_scan_fwd(d, x, dt, A, Bm, Cm, skip, z, dt_bias, lengths, state, y, out, ckpt, _scratch(size(d), x.device)))
        ctx.d, ctx.ckpt = d, ckpt
        ctx.save_for_backward(x, dt, A, Bm, Cm, skip, z, dt_bias, lengths)
        return y, out

    @staticmethod
    @once_differentiable
    def backward(ctx, dy, dout):
        *saved, lengths = ctx.saved_tensors
        x, dt, A, Bm, Cm, skip, z, dt_bias = saved
        dx, ddt, dA, dB, dC, dskip, dz, dbias = (torch.empty_like(t) for t in saved)
        dstate = torch.empty_like(dout, memory_format=torch.contiguous_format)
        K.check(K.cawn_selective_scan_bwd(ctx.d, x, dt, A, Bm, Cm, skip, z, dt_bias, lengths, ctx.ckpt, dy.contiguous(), dout.contiguous(), dx, ddt, dA,
                                          dB, dC, dskip, dz, dbias, dstate, _scratch(K.cawn_selective_scan_workspace_bytes(ctx.d), x.device)))
        return dx, ddt, dA, dB, dC, dskip, dz, dbias, dstate, None, None


class SelectLayer(torch.nn.Module):
    def __init__(self, width, channels, states, groups=1, rank=8, taps=4):
        super().__init__()
        self.channels, self.states, self.groups, self.rank, self.taps = channels, states, groups, rank, taps
        self.norm = torch.nn.Parameter(torch.ones(width))
        self.into = torch.nn.Linear(width, 2 * channels, bias=False)
        self.conv_w = torch.nn.Parameter(torch.randn(channels, taps) / math.sqrt(taps))
        self.conv_b = torch.nn.Parameter(torch.zeros(channels))
        self.select = torch.nn.Linear(channels, rank + 2 * groups * states, bias=False)
        self.steps = torch.nn.Linear(rank, channels, bias=False)
        step = torch.exp(torch.empty(channels).uniform_(math.log(1e-3), math.log(1e-1)))
        self.dt_bias = torch.nn.Parameter(step + torch.log(-torch.expm1(-step)))          # what softplus makes the step of
        self.log_rate = torch.nn.Parameter(torch.log(torch.arange(1, states + 1, dtype=torch.float32)).repeat(channels, 1))
        self.skip = torch.nn.Parameter(torch.ones(channels))
        self.out = torch.nn.Linear(channels, width, bias=False)

    def empty_state(self, rows):
        new = lambda *shape: torch.zeros(shape, device=self.norm.device)  # noqa: E731
        return new(rows, self.taps - 1, self.channels), new(rows, self.channels, self.states)

    def forward(self, x, residual, state=None, lengths=None):
        """x [B,L,width], what is to be added to the residual stream -> the layer's own, the stream, and the states to go on from."""
        B, L, width = x.shape
        conv, ssm = self.empty_state(B) if state is None else state
        h, y = AddNorm.apply(x.reshape(B * L, width), residual.reshape(B * L, width), self.norm, 1e-5)
        u, z = self.into(y).view(B, L, 2, self.channels).unbind(2)
        u, conv = ShortConv.apply(u, self.conv_w, self.conv_b, conv, lengths)
        dt, Bm, Cm = self.select(u).split([self.rank, self.groups * self.states, self.groups * self.states], -1)
        Bm, Cm = (t.reshape(B, L, self.groups, self.states) for t in (Bm, Cm))
        u, ssm = SelectiveScan.apply(u, self.steps(dt), -torch.exp(self.log_rate), Bm, Cm, self.skip, z, self.dt_bias, ssm, lengths,
                                     torch.is_grad_enabled())
        return self.out(u), h.view(B, L, width), (conv, ssm)


class Repeat(torch.nn.Module):
    """Symbols, then a sign for each of them: they are to be named again."""

    def __init__(self, symbols, width=64, layers=2, channels=128, states=16):
        super().__init__()
        self.embed = torch.nn.Embedding(symbols + 1, width)
        self.layers = torch.nn.ModuleList(SelectLayer(width, channels, states) for _ in range(layers))
        self.norm = torch.nn.Parameter(torch.ones(width))
        self.head = torch.nn.Linear(width, symbols)

    def forward(self, ids, states=None):
        x = self.embed(ids)
        residual, kept = torch.zeros_like(x), []
        for i, layer in enumerate(self.layers):
            x, residual, s = layer(x, residual, None if states is None else states[i])
            kept.append(s)
        rows = x.shape[0] * x.shape[1]
        _, y = AddNorm.apply(x.reshape(rows, -1), residual.reshape(rows, -1), self.norm, 1e-5)
        return self.head(y.view_as(x)), kept


def shown(rows, symbols, n, gen, device):
    first = torch.randint(symbols, (rows, n), generator=gen)
    return torch.cat([first, torch.full_like(first, symbols)], 1).to(device), first.to(device)


def train(model, steps, symbols, n, rows=64, lr=3e-3, seed=3):
    gen = torch.Generator().manual_seed(seed)
    opt = torch.optim.AdamW(model.parameters(), lr=lr, weight_decay=0.0)
    losses = []
    for _ in range(steps):
        ids, answer = shown(rows, symbols, n, gen, model.norm.device)
        logits, _ = model(ids)
        loss = F.cross_entropy(logits[:, n:].float().reshape(-1, symbols), answer.reshape(-1))
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(loss.detach())
    return torch.stack(losses).tolist()


@torch.no_grad()
def serve(model, ids, n):
    """The first n tokens at once, then one at a time from the states they left."""
    _, states = model(ids[:, :n])
    answers = []
    for t in range(n, ids.shape[1]):
        logits, states = model(ids[:, t:t + 1], states)
        answers.append(logits)
    return torch.cat(answers, 1)


def main():
    torch.manual_seed(0)
    symbols, n = 12, 10
    model = Repeat(symbols).to("cuda:0")
    losses = train(model, 400, symbols, n)
    ids, answer = shown(64, symbols, n, torch.Generator().manual_seed(99), "cuda:0")
    answers = serve(model, ids, n)
    with torch.no_grad():
        whole = model(ids)[0][:, n:]
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f}; repeated token by token {(answers.argmax(-1) == answer).float().mean().item():.3f} "
          f"of the symbols; largest difference from the whole sequence at once {(answers - whole).abs().max().item():.1e}")


if __name__ == "__main__":
    main()
