"""A layer of the gated delta rule, trained and served through the library's entry points.

The layer: projections of x give q, k, v, a decay and a beta per head; the gated delta rule mixes along the tokens; a norm over each
head with SiLU behind it; a projection; dropout joined with the residual addition.  The mixer, the norm and the dropout are the
library's, forward and backward; the projections are torch's.

    python examples/delta_layer.py          # on an MI355X: learns to recall pairs, then answers token by token

The task: a sequence shows pairs of symbols and then asks for the second of each by the first.
"""
from __future__ import annotations

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


class DeltaRule(torch.autograd.Function):
    """q, k [B,L,Hk,K], v [B,L,H,V], decay, beta [B,L,H] fp32, state [B,H,K,V] fp32 -> o [B,L,H,V], state behind the last token."""

    @staticmethod
    def forward(ctx, q, k, v, decay, beta, state, lengths):
        B, L, H, V = v.shape
        Hk, Kw = k.shape[2:]
        _types(torch.bfloat16 if v.dtype == torch.bfloat16 else torch.float32, q=q, k=k, v=v)
        _types(torch.float32, decay=decay, beta=beta, state=state)
        _types(torch.int32, lengths=lengths)
        _shapes(q=(q, (B, L, Hk, Kw)), k=(k, (B, L, Hk, Kw)), decay=(decay, (B, L, H)), beta=(beta, (B, L, H)), state=(state, (B, H, Kw, V)),
                lengths=(lengths, (B,)))
        d = K.make_delta_desc(B, L, H, Kw, V, Hk=Hk, scale=Kw ** -0.5, qk_norm=1, bf16=int(v.dtype == torch.bfloat16))
        q, k, v, decay, beta, state = (t.contiguous() for t in (q, k, v, decay, beta, state))
        lengths = None if lengths is None else lengths.contiguous()
        train = any(ctx.needs_input_grad)
        ckpt = _scratch(K.cawn_delta_ckpt_bytes(d), v.device) if train else None
        workspace = _scratch(K.cawn_delta_workspace_bytes(d), v.device)
        o, state_out = torch.empty_like(v), torch.empty((B, H, Kw, V), device=v.device)
        K.check(K.cawn_delta_rule_fwd(d, q, k, v, decay, beta, lengths, state, o, state_out, ckpt, workspace))
        ctx.d, ctx.ckpt, ctx.workspace = d, ckpt, workspace
        ctx.save_for_backward(q, k, v, decay, beta, lengths)
        return o, state_out

    @staticmethod
    @once_differentiable
    def backward(ctx, do, dstate_out):
        q, k, v, decay, beta, lengths = ctx.saved_tensors
        do, dstate_out = do.contiguous(), dstate_out.contiguous()
        dq, dk, dv, ddecay, dbeta = (torch.empty_like(t) for t in (q, k, v, decay, beta))
        dstate = torch.empty_like(dstate_out) if ctx.needs_input_grad[5] else None
        K.check(K.cawn_delta_rule_bwd(ctx.d, q, k, v, decay, beta, lengths, ctx.ckpt, do, dstate_out, dq, dk, dv, ddecay,
                                      dbeta, dstate, ctx.workspace))
        return dq, dk, dv, ddecay, dbeta, dstate, None


class HeadNorm(torch.autograd.Function):
    """SiLU(norm(x) weight + bias) of [tokens, C], every token's `groups` heads by themselves; weight and bias of any type, taken in fp32."""

    @staticmethod
    def forward(ctx, x, weight, bias, groups):
        _types(torch.bfloat16 if x.dtype == torch.bfloat16 else torch.float32, x=x)
        _shapes(weight=(weight, (x.shape[-1],)), bias=(bias, (x.shape[-1],)))
        ctx.types = weight.dtype, bias.dtype
        x, weight, bias = x.contiguous(), weight.float().contiguous(), bias.float().contiguous()
        d = K.make_norm_desc(x.shape[0], 1, x.shape[1], groups, act=1, bf16=int(x.dtype == torch.bfloat16))
        y, stats = torch.empty_like(x), torch.empty((x.shape[0], groups, 2), device=x.device)
        workspace = _scratch(K.cawn_group_norm_workspace_bytes(d), x.device)
        K.check(K.cawn_group_norm_fwd(d, x, weight, bias, y, stats, workspace))
        ctx.d, ctx.workspace = d, workspace
        ctx.save_for_backward(x, weight, bias, stats)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x, weight, bias, stats = ctx.saved_tensors
        dx, dw, db = torch.empty_like(x), torch.empty_like(weight), torch.empty_like(bias)
        K.check(K.cawn_group_norm_bwd(ctx.d, x, weight, bias, stats, dy.contiguous(), dx, dw, db, ctx.workspace))
        return dx, dw.to(ctx.types[0]), db.to(ctx.types[1]), None


class DropoutAdd(torch.autograd.Function):
    """residual + dropout(x) of [rows, cols]; rng: int64 {seed, offset} on the device, from which the backward makes the mask again."""

    @staticmethod
    def forward(ctx, x, residual, rng, p):
        _types(torch.bfloat16 if x.dtype == torch.bfloat16 else torch.float32, x=x, residual=residual)
        _types(torch.int64, rng=rng)
        _shapes(residual=(residual, tuple(x.shape)), rng=(rng, (2,)))
        d = K.make_dropout_desc(*x.shape, p=p, bf16=int(x.dtype == torch.bfloat16))
        x, residual = x.contiguous(), residual.contiguous()
        y = torch.empty_like(x)
        K.check(K.cawn_dropout_add_fwd(d, x, residual, rng, y))
        ctx.d = d
        ctx.save_for_backward(rng)
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        rng, = ctx.saved_tensors
        dy = dy.contiguous()
        dx = torch.empty_like(dy)
        K.check(K.cawn_dropout_add_bwd(ctx.d, dy, rng, dx))
        return dx, dy, None, None


class DeltaLayer(torch.nn.Module):
    def __init__(self, width, heads, key_heads, key, value, p=0.1, seed=1):
        super().__init__()
        self.heads, self.key_heads, self.key, self.value, self.p = heads, key_heads, key, value, p
        self.qk = torch.nn.Linear(width, 2 * key_heads * key, bias=False)
        self.v = torch.nn.Linear(width, heads * value, bias=False)
        self.gates = torch.nn.Linear(width, 2 * heads)
        self.out = torch.nn.Linear(heads * value, width, bias=False)
        self.norm_w, self.norm_b = torch.nn.Parameter(torch.ones(heads * value)), torch.nn.Parameter(torch.zeros(heads * value))
        self.register_buffer("rng", torch.tensor([seed, 0], dtype=torch.int64))
        torch.nn.init.constant_(self.gates.bias[:heads].data, -4.0)        # little is forgotten at first

    def empty_state(self, rows):
        return torch.zeros((rows, self.heads, self.key, self.value), device=self.norm_w.device)

    def forward(self, x, state=None, lengths=None):
        """x [B,L,width] -> the same, and the state to go on from."""
        B, L, width = x.shape
        q, k = self.qk(x).view(B, L, 2, self.key_heads, self.key).unbind(2)
        v = self.v(x).view(B, L, self.heads, self.value)
        forget, beta = self.gates(x).float().view(B, L, 2, self.heads).unbind(2)
        o, state = DeltaRule.apply(q, k, v, -F.softplus(forget), torch.sigmoid(beta), self.empty_state(B) if state is None else state, lengths)
        o = HeadNorm.apply(o.view(B * L, -1), self.norm_w, self.norm_b, self.heads)
        y, residual = self.out(o), x.reshape(B * L, width)
        rng = self.rng.clone()
        self.rng[1] += (y.numel() + 3) // 4                                 # blocks of four elements: the next call's are others
        y = DropoutAdd.apply(y, residual, rng, self.p if self.training else 0.0)
        return y.view(B, L, width), state


class Recall(torch.nn.Module):
    """Pairs (first, second), then firsts alone: the seconds are to be named."""

    def __init__(self, symbols, width=64, heads=4, key_heads=2, key=32, value=32):
        super().__init__()
        self.first, self.second = torch.nn.Embedding(symbols, width), torch.nn.Embedding(symbols + 1, width)
        self.layer = DeltaLayer(width, heads, key_heads, key, value)
        self.head = torch.nn.Linear(width, symbols)

    def forward(self, first, second, state=None):
        y, state = self.layer(self.first(first) + self.second(second), state)
        return self.head(y), state


def pairs(rows, symbols, n, gen, device):
    first = torch.stack([torch.randperm(symbols, generator=gen)[:n] for _ in range(rows)])
    second = torch.randint(symbols, (rows, n), generator=gen)
    order = torch.stack([torch.randperm(n, generator=gen) for _ in range(rows)])
    asked = torch.gather(first, 1, order)
    return (torch.cat([first, asked], 1).to(device), torch.cat([second, torch.full_like(asked, symbols)], 1).to(device),
            torch.gather(second, 1, order).to(device))


def train(model, steps, symbols, n, rows=64, lr=4e-3, seed=3):
    gen = torch.Generator().manual_seed(seed)
    opt = torch.optim.AdamW(model.parameters(), lr=lr, weight_decay=0.0)
    model.train()
    losses = []
    for _ in range(steps):
        first, second, answer = pairs(rows, symbols, n, gen, model.head.weight.device)
        logits, _ = model(first, second)
        loss = F.cross_entropy(logits[:, n:].float().reshape(-1, symbols), answer.reshape(-1))
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        losses.append(loss.detach())
    return torch.stack(losses).tolist()


@torch.no_grad()
def serve(model, first, second, n):
    """The pairs at once, then one question at a time from the state they left."""
    model.eval()
    _, state = model(first[:, :n], second[:, :n])
    answers = []
    for t in range(n, first.shape[1]):
        logits, state = model(first[:, t:t + 1], second[:, t:t + 1], state)
        answers.append(logits)
    return torch.cat(answers, 1)


def main():
    torch.manual_seed(0)
    symbols, n = 24, 20
    model = Recall(symbols).to("cuda:0")
    losses = train(model, 300, symbols, n)
    first, second, answer = pairs(64, symbols, n, torch.Generator().manual_seed(99), "cuda:0")
    answers = serve(model, first, second, n)
    with torch.no_grad():
        whole = model(first, second)[0][:, n:]
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.3f}; recalled token by token {(answers.argmax(-1) == answer).float().mean().item():.3f} "
          f"of the pairs; largest difference from the whole sequence at once {(answers - whole).abs().max().item():.1e}")


if __name__ == "__main__":
    main()
