"""Timing cases of the operators around a second recurrent mixer of the layer: the gated delta rule (prefill, training
step, single tokens), the group norm with an activation behind it, and dropout joined with the residual addition.

    S[t] = exp(decay[t]) (I - beta[t] k[t] k[t]^T) S[t-1] + beta[t] k[t] v[t]^T,   o[t] = scale S[t]^T q[t]

`run` computes a case with elementary torch operations in fp32 (`own` false) or with libcawn's kernels (`own` true);
`exact` computes it again in 64 bits, token by token, from the definition.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
CHUNK = 64          # tokens that the plain form treats at once


def listed():
    return [
        # one token of one stream, 12 heads of 64: what a decoding step of a single user waits for
        dict(name="delta step, one row", op="delta", train=False, B=1, L=1, H=12, Hk=12, K=64, V=64, bf16=True, norm=True, ragged=False),
        # one token of a serving batch, 32 heads of 128, an eighth of the slots without a request
        dict(name="delta step, batch", op="delta", train=False, B=128, L=1, H=32, Hk=32, K=128, V=128, bf16=True, norm=True, ragged=True),
        # one chunk of a streamed prefill of one sequence, fp32, the state carried
        dict(name="delta prefill chunk", op="delta", train=False, B=1, L=4096, H=12, Hk=12, K=64, V=64, bf16=False, norm=True, ragged=False),
        # forward of a layer of 12 heads of 64
        dict(name="delta layer forward", op="delta", train=False, B=4, L=2048, H=12, Hk=12, K=64, V=64, bf16=True, norm=False, ragged=False),
        # long prefill of 32 heads of 128
        dict(name="delta wide prefill", op="delta", train=False, B=2, L=32768, H=32, Hk=32, K=128, V=128, bf16=True, norm=True, ragged=False),
        # training step on a padded batch of short documents: heads that share keys, an odd length, an empty row
        dict(name="delta train, ragged", op="delta", train=True, B=5, L=777, H=4, Hk=2, K=64, V=128, bf16=False, norm=True, ragged=True),
        # training step of a layer, 65,536 tokens
        dict(name="delta train, layer", op="delta", train=True, B=8, L=8192, H=12, Hk=12, K=64, V=64, bf16=True, norm=True, ragged=False),
        # the norm over each head of one token behind a decoding step
        dict(name="norm step", op="norm", train=False, B=1, T=1, C=768, G=12, bf16=True, act=1),
        # the same in a training step: every token's heads are normalised by themselves
        dict(name="norm train, heads", op="norm", train=True, B=65536, T=1, C=768, G=12, bf16=True, act=1),
        # a front-end's norm over whole clips, channels last, with odd lengths
        dict(name="norm train, clips", op="norm", train=True, B=8, T=8191, C=768, G=12, bf16=False, act=2),
        # dropout on a short batch whose rows are no multiple of four
        dict(name="dropout train, short", op="dropout", train=True, rows=1021, cols=97, bf16=False, p=0.1),
        # dropout behind the layer of a training step of 65,536 tokens
        dict(name="dropout train, layer", op="dropout", train=True, rows=65536, cols=768, bf16=True, p=0.1),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["step", "forward", "forward", "train", "train", "norm", "dropout"])
    bf16 = rng.random() < 0.5
    if kind == "norm":
        G = rng.choice([1, 2, 4, 8, 12, 32])
        C = G * rng.choice([16, 24, 30, 64, 128])
        rows = _log(rng, 1, 40_000_000 // C)
        T = 1 if rng.random() < 0.5 else _log(rng, 1, min(rows, 16384))
        return dict(op="norm", train=rng.random() < 0.6, B=max(1, rows // T), T=T, C=C, G=G, bf16=bf16, act=rng.choice([0, 1, 2]))
    if kind == "dropout":
        cols = _log(rng, 1, 8192)
        return dict(op="dropout", train=True, rows=_log(rng, 1, 40_000_000 // cols), cols=cols, bf16=bf16, p=rng.choice([0.05, 0.1, 0.25, 0.5]))
    Hk = rng.choice([1, 2, 4, 8, 12])
    H = Hk * rng.choice([1, 1, 2, 4])
    K, V = rng.choice([16, 32, 64, 64, 96, 128]), rng.choice([16, 40, 64, 64, 128, 256])
    most = {"step": 1 << 27, "forward": 3 << 25, "train": 3 << 24}[kind]       # value elements (a step's: state elements)
    if kind == "step":
        return dict(op="delta", train=False, B=_log(rng, 1, min(512, most // (H * K * V))), L=1, H=H, Hk=Hk, K=K, V=V, bf16=bf16, norm=rng.random() < 0.5, ragged=rng.random() < 0.5)
    L = _log(rng, 2, 16384)
    B = _log(rng, 1, max(1, min(64, most // (L * H * max(K, V)))))
    L = max(2, min(L, most // (B * H * max(K, V))))
    return dict(op="delta", train=kind == "train", B=B, L=L, H=H, Hk=Hk, K=K, V=V, bf16=bf16, norm=rng.random() < 0.5, ragged=rng.random() < 0.3)


def work(case):
    e = 2 if case["bf16"] else 4
    if case["op"] == "dropout":
        n = case["rows"] * case["cols"]
        return {"bytes": n * e * 5, "flops": 3 * n}                      # x, residual -> y; dy -> dx
    if case["op"] == "norm":
        n = case["B"] * case["T"] * case["C"]
        return {"bytes": n * e * (5 if case["train"] else 2) + 8 * case["C"], "flops": (30 if case["train"] else 12) * n}
    B, L, H, Hk, K, V = (case[k] for k in ("B", "L", "H", "Hk", "K", "V"))
    tokens, rows = B * L, B
    if case["ragged"]:
        n = _lengths(case)
        tokens, rows = int(n.sum()), int((n > 0).sum())
    qk, vo, gates, state = 2 * tokens * Hk * K * e, tokens * H * V * e, 2 * tokens * H * 4, rows * H * K * V * 4
    if case["train"]:       # inputs, do, dstate_out in; o, state, gradients of the inputs and of the state out
        return {"bytes": 2 * qk + 4 * vo + 2 * gates + 4 * state, "flops": 21 * tokens * H * K * V}
    return {"bytes": qk + 2 * vo + gates + 2 * state, "flops": 7 * tokens * H * K * V}


def _lengths(case):
    """Tokens of each row: a padded batch with empty rows, rows of one token and full rows; a step's slots are in use or not."""
    B, L = case["B"], case["L"]
    b = np.arange(B)
    if L == 1:
        return (b % 8 != 5).astype(np.int64)
    n = (L * ((b * 37 + 11) % 64 + 1)) // 64
    n[b % 5 == 1] = L
    n[b % 5 == 2] = 0
    n[b % 5 == 3] = np.maximum(n[b % 5 == 3] // 9, 1)
    return n


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt = torch.bfloat16 if case["bf16"] else torch.float32

    def normal(*shape, dtype=dt):
        return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(dtype)

    s = dict(case=case)
    if case["op"] == "dropout":
        shape = (case["rows"], case["cols"])
        s.update(x=normal(*shape), residual=normal(*shape), dy=normal(*shape), rng=torch.tensor([seed * 2654435761 + 17, 1 << 33], device=DEV),
                 y=torch.empty(shape, device=DEV, dtype=dt), dx=torch.empty(shape, device=DEV, dtype=dt))
    elif case["op"] == "norm":
        shape, C = (case["B"], case["T"], case["C"]), case["C"]
        s.update(x=normal(*shape) * 1.7 + 0.3, weight=1 + 0.2 * normal(C, dtype=torch.float32), bias=0.1 * normal(C, dtype=torch.float32),
                 y=torch.empty(shape, device=DEV, dtype=dt))
        if case["train"]:
            s.update(dy=normal(*shape), dx=torch.empty(shape, device=DEV, dtype=dt), dweight=torch.empty(C, device=DEV), dbias=torch.empty(C, device=DEV),
                     stats=torch.empty(case["B"], case["G"], 2, device=DEV))
    else:
        B, L, H, Hk, K, V = (case[k] for k in ("B", "L", "H", "Hk", "K", "V"))
        q, k = normal(B, L, Hk, K, dtype=torch.float32), normal(B, L, Hk, K, dtype=torch.float32)
        if not case["norm"]:        # the projections' own norm came before
            q, k = (t / t.square().sum(-1, keepdim=True).sqrt() for t in (q, k))
        u = torch.rand((B, L, H), generator=gen, device=DEV)
        s.update(q=q.to(dt), k=k.to(dt), v=normal(B, L, H, V), decay=-torch.exp(math.log(1e-3) * (1 - u)), beta=torch.sigmoid(normal(B, L, H, dtype=torch.float32)),
                 state_in=0.3 * normal(B, H, K, V, dtype=torch.float32), lengths=None,
                 o=torch.empty((B, L, H, V), device=DEV, dtype=dt), state_out=torch.empty((B, H, K, V), device=DEV))
        if case["ragged"]:
            s["lengths"] = torch.from_numpy(_lengths(case)).to(torch.int32).to(DEV)
        if case["train"]:
            s.update(do=normal(B, L, H, V), dstate_out=0.1 * normal(B, H, K, V, dtype=torch.float32))
            for n in ("q", "k", "v", "decay", "beta"):
                s["d" + n] = torch.empty_like(s[n])
            s["dstate_in"] = torch.empty_like(s["state_in"])
    if own:
        s["plan"] = _plan(case)
    return s


def _plan(case):
    """Descriptor, checkpoint and workspace, which a program makes once for its sizes."""
    from paper_2604_04250_amd import binding as K
    ck = ws = None
    if case["op"] == "dropout":
        d = K.make_dropout_desc(case["rows"], case["cols"], p=case["p"], bf16=int(case["bf16"]))
    elif case["op"] == "norm":
        d = K.make_norm_desc(case["B"], case["T"], case["C"], case["G"], act=case["act"], bf16=int(case["bf16"]))
        ws = torch.empty(max(1, K.cawn_group_norm_workspace_bytes(d)), dtype=torch.uint8, device=DEV)
    else:
        d = K.make_delta_desc(case["B"], case["L"], case["H"], case["K"], case["V"], Hk=case["Hk"], scale=case["K"] ** -0.5,
                              qk_norm=int(case["norm"]), bf16=int(case["bf16"]))
        ws = torch.empty(max(1, K.cawn_delta_workspace_bytes(d)), dtype=torch.uint8, device=DEV)
        if case["train"]:
            ck = torch.empty(max(1, K.cawn_delta_ckpt_bytes(d)), dtype=torch.uint8, device=DEV)
    return d, ck, ws


def run(s):
    case = s["case"]
    if own:
        return _run_own(case, s)
    return {"delta": _plain_delta, "norm": _plain_norm, "dropout": _plain_dropout}[case["op"]](case, s)


def _run_own(case, s):
    from paper_2604_04250_amd import binding as K
    d, ck, ws = s["plan"]
    if case["op"] == "dropout":
        K.check(K.cawn_dropout_add_fwd(d, s["x"], s["residual"], s["rng"], s["y"]))
        K.check(K.cawn_dropout_add_bwd(d, s["dy"], s["rng"], s["dx"]))
        return {"y": s["y"], "dx": s["dx"]}
    if case["op"] == "norm":
        K.check(K.cawn_group_norm_fwd(d, s["x"], s["weight"], s["bias"], s["y"], s.get("stats"), ws))
        if not case["train"]:
            return {"y": s["y"]}
        K.check(K.cawn_group_norm_bwd(d, s["x"], s["weight"], s["bias"], s["stats"], s["dy"], s["dx"], s["dweight"], s["dbias"], ws))
        return {n: s[n] for n in ("y", "dx", "dweight", "dbias")}
    K.check(K.cawn_delta_rule_fwd(d, s["q"], s["k"], s["v"], s["decay"], s["beta"], s["lengths"], s["state_in"], s["o"], s["state_out"], ck, ws))
    if not case["train"]:
        return {n: s[n] for n in ("o", "state_out")}
    K.check(K.cawn_delta_rule_bwd(d, s["q"], s["k"], s["v"], s["decay"], s["beta"], s["lengths"], ck, s["do"], s["dstate_out"],
                                  s["dq"], s["dk"], s["dv"], s["ddecay"], s["dbeta"], s["dstate_in"], ws))
    return {n: s[n] for n in ("o", "state_out", "dq", "dk", "dv", "ddecay", "dbeta", "dstate_in")}


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _inverse_unit_lower(a):
    """(I + a)^-1 of strictly lower triangular a, from blocks of one doubled to the whole: [[P,0],[C,Q]]^-1 = [[P^-1,0],[-Q^-1 C P^-1, Q^-1]]."""
    n = a.shape[-1]
    t = a.new_ones(*a.shape[:-2], n, 1, 1)                  # inverses of the diagonal blocks
    size = 1
    while size < n:
        m = n // (2 * size)
        blocks = a.reshape(*a.shape[:-2], m, 2 * size, m, 2 * size).diagonal(dim1=-4, dim2=-2).movedim(-1, -3)
        c = blocks[..., size:, :size]
        p, q = t[..., 0::2, :, :], t[..., 1::2, :, :]
        low = -q.contiguous() @ (c.contiguous() @ p.contiguous())
        t = torch.cat([torch.cat([p, torch.zeros_like(p)], -1), torch.cat([low, q], -1)], -2)
        size *= 2
    return t[..., 0, :, :]


def _plain_rule(q, k, v, decay, beta, state, scale, norm):
    """The rule by chunks: q, k [B,L,H,K], v [B,L,H,V], decay, beta [B,L,H] and state [B,H,K,V], all fp32; L a multiple of the chunk, or one token."""
    if norm:
        q, k = (t * torch.rsqrt(t.square().sum(-1, keepdim=True) + 1e-6) for t in (q, k))
    B, L, H, K = q.shape
    if L == 1:
        q, k, v, a, b = q[:, 0], k[:, 0], v[:, 0], decay[:, 0].exp()[..., None, None], beta[:, 0][..., None]
        state = a * state
        u = b * (v - (k[..., None] * state).sum(-2))
        state = state + k[..., None] * u[..., None, :]
        return scale * (q[..., None] * state).sum(-2)[:, None], state
    C = CHUNK
    chunks = lambda t: t.reshape(B, L // C, C, H, -1).permute(1, 0, 3, 2, 4).contiguous()  # noqa: E731
    q, k, v, beta = chunks(q), chunks(k), chunks(v), chunks(beta)
    g = chunks(decay)[..., 0].cumsum(-1)
    lower = torch.ones(C, C, device=q.device, dtype=torch.bool).tril()
    dec = torch.exp((g[..., :, None] - g[..., None, :]).masked_fill(~lower, -math.inf))
    kt = k.transpose(-1, -2).contiguous()
    t = _inverse_unit_lower((beta * dec * (k @ kt)).tril(-1)) * beta.transpose(-1, -2)
    eg = g.exp()[..., None]
    w, ub, p = t @ (eg * k), t @ v, dec * (q @ kt)
    qg, kd = eg * q, (torch.exp(g[..., -1:] - g)[..., None] * k).transpose(-1, -2).contiguous()
    o = []
    for n in range(L // C):
        u = ub[n] - w[n] @ state
        o.append(scale * (qg[n] @ state + p[n] @ u))
        state = eg[n, ..., -1:, :] * state + kd[n] @ u
    return torch.stack(o).permute(1, 0, 3, 2, 4).reshape(B, L, H, -1), state


def _plain_delta(case, s):
    L, H, Hk, dt = case["L"], case["H"], case["Hk"], s["q"].dtype
    x = {n: s[n].float() for n in ("q", "k", "v", "decay", "beta", "state_in")}
    if case["train"]:
        x = {n: t.detach().requires_grad_() for n, t in x.items()}
    q, k, v, decay, beta = (x[n] for n in ("q", "k", "v", "decay", "beta"))
    if s["lengths"] is not None:        # padding leaves the state alone and answers zero
        keep = torch.arange(L, device=DEV)[None, :, None] < s["lengths"][:, None, None]
        q, k, v = (torch.where(keep[..., None], t, 0.0) for t in (q, k, v))
        decay, beta = torch.where(keep, decay, 0.0), torch.where(keep, beta, 0.0)
    pad = -L % CHUNK if L > 1 else 0
    if pad:
        q, k, v, decay, beta = (torch.nn.functional.pad(t, (0, 0) * (t.dim() - 2) + (0, pad)) for t in (q, k, v, decay, beta))
    if H != Hk:
        q, k = (t.repeat_interleave(H // Hk, 2) for t in (q, k))
    o, state = _plain_rule(q, k, v, decay, beta, x["state_in"], case["K"] ** -0.5, case["norm"])
    o = o[:, :L]
    if not case["train"]:
        return {"o": o.to(dt), "state_out": state}
    names = ("q", "k", "v", "decay", "beta", "state_in")
    grads = torch.autograd.grad([o, state], [x[n] for n in names], [s["do"].float(), s["dstate_out"]])
    out = {"o": o.detach().to(dt), "state_out": state.detach()}
    return out | {"d" + n: g.to(s[n].dtype) for n, g in zip(names, grads)}


def _act(z, act):
    if act == 1:
        return z / (1 + torch.exp(-z))
    return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5))) if act == 2 else z


def _plain_norm(case, s):
    B, T, C, G = (case[k] for k in ("B", "T", "C", "G"))
    x, w, b = s["x"].float(), s["weight"], s["bias"]
    xg = x.reshape(B, T, G, C // G)
    mean = xg.mean((1, 3), keepdim=True)
    rstd = torch.rsqrt((xg - mean).square().mean((1, 3), keepdim=True) + 1e-5)
    xh = (xg - mean) * rstd
    z = xh.reshape(B, T, C) * w + b
    y = _act(z, case["act"])
    if not case["train"]:
        return {"y": y.to(s["x"].dtype)}
    dz = s["dy"].float()
    if case["act"] == 1:
        sig = 1 / (1 + torch.exp(-z))
        dz = dz * sig * (1 + z * (1 - sig))
    elif case["act"] == 2:
        dz = dz * (0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi))
    flat = xh.reshape(B, T, C)
    dxh = (dz * w).reshape(B, T, G, C // G)
    dx = rstd * (dxh - dxh.mean((1, 3), keepdim=True) - xh * (dxh * xh).mean((1, 3), keepdim=True))
    return {"y": y.to(s["x"].dtype), "dx": dx.reshape(B, T, C).to(s["x"].dtype), "dweight": (dz * flat).sum((0, 1)), "dbias": dz.sum((0, 1))}


def _mul32(a, m):
    """High and low 32 bits of the product of 32-bit numbers held in 64."""
    p, q = (m & 0xffff) * a, (m >> 16) * a
    return (q + (p >> 16)) >> 16, ((q << 16) + p) & 0xffffffff


def _plain_keep(rows, cols, rng, p):
    """Philox-4x32-10 (Salmon et al. 2011): element e takes word e % 4 of block offset + e // 4 under the 64-bit seed."""
    n = rows * cols
    block = torch.arange((n + 3) // 4, device=rng.device) + rng[1]
    c = [block & 0xffffffff, (block >> 32) & 0xffffffff, torch.zeros_like(block), torch.zeros_like(block)]
    k0, k1 = rng[0] & 0xffffffff, (rng[0] >> 32) & 0xffffffff
    for _ in range(10):
        h0, l0 = _mul32(c[0], 0xD2511F53)
        h1, l1 = _mul32(c[2], 0xCD9E8D57)
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    return (torch.stack(c, 1).reshape(-1)[:n] >= int(p * 4294967296.0)).reshape(rows, cols)


def _plain_dropout(case, s):
    p, dt = case["p"], s["x"].dtype
    keep = _plain_keep(case["rows"], case["cols"], s["rng"], p)
    scale = 1.0 / (1.0 - p)
    y = s["residual"].float() + torch.where(keep, s["x"].float() * scale, 0.0)
    return {"y": y.to(dt), "dx": torch.where(keep, s["dy"].float() * scale, 0.0).to(dt)}


# ---- 64 bits, from the definitions ------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "dropout":
        return _exact_dropout(case, s)
    return _exact_norm(case, s) if case["op"] == "norm" else _exact_delta(case, s)


def _exact_dropout(case, s):
    n = case["rows"] * case["cols"]
    seed, offset = (int(v) & 0xffffffffffffffff for v in s["rng"].tolist())
    at = (np.arange((n + 3) // 4, dtype=np.uint64) + np.uint64(offset))
    low = np.uint64(0xffffffff)
    x0, x1, x2, x3 = at & low, at >> np.uint64(32), np.uint64(0) * at, np.uint64(0) * at
    k0, k1 = seed & 0xffffffff, seed >> 32
    for r in range(10):
        a, b = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
        x0, x1, x2, x3 = (b >> np.uint64(32)) ^ x1 ^ np.uint64((k0 + r * 0x9E3779B9) & 0xffffffff), b & low, (a >> np.uint64(32)) ^ x3 ^ np.uint64((k1 + r * 0xBB67AE85) & 0xffffffff), a & low
    word = np.stack([x0, x1, x2, x3], 1).reshape(-1)[:n]
    keep = torch.from_numpy((word >= np.uint64(math.floor(case["p"] * 2.0 ** 32))).reshape(case["rows"], case["cols"])).to(DEV).double()
    m = keep / (1 - case["p"])
    return {"y": s["residual"].double() + s["x"].double() * m, "dx": s["dy"].double() * m}


def _exact_norm(case, s):
    B, T, C, G = (case[k] for k in ("B", "T", "C", "G"))
    x, w, b = s["x"].double().reshape(B, T, G, -1), s["weight"].double().reshape(G, -1), s["bias"].double().reshape(G, -1)
    var, mean = torch.var_mean(x, (1, 3), correction=0, keepdim=True)
    sd = (var + 1e-5).sqrt()
    h = (x - mean) / sd
    z = h * w + b
    if case["act"] == 1:
        f = torch.sigmoid(z)
        y, slope = z * f, f + z * f * (1 - f)
    elif case["act"] == 2:
        f = 0.5 * torch.erfc(-z / math.sqrt(2))
        y, slope = z * f, f + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    else:
        y, slope = z, torch.ones_like(z)
    if not case["train"]:
        return {"y": y.reshape(B, T, C)}
    dz = s["dy"].double().reshape(B, T, G, -1) * slope
    t = dz * w
    n = T * (C // G)
    dx = (t - t.sum((1, 3), keepdim=True) / n - h * (t * h).sum((1, 3), keepdim=True) / n) / sd
    return {"y": y.reshape(B, T, C), "dx": dx.reshape(B, T, C), "dweight": (dz * h).sum((0, 1)).reshape(C), "dbias": dz.sum((0, 1)).reshape(C)}


def _exact_delta(case, s):
    """Token by token; gradients by the adjoint recurrence, with the states of one run of tokens kept at a time."""
    L, H, Hk, K, scale = case["L"], case["H"], case["Hk"], case["K"], case["K"] ** -0.5
    if L * (4 if case["train"] else 1) > 40000:
        return None
    q0, k0 = s["q"].double(), s["k"].double()
    rq, rk = ((t.square().sum(-1, keepdim=True) + 1e-6).rsqrt() if case["norm"] else torch.ones_like(t[..., :1]) for t in (q0, k0))
    q, k = ((t * r).repeat_interleave(H // Hk, 2) for t, r in ((q0, rq), (k0, rk)))
    v, alpha, beta = s["v"].double(), s["decay"].double().exp(), s["beta"].double()
    n = s["lengths"]
    live = torch.ones(q.shape[0], L, device=DEV, dtype=torch.float64) if n is None else (torch.arange(L, device=DEV) < n[:, None]).double()
    alpha = 1 - live[..., None] * (1 - alpha)
    k, q, v, beta = k * live[..., None, None], q * live[..., None, None], v * live[..., None, None], beta * live[..., None]
    # time first, so that a token's rows lie together
    q, k, v, alpha, beta = (t.movedim(1, 0).contiguous() for t in (q, k, v, alpha, beta))

    def token(S, t):
        decayed = alpha[t][..., None, None] * S
        e = v[t] - (k[t][..., None] * decayed).sum(-2)
        return decayed, e, decayed + k[t][..., None] * (beta[t][..., None] * e)[..., None, :]

    S, o, held = s["state_in"].double(), torch.empty_like(v), []
    for t in range(L):
        if case["train"] and t % 64 == 0:
            held.append(S)
        S = token(S, t)[2]
        o[t] = scale * (q[t][..., None] * S).sum(-2)
    out = {"o": o.movedim(0, 1), "state_out": S}
    if not case["train"]:
        return out
    do = s["do"].double() * live[..., None, None]
    do = do.movedim(1, 0).contiguous()
    dq, dk, dv, da, db = (torch.empty_like(t) for t in (q, k, v, alpha, beta))
    D = s["dstate_out"].double()
    for c in reversed(range(len(held))):
        S, run_ = held[c], []
        for t in range(64 * c, min(L, 64 * c + 64)):
            decayed, e, after = token(S, t)
            run_.append((decayed, e, after))
            S = after
        for t in reversed(range(64 * c, 64 * c + len(run_))):
            decayed, e, after = run_[t - 64 * c]
            dq[t] = scale * (after * do[t][..., None, :]).sum(-1)
            D = D + scale * q[t][..., None] * do[t][..., None, :]
            du = (k[t][..., None] * D).sum(-2)
            db[t] = (du * e).sum(-1)
            de = beta[t][..., None] * du
            dv[t] = de
            dk[t] = (D * (beta[t][..., None] * e)[..., None, :] - decayed * de[..., None, :]).sum(-1)
            D = D - k[t][..., None] * de[..., None, :]
            da[t] = (D * decayed).sum((-2, -1))
            D = alpha[t][..., None, None] * D
    back = lambda t: t.movedim(0, 1)  # noqa: E731
    grads = []
    for x, r, dxh in ((q0, rq, back(dq)), (k0, rk, back(dk))):
        dxh = dxh * live[..., None, None]
        dxh = dxh.reshape(*x.shape[:2], Hk, H // Hk, K).sum(3)
        if case["norm"]:
            xh = x * r
            dxh = r * (dxh - xh * (xh * dxh).sum(-1, keepdim=True))
        grads.append(dxh)
    m = live[..., None]
    return out | {"dq": grads[0], "dk": grads[1], "dv": back(dv) * m[..., None], "ddecay": back(da) * m, "dbeta": back(db) * m, "dstate_in": D}
