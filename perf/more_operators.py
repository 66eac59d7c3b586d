"""Timing cases of the operators of a selective state space layer: the scan itself (prefill, training step, single tokens), its short
causal convolution, and the root-mean-square norm joined with the residual addition, its output in 8 bits with scales among them.

    S[t] = exp(delta[t] A) S[t-1] + delta[t] x[t] B[t],   y[t] = (C[t] . S[t] + D x[t]) SiLU(z[t]),   delta = softplus(dt + dt_bias)

`run` computes a case with elementary torch operations in fp32 (`own` false) or with libcawn's kernels (`own` true);
`exact` computes it again in 64 bits from the definition, the scan token by token.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
CHUNK = 64          # tokens that the plain form of the scan treats at once
E4M3 = torch.float8_e4m3fn


def listed():
    return [
        # one token of one stream, 768 channels of 16 states: what a decoding step of a single user waits for
        dict(name="scan step, one row", op="scan", train=False, B=1, L=1, D=768, N=16, G=1, bf16=True, z=True, ragged=False),
        # one token of a serving batch of 4,096 channels, an eighth of the slots without a request
        dict(name="scan step, batch", op="scan", train=False, B=128, L=1, D=4096, N=16, G=1, bf16=True, z=True, ragged=True),
        # one chunk of a streamed prefill of one sequence, fp32, the state carried
        dict(name="scan prefill chunk", op="scan", train=False, B=1, L=4096, D=768, N=16, G=1, bf16=False, z=True, ragged=False),
        # long prefill of two sequences, 4,096 channels
        dict(name="scan wide prefill", op="scan", train=False, B=2, L=32768, D=4096, N=16, G=1, bf16=True, z=True, ragged=False),
        # training step on a padded batch of short documents: an odd length, two groups of 164 channels, 24 states, no gate, an empty row
        dict(name="scan train, ragged", op="scan", train=True, B=5, L=777, D=328, N=24, G=2, bf16=False, z=False, ragged=True),
        # training step of a layer, 65,536 tokens
        dict(name="scan train, layer", op="scan", train=True, B=8, L=8192, D=768, N=16, G=1, bf16=True, z=True, ragged=False),
        # the convolution of one token of a serving batch
        dict(name="conv step, batch", op="conv", train=False, B=128, L=1, C=4096, k=4, bf16=True, act=1, ragged=True),
        # its training step, 65,536 tokens
        dict(name="conv train, layer", op="conv", train=True, B=8, L=8192, C=768, k=4, bf16=True, act=1, ragged=False),
        # the norm before a product in 8 bits: one scale for each of 4 decoded rows
        dict(name="norm step, 8 bits", op="rms", train=False, rows=4, C=768, bf16=True, res_bf16=True, block=0, quant=True),
        # the same for a long prefill, a scale for every 128 channels
        dict(name="norm prefill, 8 bits", op="rms", train=False, rows=32768, C=4096, bf16=True, res_bf16=True, block=128, quant=True),
        # training step of a layer with its residual stream in fp32, 65,536 tokens
        dict(name="norm train, layer", op="rms", train=True, rows=65536, C=768, bf16=True, res_bf16=False, block=0, quant=False),
        # a short batch of odd width, fp32
        dict(name="norm train, odd", op="rms", train=True, rows=1021, C=1001, bf16=False, res_bf16=False, block=0, quant=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["step", "forward", "forward", "train", "train", "conv", "conv", "rms", "rms"])
    bf16 = rng.random() < 0.5
    if kind == "rms":
        C = _log(rng, 16, 16384)
        if rng.random() < 0.6:
            C = max(16, C // 64 * 64)
        quant = rng.random() < 0.5
        return dict(op="rms", train=not quant and rng.random() < 0.7, rows=_log(rng, 1, 50_000_000 // C), C=C, bf16=bf16, res_bf16=bf16 and rng.random() < 0.5,
                    block=rng.choice([0, 0, 32, 128]) if quant else 0, quant=quant)
    if kind == "conv":
        C = _log(rng, 8, 8192)
        if rng.random() < 0.6:
            C = max(8, C // 8 * 8)
        L = _log(rng, 1, 16384) if rng.random() < 0.8 else 1
        return dict(op="conv", train=rng.random() < 0.6, B=_log(rng, 1, max(1, min(512, 50_000_000 // (L * C)))), L=L, C=C, k=rng.choice([2, 3, 4, 4]), bf16=bf16,
                    act=rng.choice([0, 1, 1]), ragged=rng.random() < 0.3)
    N, G = rng.choice([4, 8, 16, 16, 16, 24, 64, 128]), rng.choice([1, 1, 1, 2, 4])
    D = G * max(8, _log(rng, 64, 8192) // G)
    if rng.random() < 0.6:
        D = max(64 * G, D // (64 * G) * (64 * G))
    most = {"step": 1 << 26, "forward": 1 << 30, "train": 3 << 27}[kind]       # values of the states (a step's: of its batch)
    case = dict(op="scan", train=kind == "train", D=D, N=N, G=G, bf16=bf16, z=rng.random() < 0.7)
    if kind == "step":
        return case | dict(B=_log(rng, 1, max(1, min(512, most // (D * N)))), L=1, ragged=rng.random() < 0.5)
    L = _log(rng, 2, max(2, min(16384, most // (D * N))))
    return case | dict(B=_log(rng, 1, max(1, min(64, most // (L * D * N)))), L=L, ragged=rng.random() < 0.3)


def work(case):
    e = 2 if case["bf16"] else 4
    if case["op"] == "rms":
        n, C, rows, r = case["rows"] * case["C"], case["C"], case["rows"], 2 if case["res_bf16"] else 4
        if case["quant"]:           # x, residual -> h, q and its scales
            return {"bytes": n * (e + 2 * r + 1) + 4 * rows * _blocks(case) + 4 * C, "flops": 8 * n}
        if case["train"]:           # and h, dy, dh -> dx, dresidual
            return {"bytes": n * (e + 2 * r + e) + n * (r + e + r + e + r) + 8 * rows + 12 * C, "flops": 20 * n}
        return {"bytes": n * (e + 2 * r + e) + 4 * C, "flops": 6 * n}
    B, L = case["B"], case["L"]
    tokens, rows = B * L, B
    if case["ragged"]:
        n = _lengths(case)
        tokens, rows = int(n.sum()), int((n > 0).sum())
    tokens, rows = max(1, tokens), max(1, rows)
    if case["op"] == "conv":
        C, k = case["C"], case["k"]
        state = 8 * rows * (k - 1) * C
        if case["train"]:           # x -> y;  x, dy -> dx, dw, dbias; states and their gradients
            return {"bytes": 5 * tokens * C * e + 2 * state + 8 * C * (k + 1), "flops": 8 * k * tokens * C}
        return {"bytes": 2 * tokens * C * e + state + 4 * C * (k + 1), "flops": 2 * k * tokens * C}
    D, N, G = case["D"], case["N"], case["G"]
    wide, narrow, state, params = tokens * D * e, tokens * G * N * e, rows * D * N * 4, 4 * D * (N + 2)
    streams = 4 if case["z"] else 3                  # x, dt, y and z
    if case["train"]:               # and dy, dx, ddt, dz; B, C and theirs; states and theirs
        return {"bytes": (2 * streams) * wide + 4 * narrow + 4 * state + 2 * params, "flops": 20 * tokens * D * N}
    return {"bytes": streams * wide + 2 * narrow + 2 * state + params, "flops": 7 * tokens * D * N}


def _blocks(case):
    return -(-case["C"] // case["block"]) if case["block"] else 1


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


SCAN_GRADS = ("x", "dt", "A", "Bm", "Cm", "D", "z", "dt_bias", "state_in")


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    dt = torch.bfloat16 if case["bf16"] else torch.float32

    def normal(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=gen, device=DEV, dtype=torch.float32).to(dtype)

    def empty(*shape, dtype=torch.float32):
        return torch.empty(shape, device=DEV, dtype=dtype)

    s = dict(case=case)
    if case["op"] == "rms":
        rows, C, rt = case["rows"], case["C"], torch.bfloat16 if case["res_bf16"] else torch.float32
        s.update(x=normal(rows, C, dtype=dt), residual=(4 * normal(rows, C)).to(rt), weight=1 + 0.2 * normal(C), h=empty(rows, C, dtype=rt))
        if case["quant"]:
            s.update(q=empty(rows, C, dtype=E4M3), scales=empty(rows, _blocks(case)))
        else:
            s.update(y=empty(rows, C, dtype=dt))
        if case["train"]:
            s.update(dy=normal(rows, C, dtype=dt), dh=normal(rows, C, dtype=rt), rstd=empty(rows), dx=empty(rows, C, dtype=dt), dresidual=empty(rows, C, dtype=rt), dweight=empty(C))
    else:
        B, L = case["B"], case["L"]
        s["lengths"] = torch.from_numpy(_lengths(case)).to(torch.int32).to(DEV) if case["ragged"] else None
        if case["op"] == "conv":
            C, k = case["C"], case["k"]
            s.update(x=normal(B, L, C, dtype=dt), w=normal(C, k) / math.sqrt(k), bias=0.1 * normal(C), state_in=normal(B, k - 1, C, dtype=dt).float(),
                     y=empty(B, L, C, dtype=dt), state_out=empty(B, k - 1, C))
            if case["train"]:
                s.update(dy=normal(B, L, C, dtype=dt), dstate_out=0.1 * normal(B, k - 1, C))
                for n in ("x", "w", "bias", "state_in"):
                    s["d" + n] = torch.empty_like(s[n])
        else:
            D, N, G = case["D"], case["N"], case["G"]
            step = torch.exp(math.log(1e-3) + math.log(1e2) * torch.rand(D, generator=gen, device=DEV))      # 0.001 to 0.1
            s.update(x=normal(B, L, D, dtype=dt), dt=(0.5 * normal(B, L, D)).to(dt), A=-torch.arange(1, N + 1, device=DEV, dtype=torch.float32) * torch.exp(0.1 * normal(D, N)),
                     Bm=normal(B, L, G, N, dtype=dt), Cm=normal(B, L, G, N, dtype=dt), D=1 + 0.1 * normal(D), z=normal(B, L, D, dtype=dt) if case["z"] else None,
                     dt_bias=step + torch.log(-torch.expm1(-step)), state_in=0.3 * normal(B, D, N), y=empty(B, L, D, dtype=dt), state_out=empty(B, D, N))
            if case["train"]:
                s.update(dy=normal(B, L, D, dtype=dt), dstate_out=0.1 * normal(B, D, N))
                for n in SCAN_GRADS:
                    s["d" + n] = None if s[n] is None else torch.empty_like(s[n])
    if own:
        s["plan"] = _plan(case)
    return s


def _plan(case):
    """Descriptor, checkpoint and workspace, which a program makes once for its sizes."""
    from paper_2604_04250_amd import binding as K
    bf16, ck, ws = int(case["bf16"]), None, 0
    if case["op"] == "rms":
        d = K.make_rms_desc(case["rows"], case["C"], bf16=bf16, residual_bf16=int(case["res_bf16"]), block=case["block"])
        ws = K.cawn_rms_norm_add_workspace_bytes(d)
    elif case["op"] == "conv":
        d = K.make_conv_desc(case["B"], case["L"], case["C"], case["k"], act=case["act"], bf16=bf16)
        ws = K.cawn_causal_conv_workspace_bytes(d)
    else:
        d = K.make_scan_desc(case["B"], case["L"], case["D"], case["N"], G=case["G"], dt_softplus=1, bf16=bf16)
        ws = K.cawn_selective_scan_workspace_bytes(d)
        if case["train"]:
            ck = torch.empty(max(1, K.cawn_selective_scan_ckpt_bytes(d)), dtype=torch.uint8, device=DEV)
    return d, ck, torch.empty(max(1, ws), dtype=torch.uint8, device=DEV)


def run(s):
    case = s["case"]
    if own:
        return _run_own(case, s)
    return {"scan": _plain_scan, "conv": _plain_conv, "rms": _plain_rms}[case["op"]](case, s)


def _run_own(case, s):
    from paper_2604_04250_amd import binding as K
    d, ck, ws = s["plan"]
    if case["op"] == "rms":
        K.check(K.cawn_rms_norm_add_fwd(d, s["x"], s["residual"], s["weight"], s["h"], s.get("y"), s.get("q"), s.get("scales"), s.get("rstd")))
        if case["quant"]:
            return {n: s[n] for n in ("h", "q", "scales")}
        if not case["train"]:
            return {n: s[n] for n in ("h", "y")}
        K.check(K.cawn_rms_norm_add_bwd(d, s["h"], s["weight"], s["rstd"], s["dy"], s["dh"], s["dx"], s["dresidual"], s["dweight"], ws))
        return {n: s[n] for n in ("h", "y", "dx", "dresidual", "dweight")}
    if case["op"] == "conv":
        K.check(K.cawn_causal_conv_fwd(d, s["x"], s["w"], s["bias"], s["lengths"], s["state_in"], s["y"], s["state_out"]))
        if not case["train"]:
            return {n: s[n] for n in ("y", "state_out")}
        K.check(K.cawn_causal_conv_bwd(d, s["x"], s["w"], s["bias"], s["lengths"], s["state_in"], s["dy"], s["dstate_out"], s["dx"], s["dw"], s["dbias"], s["dstate_in"], ws))
        return {n: s[n] for n in ("y", "state_out", "dx", "dw", "dbias", "dstate_in")}
    K.check(K.cawn_selective_scan_fwd(d, s["x"], s["dt"], s["A"], s["Bm"], s["Cm"], s["D"], s["z"], s["dt_bias"], s["lengths"], s["state_in"], s["y"], s["state_out"], ck, ws))
    if not case["train"]:
        return {n: s[n] for n in ("y", "state_out")}
    K.check(K.cawn_selective_scan_bwd(d, s["x"], s["dt"], s["A"], s["Bm"], s["Cm"], s["D"], s["z"], s["dt_bias"], s["lengths"], ck, s["dy"], s["dstate_out"],
                                      s["dx"], s["ddt"], s["dA"], s["dBm"], s["dCm"], s["dD"], s["dz"], s["ddt_bias"], s["dstate_in"], ws))
    return {n: s[n] for n in ("y", "state_out") + tuple("d" + n for n in SCAN_GRADS if s[n] is not None)}


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _silu(z):
    """SiLU and its slope."""
    f = 1 / (1 + torch.exp(-z))
    return z * f, f * (1 + z * (1 - f))


def _softplus(v):
    """log(1 + e^v) and its slope."""
    e = torch.exp(-v.abs())
    return v.clamp(min=0) + torch.log1p(e), torch.where(v >= 0, 1 / (1 + e), e / (1 + e))


def _prefixes(a, b):
    """S[t] = a[t] S[t-1] + b[t] along axis 1 from S = 0, and the running products of a, by doubling."""
    n, step = a.shape[1], 1
    while step < n:
        b = torch.cat([b[:, :step], b[:, step:] + a[:, step:] * b[:, :-step]], 1)
        a = torch.cat([a[:, :step], a[:, step:] * a[:, :-step]], 1)
        step *= 2
    return a, b


def _plain_scan(case, s):
    B, L, D, N, G = (case[k] for k in ("B", "L", "D", "N", "G"))
    kind, train = s["x"].dtype, case["train"]
    x, v, A = s["x"].float(), s["dt"].float() + s["dt_bias"], s["A"]
    Bm, Cm = s["Bm"].float(), s["Cm"].float()
    delta, slope = _softplus(v)
    if s["lengths"] is not None:        # padding leaves the state alone and answers zero
        keep = torch.arange(L, device=DEV)[None, :, None] < s["lengths"][:, None, None]
        delta, slope, x = (torch.where(keep, t, 0.0) for t in (delta, slope, x))
        Bm, Cm = (torch.where(keep[..., None], t, 0.0) for t in (Bm, Cm))
    gate, gate_slope = _silu(s["z"].float()) if case["z"] else (None, None)
    u = delta * x
    wide = lambda t: t.repeat_interleave(D // G, 2)  # noqa: E731    a group's values, for each of its channels
    S, begins, core = s["state_in"], [], torch.empty_like(x)
    spans = [(t, min(L, t + CHUNK)) for t in range(0, L, CHUNK)]
    for lo, hi in spans:
        begins.append(S)
        a, b = _prefixes(torch.exp(delta[:, lo:hi, :, None] * A), u[:, lo:hi, :, None] * wide(Bm[:, lo:hi]))
        states = b + a * S[:, None]
        core[:, lo:hi] = (wide(Cm[:, lo:hi]) * states).sum(-1)
        S = states[:, -1]
    core = core + s["D"] * x
    y = core * gate if case["z"] else core
    if s["lengths"] is not None:
        y = torch.where(keep, y, 0.0)
    out = {"y": y.to(kind), "state_out": S}
    if not train:
        return out
    dy = s["dy"].float()
    if s["lengths"] is not None:
        dy = torch.where(keep, dy, 0.0)
    g = dy * gate if case["z"] else dy
    dS, dA = s["dstate_out"], torch.zeros(D, N, device=DEV, dtype=torch.float64)
    du, dd = torch.empty_like(x), torch.empty_like(x)
    dB, dC = torch.empty_like(Bm), torch.empty_like(Cm)
    for (lo, hi), S in zip(reversed(spans), reversed(begins)):
        bw, cw, uc = wide(Bm[:, lo:hi]), wide(Cm[:, lo:hi]), u[:, lo:hi, :, None]
        a = torch.exp(delta[:, lo:hi, :, None] * A)
        pa, pb = _prefixes(a, uc * bw)
        states = pb + pa * S[:, None]
        before = torch.cat([S[:, None], states[:, :-1]], 1)
        # D[t] = C[t] g[t] + a[t+1] D[t+1]: the same along the axis turned round, from what reaches the last token
        later = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1).flip(1)
        qa, qb = _prefixes(later, (cw * g[:, lo:hi, :, None]).flip(1))
        grads = (qb + qa * dS[:, None]).flip(1)
        p = grads * a
        dS = p[:, 0]
        p = p * before
        du[:, lo:hi] = (grads * bw).sum(-1)
        dd[:, lo:hi] = (p * A).sum(-1)
        dA += (p * delta[:, lo:hi, :, None]).sum((0, 1)).double()
        shape = (B, hi - lo, G, D // G, N)
        dB[:, lo:hi] = (grads * uc).reshape(shape).sum(3)
        dC[:, lo:hi] = (states * g[:, lo:hi, :, None]).reshape(shape).sum(3)
    dv = (dd + du * x) * slope
    dx = du * delta + s["D"] * g
    if s["lengths"] is not None:
        dx, dB, dC = torch.where(keep, dx, 0.0), torch.where(keep[..., None], dB, 0.0), torch.where(keep[..., None], dC, 0.0)
    out |= {"dx": dx.to(kind), "ddt": dv.to(kind), "dA": dA.float(), "dBm": dB.to(kind), "dCm": dC.to(kind),
            "dD": (g * x).sum((0, 1)), "ddt_bias": dv.sum((0, 1)), "dstate_in": dS}
    if case["z"]:
        out["dz"] = (dy * core * gate_slope).to(kind)
    return out


def _plain_conv(case, s):
    B, L, C, k = (case[n] for n in ("B", "L", "C", "k"))
    x, w, dt = s["x"].float(), s["w"], s["x"].dtype
    n = torch.full((B,), L, device=DEV) if s["lengths"] is None else s["lengths"].long()
    keep = (torch.arange(L, device=DEV)[None, :] < n[:, None])[..., None]
    x = torch.where(keep, x, 0.0)
    line = torch.cat([s["state_in"], x], 1)                     # what a token sees begins at its own number
    z = s["bias"] + sum(w[:, i] * line[:, i:i + L] for i in range(k))
    y, slope = _silu(z) if case["act"] else (z, torch.ones_like(z))
    at = (n[:, None] + torch.arange(k - 1, device=DEV))[..., None].expand(B, k - 1, C)
    out = {"y": torch.where(keep, y, 0.0).to(dt), "state_out": torch.gather(line, 1, at)}
    if not case["train"]:
        return out
    dz = torch.where(keep, s["dy"].float() * slope, 0.0)
    dline = torch.zeros_like(line).scatter_add_(1, at, s["dstate_out"])
    for i in range(k):
        dline[:, i:i + L] += w[:, i] * dz
    out |= {"dx": dline[:, k - 1:].to(dt), "dstate_in": dline[:, :k - 1], "dbias": dz.sum((0, 1)),
            "dw": torch.stack([(dz * line[:, i:i + L]).sum((0, 1)) for i in range(k)], 1)}
    return out


def _plain_rms(case, s):
    rows, C, w = case["rows"], case["C"], s["weight"]
    dt, rt = s["x"].dtype, s["residual"].dtype
    h = (s["x"].float() + s["residual"].float()).to(rt)
    hf = h.float()
    rstd = torch.rsqrt(hf.square().mean(1, keepdim=True) + 1e-5)
    hh = hf * rstd
    y = hh * w
    if case["quant"]:
        m, width = _blocks(case), case["block"] or C
        padded = torch.nn.functional.pad(y, (0, m * width - C)).reshape(rows, m, width)
        scale = padded.abs().amax(-1, keepdim=True) / 448.0
        q = torch.where(scale > 0, padded / scale, 0.0).reshape(rows, m * width)[:, :C]
        return {"h": h, "q": q.to(E4M3), "scales": scale[..., 0]}
    out = {"h": h, "y": y.to(dt)}
    if not case["train"]:
        return out
    dy = s["dy"].float()
    t = dy * w
    dr = s["dh"].float() + rstd * (t - hh * (t * hh).mean(1, keepdim=True))
    return out | {"dx": dr.to(dt), "dresidual": dr.to(rt), "dweight": (dy * hh).sum(0)}


# ---- 64 bits, from the definitions ------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"scan": _exact_scan, "conv": _exact_conv, "rms": _exact_rms}[case["op"]](case, s)


def _exact_rms(case, s):
    C, w = case["C"], s["weight"].double()
    h = s["x"].double() + s["residual"].double()
    held = h.to(s["residual"].dtype).double() if case["res_bf16"] else h        # (fp32: its rounding is below what is compared)
    sd = (held.pow(2).sum(1, keepdim=True) / C + 1e-5).sqrt()
    y = w * held / sd
    if case["quant"]:       # what is rounded to 8 bits, in units of its scale
        width = case["block"] or C
        scales = torch.stack([y[:, lo:lo + width].abs().max(1).values / 448 for lo in range(0, C, width)], 1)
        each = scales.repeat_interleave(width, 1)[:, :C]
        return {"h": h, "q": y / torch.where(each == 0, 1.0, each), "scales": scales}
    if not case["train"]:
        return {"h": h, "y": y}
    dy, unit = s["dy"].double(), held / sd
    t = dy * w
    dr = s["dh"].double() + (t - unit * (t * unit).sum(1, keepdim=True) / C) / sd
    return {"h": h, "y": y, "dx": dr, "dresidual": dr, "dweight": (dy * unit).sum(0)}


def _exact_conv(case, s):
    B, L, C, k = (case[n] for n in ("B", "L", "C", "k"))
    x, w = s["x"].double(), s["w"].double()
    n = [L] * B if s["lengths"] is None else s["lengths"].tolist()
    y = torch.zeros_like(x)
    state = torch.empty(B, k - 1, C, device=DEV, dtype=torch.float64)
    grads = {"dx": torch.zeros_like(x), "dw": torch.zeros_like(w), "dbias": torch.zeros(C, device=DEV, dtype=torch.float64), "dstate_in": torch.empty_like(state)}
    for b in range(B):
        line = torch.cat([s["state_in"][b].double(), x[b, :n[b]]])
        state[b] = line[n[b]:]
        z = s["bias"].double() + (line.unfold(0, k, 1) * w).sum(-1) if n[b] else x[b, :0]
        f = torch.sigmoid(z)
        y[b, :n[b]] = z * f if case["act"] else z
        if case["train"]:
            dz = s["dy"][b, :n[b]].double() * (f + z * f * (1 - f) if case["act"] else 1.0)
            dline = torch.zeros_like(line)
            dline[n[b]:] += s["dstate_out"][b].double()
            for i in range(k):
                dline[i:i + n[b]] += w[:, i] * dz
                grads["dw"][:, i] += (dz * line[i:i + n[b]]).sum(0)
            grads["dbias"] += dz.sum(0)
            grads["dx"][b, :n[b]], grads["dstate_in"][b] = dline[k - 1:], dline[:k - 1]
    return {"y": y, "state_out": state} | (grads if case["train"] else {})


def _exact_scan(case, s):
    """Token by token; gradients by the adjoint recurrence, with the states of one run of tokens kept at a time."""
    B, L, D, N, G = (case[k] for k in ("B", "L", "D", "N", "G"))
    if L * (4 if case["train"] else 1) > 40000:
        return None
    n = s["lengths"]
    live = torch.ones(B, L, 1, device=DEV, dtype=torch.float64) if n is None else (torch.arange(L, device=DEV) < n[:, None]).double()[..., None]
    v = s["dt"].double() + s["dt_bias"].double()
    delta, sig = torch.logaddexp(v, torch.zeros_like(v)) * live, torch.sigmoid(v) * live
    x, A, Dk = s["x"].double() * live, s["A"].double(), s["D"].double()
    # time first, so that a token's rows lie together
    x, delta, sig = (t.movedim(1, 0).contiguous() for t in (x, delta, sig))
    Bm, Cm = ((s[m].double() * live[..., None]).movedim(1, 0).contiguous() for m in ("Bm", "Cm"))
    spread = lambda t: t[:, :, None, :].expand(B, G, D // G, N).reshape(B, D, N)  # noqa: E731

    def token(S, t):
        return torch.exp(delta[t][..., None] * A) * S + (delta[t] * x[t])[..., None] * spread(Bm[t])

    S, core, held = s["state_in"].double(), torch.empty_like(x), []
    for t in range(L):
        if case["train"] and t % 64 == 0:
            held.append(S)
        S = token(S, t)
        core[t] = (spread(Cm[t]) * S).sum(-1) + Dk * x[t]
    core = core.movedim(0, 1)
    if case["z"]:
        z = s["z"].double()
        f = torch.sigmoid(z)
        gate, gate_slope = z * f, f + z * f * (1 - f)
    else:
        gate = torch.ones_like(core)
    out = {"y": core * gate * live, "state_out": S}
    if not case["train"]:
        return out
    dy = s["dy"].double() * live
    g = (dy * gate).movedim(1, 0).contiguous()
    du, dd, dA = torch.empty_like(x), torch.empty_like(x), torch.zeros_like(A)
    dB, dC = torch.empty_like(Bm), torch.empty_like(Cm)
    grad = s["dstate_out"].double()
    for c in reversed(range(len(held))):
        run_ = [held[c]]
        for t in range(64 * c, min(L, 64 * c + 64)):
            run_.append(token(run_[-1], t))
        for t in reversed(range(64 * c, 64 * c + len(run_) - 1)):
            before, after = run_[t - 64 * c], run_[t - 64 * c + 1]
            grad = grad + spread(Cm[t]) * g[t][..., None]
            dC[t] = (after * g[t][..., None]).reshape(B, G, -1, N).sum(2)
            dB[t] = (grad * (delta[t] * x[t])[..., None]).reshape(B, G, -1, N).sum(2)
            du[t] = (grad * spread(Bm[t])).sum(-1)
            grad = grad * torch.exp(delta[t][..., None] * A)
            p = grad * before
            dd[t] = (p * A).sum(-1)
            dA += (p * delta[t][..., None]).sum(0)
    back = lambda t: t.movedim(0, 1)  # noqa: E731
    dv = (dd + du * x) * sig
    mask = live[..., None]
    out |= {"dx": back(du * delta + Dk * g) * live, "ddt": back(dv), "dA": dA, "dBm": back(dB) * mask, "dCm": back(dC) * mask,
            "dD": (g * x).sum((0, 1)), "ddt_bias": dv.sum((0, 1)), "dstate_in": grad}
    if case["z"]:
        out["dz"] = dy * core * gate_slope
    return out
