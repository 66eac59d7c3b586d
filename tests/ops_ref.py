"""The operators beside the scan in 64 bits, from their definitions: numpy, token by token, no code of the library."""
from __future__ import annotations

import math

import numpy as np


def _unit(x, eps, on):
    r = 1.0 / np.sqrt((x * x).sum(-1, keepdims=True) + eps) if on else np.ones(x.shape[:-1] + (1,))
    return x * r, r


def _tokens(L, lengths, b):
    return L if lengths is None else int(min(max(lengths[b], 0), L))


def delta_fwd(q, k, v, decay, beta, scale=1.0, qk_norm=0, eps=1e-6, lengths=None, state_in=None, keep=None):
    """q, k [B,L,Hk,K], v [B,L,H,V], decay, beta [B,L,H], state [B,H,K,V] -> o, state_out; `keep`: a list that gets (r, e, S) per token."""
    q, k, v, decay, beta = (np.asarray(t, np.float64) for t in (q, k, v, decay, beta))
    B, L, H, V = v.shape
    rep = H // k.shape[2]
    qh, kh = (np.repeat(_unit(t, eps, qk_norm)[0], rep, axis=2) for t in (q, k))
    S = np.zeros((B, H, k.shape[3], V)) if state_in is None else np.asarray(state_in, np.float64).copy()
    o = np.zeros((B, L, H, V))
    for b in range(B):
        for t in range(_tokens(L, lengths, b)):
            r = np.exp(decay[b, t])[:, None, None] * S[b]
            e = v[b, t] - np.einsum("hk,hkv->hv", kh[b, t], r)
            S[b] = r + kh[b, t][:, :, None] * (beta[b, t][:, None] * e)[:, None, :]
            o[b, t] = scale * np.einsum("hk,hkv->hv", qh[b, t], S[b])
            if keep is not None:
                keep.append((b, t, r, e, S[b].copy()))
    return o, S


def delta_bwd(q, k, v, decay, beta, do, dstate_out=None, scale=1.0, qk_norm=0, eps=1e-6, lengths=None, state_in=None):
    """Gradients dict(dq, dk, dv, ddecay, dbeta, dstate_in)."""
    q, k, v, decay, beta, do = (np.asarray(t, np.float64) for t in (q, k, v, decay, beta, do))
    B, L, H, V = v.shape
    Hk, K = k.shape[2:]
    rep = H // Hk
    (qu, rq), (ku, rk) = _unit(q, eps, qk_norm), _unit(k, eps, qk_norm)
    qh, kh = np.repeat(qu, rep, axis=2), np.repeat(ku, rep, axis=2)
    kept = []
    delta_fwd(q, k, v, decay, beta, scale, qk_norm, eps, lengths, state_in, kept)
    D = np.zeros((B, H, K, V)) if dstate_out is None else np.asarray(dstate_out, np.float64).copy()
    dqh, dkh, dv, dg, db = np.zeros_like(qh), np.zeros_like(kh), np.zeros_like(v), np.zeros_like(decay), np.zeros_like(beta)
    for b, t, r, e, S in reversed(kept):
        dqh[b, t] = scale * np.einsum("hkv,hv->hk", S, do[b, t])
        D[b] += scale * qh[b, t][:, :, None] * do[b, t][:, None, :]
        u = beta[b, t][:, None] * e
        du = np.einsum("hk,hkv->hv", kh[b, t], D[b])
        db[b, t] = (du * e).sum(-1)
        dv[b, t] = beta[b, t][:, None] * du
        dkh[b, t] = np.einsum("hkv,hv->hk", D[b], u) - np.einsum("hkv,hv->hk", r, dv[b, t])
        D[b] -= kh[b, t][:, :, None] * dv[b, t][:, None, :]
        dg[b, t] = (D[b] * r).sum((-2, -1))
        D[b] *= np.exp(decay[b, t])[:, None, None]
    out = dict(dv=dv, ddecay=dg, dbeta=db, dstate_in=D)
    for n, d, xu, r in (("dq", dqh, qu, rq), ("dk", dkh, ku, rk)):
        d = d.reshape(B, L, Hk, rep, K).sum(3)
        out[n] = r * (d - xu * (xu * d).sum(-1, keepdims=True)) if qk_norm else d
    return out


def _erf(z):
    return np.vectorize(math.erf, otypes=[np.float64])(z)


def act(z, kind):
    if kind == 1:
        return z / (1 + np.exp(-z))
    return z * 0.5 * (1 + _erf(z / math.sqrt(2))) if kind == 2 else z


def act_slope(z, kind):
    if kind == 1:
        s = 1 / (1 + np.exp(-z))
        return s * (1 + z * (1 - s))
    if kind == 2:
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    return np.ones_like(z)


def norm_fwd(x, w, b, groups, kind=0, eps=1e-5):
    """x [B,T,C] -> y, xh, 1 / deviation [B,1,G,1], mean."""
    x = np.asarray(x, np.float64)
    B, T, C = x.shape
    xg = x.reshape(B, T, groups, C // groups)
    mean = xg.mean((1, 3), keepdims=True)
    rstd = 1 / np.sqrt(((xg - mean) ** 2).mean((1, 3), keepdims=True) + eps)
    xh = ((xg - mean) * rstd).reshape(B, T, C)
    w = np.ones(C) if w is None else np.asarray(w, np.float64)
    b = np.zeros(C) if b is None else np.asarray(b, np.float64)
    return act(xh * w + b, kind), xh, rstd, mean


def norm_bwd(x, w, b, dy, groups, kind=0, eps=1e-5):
    _, xh, rstd, _ = norm_fwd(x, w, b, groups, kind, eps)
    B, T, C = xh.shape
    w = np.ones(C) if w is None else np.asarray(w, np.float64)
    b = np.zeros(C) if b is None else np.asarray(b, np.float64)
    dz = np.asarray(dy, np.float64) * act_slope(xh * w + b, kind)
    t, h = (dz * w).reshape(B, T, groups, -1), xh.reshape(B, T, groups, -1)
    dx = rstd * (t - t.mean((1, 3), keepdims=True) - h * (t * h).mean((1, 3), keepdims=True))
    return dict(dx=dx.reshape(B, T, C), dweight=(dz * xh).sum((0, 1)), dbias=dz.sum((0, 1)))


def philox(block, seed):
    """Philox-4x32-10 of one 128-bit counter (block, 0), in whole numbers: four 32-bit words."""
    m = 0xffffffff
    c = [block & m, (block >> 32) & m, 0, 0]
    k = [seed & m, (seed >> 32) & m]
    for _ in range(10):
        p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & m, (p0 >> 32) ^ c[3] ^ k[1], p0 & m]
        k = [(k[0] + 0x9E3779B9) & m, (k[1] + 0xBB67AE85) & m]
    return c


def keep_mask(rows, cols, seed, offset, p):
    n = rows * cols
    words = [w for b in range((n + 3) // 4) for w in philox((offset + b) & 0xffffffffffffffff, seed)]
    return (np.array(words[:n], np.uint64) >= np.uint64(int(p * 2 ** 32)) if p < 1 else np.zeros(n, bool)).reshape(rows, cols)
