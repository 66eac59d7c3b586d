"""The selective scan, its short convolution and the norm with the residual addition in 64 bits, from their definitions: numpy, token by token, no
code of the library."""
from __future__ import annotations

import numpy as np


def sigmoid(z):
    return np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))


def silu(z):
    return z * sigmoid(z)


def silu_slope(z):
    s = sigmoid(z)
    return s * (1 + z * (1 - s))


def tokens_of(L, lengths, b):
    return L if lengths is None else int(min(max(int(lengths[b]), 0), L))


def _f64(*arrays):
    return tuple(None if a is None else np.asarray(a, np.float64) for a in arrays)


def scan_fwd(x, dt, A, Bm, Cm, Dk=None, z=None, bias=None, lengths=None, state_in=None, softplus=True, keep=None):
    """x, dt, z [B,L,D], A [D,N], Bm, Cm [B,L,G,N] -> y, state_out; `keep`: a list that gets (b, t, factors, S before, S behind) per token."""
    x, dt, A, Bm, Cm, Dk, z, bias, state_in = _f64(x, dt, A, Bm, Cm, Dk, z, bias, state_in)
    B, L, D = x.shape
    N, G = A.shape[1], Bm.shape[2]
    S = np.zeros((B, D, N)) if state_in is None else state_in.copy()
    y = np.zeros((B, L, D))
    v = dt + (0.0 if bias is None else bias)
    delta = np.logaddexp(v, 0.0) if softplus else v
    for b in range(B):
        for t in range(tokens_of(L, lengths, b)):
            bm, cm = (np.repeat(m[b, t], D // G, axis=0) for m in (Bm, Cm))
            a = np.exp(delta[b, t][:, None] * A)
            before = S[b].copy()
            S[b] = a * S[b] + (delta[b, t] * x[b, t])[:, None] * bm
            core = (cm * S[b]).sum(-1) + (0.0 if Dk is None else Dk * x[b, t])
            y[b, t] = core if z is None else core * silu(z[b, t])
            if keep is not None:
                keep.append((b, t, a, before, S[b].copy(), core))
    return y, S


def scan_bwd(x, dt, A, Bm, Cm, dy, dstate_out=None, Dk=None, z=None, bias=None, lengths=None, state_in=None, softplus=True):
    """Gradients dict(dx, ddt, dA, dBm, dCm, dDskip, dz, ddt_bias, dstate_in)."""
    kept = []
    scan_fwd(x, dt, A, Bm, Cm, Dk, z, bias, lengths, state_in, softplus, kept)
    x, dt, A, Bm, Cm, dy, dstate_out, Dk, z, bias = _f64(x, dt, A, Bm, Cm, dy, dstate_out, Dk, z, bias)
    B, L, D = x.shape
    N, G = A.shape[1], Bm.shape[2]
    v = dt + (0.0 if bias is None else bias)
    delta, slope = (np.logaddexp(v, 0.0), sigmoid(v)) if softplus else (v, np.ones_like(v))
    H = np.zeros((B, D, N)) if dstate_out is None else dstate_out.copy()
    out = dict(dx=np.zeros_like(x), ddt=np.zeros_like(x), dz=np.zeros_like(x), dA=np.zeros_like(A), dBm=np.zeros_like(Bm), dCm=np.zeros_like(Cm),
               dDskip=np.zeros(D), ddt_bias=np.zeros(D))
    for b, t, a, before, after, core in reversed(kept):
        bm, cm = (np.repeat(m[b, t], D // G, axis=0) for m in (Bm, Cm))
        g = dy[b, t] if z is None else dy[b, t] * silu(z[b, t])
        if z is not None:
            out["dz"][b, t] = dy[b, t] * silu_slope(z[b, t]) * core
        dS = H[b] + cm * g[:, None]
        out["dCm"][b, t] = (after * g[:, None]).reshape(G, D // G, N).sum(1)
        out["dBm"][b, t] = (dS * (delta[b, t] * x[b, t])[:, None]).reshape(G, D // G, N).sum(1)
        du = (dS * bm).sum(-1)
        p = dS * a * before
        dv = ((p * A).sum(-1) + du * x[b, t]) * slope[b, t]
        out["dA"] += p * delta[b, t][:, None]
        out["dx"][b, t] = du * delta[b, t] + (0.0 if Dk is None else Dk * g)
        out["ddt"][b, t] = dv
        out["ddt_bias"] += dv
        out["dDskip"] += g * x[b, t]
        H[b] = a * dS
    out["dstate_in"] = H
    return out


def conv_fwd(x, w, bias=None, act=1, lengths=None, state_in=None):
    """x [B,L,C], w [C,k], state [B,k-1,C] -> y, state_out, and per row the line of inputs and the values before the activation."""
    x, w, bias, state_in = _f64(x, w, bias, state_in)
    B, L, C = x.shape
    k = w.shape[1]
    y, state, lines, zs = np.zeros_like(x), np.zeros((B, k - 1, C)), [], []
    for b in range(B):
        n = tokens_of(L, lengths, b)
        line = np.concatenate([np.zeros((k - 1, C)) if state_in is None else state_in[b], x[b, :n]])
        zz = np.zeros((n, C))
        for t in range(n):
            zz[t] = (w.T * line[t:t + k]).sum(0) + (0.0 if bias is None else bias)
            y[b, t] = silu(zz[t]) if act else zz[t]
        state[b] = line[n:n + k - 1]
        lines.append(line)
        zs.append(zz)
    return y, state, lines, zs


def conv_bwd(x, w, dy, dstate_out=None, bias=None, act=1, lengths=None, state_in=None):
    """Gradients dict(dx, dw, dbias, dstate_in)."""
    _, _, lines, zs = conv_fwd(x, w, bias, act, lengths, state_in)
    x, w, dy, dstate_out = _f64(x, w, dy, dstate_out)
    B, L, C = x.shape
    k = w.shape[1]
    out = dict(dx=np.zeros_like(x), dw=np.zeros_like(w), dbias=np.zeros(C), dstate_in=np.zeros((B, k - 1, C)))
    for b in range(B):
        n = tokens_of(L, lengths, b)
        dline = np.zeros((n + k - 1, C))
        if dstate_out is not None:
            dline[n:] += dstate_out[b]
        for t in range(n):
            dz = dy[b, t] * (silu_slope(zs[b][t]) if act else 1.0)
            out["dbias"] += dz
            out["dw"] += (dz * lines[b][t:t + k]).T
            dline[t:t + k] += dz * w.T
        out["dstate_in"][b], out["dx"][b, :n] = dline[:k - 1], dline[k - 1:]
    return out


def rms_fwd(h, w=None, eps=1e-5):
    """h [rows,C], already rounded -> y, 1 / sqrt(mean + eps) [rows]."""
    h, w = _f64(h, w)
    r = 1 / np.sqrt((h * h).mean(1) + eps)
    return h * r[:, None] * (1.0 if w is None else w), r


def rms_bwd(h, dy, w=None, dh=None, eps=1e-5):
    """Gradients of h and of w."""
    h, dy, w, dh = _f64(h, dy, w, dh)
    _, r = rms_fwd(h, None, eps)
    unit = h * r[:, None]
    t = dy * (1.0 if w is None else w)
    d = r[:, None] * (t - unit * (t * unit).mean(1, keepdims=True))
    return d + (0.0 if dh is None else dh), (dy * unit).sum(0)


def blocks_of(y, block):
    """Largest magnitudes of the blocks of each row [rows, blocks], and the block of each channel."""
    C = y.shape[1]
    width = block or C
    at = np.arange(C) // width
    return np.stack([np.abs(y[:, at == j]).max(1) for j in range(at[-1] + 1)], 1), at
