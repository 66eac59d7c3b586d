"""Helpers of the GPU tests of the selective scan, the short convolution and the norm: strided device tensors, calls through the C ABI."""
from __future__ import annotations

import numpy as np
import torch

from gpu_util import DEV, rel_err  # noqa: F401
from paper_2604_04250_amd import binding as K

EPS = 2.0 ** -24
ROUND16 = 2.0 ** -8


def rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def rounded(a, bf16):
    """The values that a tensor of the type holds, as float32."""
    t = torch.from_numpy(np.ascontiguousarray(a, np.float32))
    return (t.to(torch.bfloat16).float() if bf16 else t).numpy()


def strided(a, dtype, extra=0, offset=0):
    """A device tensor of a's values whose rows are `extra` longer, `offset` elements into its memory; NaN around it."""
    a = np.asarray(a, np.float32)
    rows = int(np.prod(a.shape[:-1]))
    flat = torch.full((rows * (a.shape[-1] + extra) + offset,), float("nan"), device=DEV, dtype=dtype)
    v = flat[offset:].view(*a.shape[:-1], a.shape[-1] + extra)[..., : a.shape[-1]]
    v.copy_(torch.from_numpy(a))
    return v


def dev(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(DEV)


def host(t):
    return None if t is None else t.float().cpu().numpy()


def scratch(n):
    return torch.full((max(256, n),), 0xff, dtype=torch.uint8, device=DEV)


def like(v, extra):
    """An output laid out like v, all NaN."""
    return strided(np.full(tuple(v.shape), np.nan, np.float32), v.dtype, extra)


def scan_inputs(B, L, D, N, G, bf16, seed, z=True, ragged=False, step=(1e-3, 0.1), skip=True, bias=True):
    r = rng(seed)
    i = dict(x=r.standard_normal((B, L, D)), dt=0.5 * r.standard_normal((B, L, D)), Bm=r.standard_normal((B, L, G, N)), Cm=r.standard_normal((B, L, G, N)),
             z=r.standard_normal((B, L, D)) if z else None, dy=r.standard_normal((B, L, D)))
    i = {n: None if a is None else rounded(a, bf16) for n, a in i.items()}
    s = np.exp(r.uniform(np.log(step[0]), np.log(step[1]), D))
    f32 = lambda a: np.asarray(a, np.float32)  # noqa: E731
    i.update(A=f32(-np.arange(1, N + 1) * np.exp(0.1 * r.standard_normal((D, N)))), Dk=f32(1 + 0.1 * r.standard_normal(D)) if skip else None,
             bias=f32(s + np.log(-np.expm1(-s))) if bias else None, state_in=f32(0.3 * r.standard_normal((B, D, N))), dstate_out=f32(0.1 * r.standard_normal((B, D, N))),
             lengths=None)
    if ragged:
        n = r.integers(0, L + 1, B)
        n[0], n[-1] = L, 0
        if B > 2:
            n[1] = 1
        i["lengths"] = n.astype(np.int32)
    return i


def reference_inputs(i):
    return {k: i[k] for k in ("x", "dt", "A", "Bm", "Cm", "Dk", "z", "bias", "lengths", "state_in")}


class Scan:
    """One call's tensors; what a padded batch holds behind its rows is NaN, and so is what lies between rows."""

    def __init__(self, i, bf16, softplus=1, extra=(0, 0, 0, 0, 0), offset=0, accumulate=0, ckpt=True, poison=True):
        self.i, self.bf16, self.extra = i, bf16, extra
        dt = torch.bfloat16 if bf16 else torch.float32
        B, L, D = i["x"].shape
        G, N = i["Bm"].shape[2:]
        self.shape = B, L, D, N, G
        a = {k: None if i[k] is None else i[k].copy() for k in ("x", "dt", "Bm", "Cm", "z", "dy")}
        if i["lengths"] is not None and poison:
            for b in range(B):
                for v in a.values():
                    if v is not None:
                        v[b, max(0, int(i["lengths"][b])):] = np.nan
        ex, ed, eb, ez, ey = extra
        self.d = K.make_scan_desc(B, L, D, N, G=G, dt_softplus=softplus, bf16=int(bf16), accumulate_param_grads=accumulate, x_stride_t=D + ex if ex else 0,
                                  dt_stride_t=D + ed if ed else 0, bc_stride_t=G * N + eb if eb else 0, z_stride_t=D + ez if ez else 0, y_stride_t=D + ey if ey else 0)
        self.x, self.dt, self.dy = strided(a["x"], dt, ex, offset), strided(a["dt"], dt, ed, offset), strided(a["dy"], dt, ey, offset)
        self.Bm, self.Cm = (strided(a[k].reshape(B, L, G * N), dt, eb, offset) for k in ("Bm", "Cm"))
        self.z = None if a["z"] is None else strided(a["z"], dt, ez, offset)
        self.A, self.Dk, self.bias, self.state_in, self.dstate_out = (dev(i[k]) for k in ("A", "Dk", "bias", "state_in", "dstate_out"))
        self.lengths = None if i["lengths"] is None else torch.from_numpy(i["lengths"]).to(DEV)
        self.y = like(self.x, ey)
        self.state_out = torch.full((B, D, N), float("nan"), device=DEV)
        self.ckpt = scratch(K.cawn_selective_scan_ckpt_bytes(self.d)) if ckpt else None
        self.ws = scratch(K.cawn_selective_scan_workspace_bytes(self.d))

    def forward(self, state_in="own", state_out="own", stream=None):
        K.check(K.cawn_selective_scan_fwd(self.d, self.x, self.dt, self.A, self.Bm, self.Cm, self.Dk, self.z, self.bias, self.lengths,
                                          self.state_in if state_in == "own" else state_in, self.y, self.state_out if state_out == "own" else state_out, self.ckpt,
                                          self.ws, stream))
        return self

    def backward(self, want=("x", "dt", "A", "Bm", "Cm", "Dskip", "z", "dt_bias", "state_in"), dstate="own", fill=float("nan"), stream=None):
        ex, ed, eb, ez, ey = self.extra
        new = lambda t: None if t is None else torch.full_like(t, fill)  # noqa: E731
        self.g = dict(x=like(self.x, ex), dt=like(self.dt, ed), A=new(self.A), Bm=like(self.Bm, eb), Cm=like(self.Cm, eb), Dskip=new(self.Dk),
                      z=None if self.z is None else like(self.z, ez), dt_bias=new(self.bias), state_in=torch.full_like(self.state_out, float("nan")))
        g = {k: v if k in want else None for k, v in self.g.items()}
        if dstate == "in place":
            self.g["state_in"] = g["state_in"] = self.dstate_out
        K.check(K.cawn_selective_scan_bwd(self.d, self.x, self.dt, self.A, self.Bm, self.Cm, self.Dk, self.z, self.bias, self.lengths, self.ckpt, self.dy,
                                          None if dstate is None else self.dstate_out, g["x"], g["dt"], g["A"], g["Bm"], g["Cm"], g["Dskip"], g["z"], g["dt_bias"],
                                          g["state_in"], self.ws, stream))
        return self

    def grads(self):
        B, L, D, N, G = self.shape
        g = {"d" + k: host(v) for k, v in self.g.items()}
        for k in ("dBm", "dCm"):
            g[k] = g[k].reshape(B, L, G, N)
        return g


def untouched(v, extra):
    """Nothing is written between a strided output's rows."""
    if not extra:
        return True
    whole = torch.as_strided(v, (int(np.prod(v.shape[:-1])), v.shape[-1] + extra), (v.shape[-1] + extra, 1), v.storage_offset())
    return bool(torch.isnan(whole[:, v.shape[-1]:]).all())
