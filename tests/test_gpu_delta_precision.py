"""bf16 calls of the gated delta rule hold the arithmetic of fp32: what a large state leaves where it has just been overwritten."""
import pytest
import torch

from gpu_util import rel_err
from test_gpu_delta import desc, fwd, host, make, num, ref_fwd
from test_gpu_delta_bwd import ref, run

pytestmark = pytest.mark.gpu

# The state is SIZE times the values.  A query of the key just written, with beta = 1, finds the value alone: products of SIZE that cancel
# to one.  Each is held to some 100 roundings of 2^-24; a bf16 output adds 2^-8 of itself.
SIZE = 1000.0
TERMS = SIZE * 100 * 2.0 ** -24
TOL16 = 2.0 ** -8 + TERMS


def _overwritten(L, Kd, V, seed):
    x = make(1, L, 2, 2, Kd, V, True, 1, seed)
    x["state_in"] *= SIZE
    x["beta"][:] = 1
    x["decay"][:] = -1e-3
    x["q"] = x["k"].clone()
    return x


@pytest.mark.parametrize("L,Kd,V", [(17, 64, 64), (64, 64, 72), (130, 128, 64), (100, 32, 40), (450, 64, 64)])
def test_values_written_over_a_large_state(L, Kd, V):
    x = _overwritten(L, Kd, V, L)
    want = ref_fwd(host(x), 1)[0]
    o = num(fwd(x, desc(x, 1))[0])
    assert rel_err(o, want) <= TOL16
    # token by token the same
    for t in range(0, 16):
        assert rel_err(o[:, t], want[:, t]) <= TOL16


def _by_chunks(x, scale=0.6):
    """The formula by chunks in plain fp32 on the CPU."""
    x = {n: None if t is None else t.float().cpu() for n, t in x.items()}
    x["k"].requires_grad_()
    q, k = (t * (t.square().sum(-1, keepdim=True) + 1e-6).rsqrt() for t in (x["q"], x["k"]))
    S, o = x["state_in"], []
    for at in range(0, q.shape[1], 64):
        Q, Kc, v, g, be = (t[:, at:at + 64].transpose(1, 2) for t in (q, k, x["v"], x["decay"], x["beta"][..., None]))
        g = g.double().cumsum(-1)
        D = torch.exp((g[..., :, None] - g[..., None, :]).float()).tril()
        eg, ed, kt = g.exp().float()[..., None], (g[..., -1:] - g).exp().float()[..., None], Kc.transpose(-1, -2)
        n = (be * D * (Kc @ kt)).tril(-1)
        u = torch.linalg.solve_triangular(n + torch.eye(n.shape[-1]), be * (v - eg * (Kc @ S)), upper=False)
        o.append((scale * (eg * (Q @ S) + (D * (Q @ kt)) @ u)).transpose(1, 2))
        S = eg[..., -1:, :] * S + (ed * Kc).transpose(-1, -2) @ u
    (torch.cat(o, 1) * x["do"]).sum().add((S * x["dstate_out"]).sum()).backward()
    return x["k"].grad.numpy()


@pytest.mark.parametrize("Kd,V", [(4, 64), (3, 64), (5, 40)])
def test_gradients_of_keys_that_have_overwritten_a_large_state(Kd, V):
    """Keys of few dimensions have overwritten all of it after a dozen tokens: the gradients of a chunk's last keys are of ordinary size, their
    terms 4000 times that.  Granted is four times what the same formula leaves in plain fp32, and the output's rounding."""
    x = _overwritten(64, Kd, V, 65)
    x["state_in"] *= 4
    x["q"] = make(1, 64, 2, 2, Kd, V, True, 1, 66)["q"]
    last = slice(48, 64)
    want = ref(host(x), 1)["dk"][:, last]
    plain = rel_err(_by_chunks(x)[:, last], want)
    assert rel_err(num(run(x, desc(x, 1), want=("dk",))["dk"])[:, last], want) <= 2.0 ** -8 + 4 * plain
