"""The 64-bit references of the selective scan, the short convolution and the norm against differences of their own forwards (CPU only)."""
import numpy as np
import pytest

import layer_ref as R

STEP = 1e-5
# central differences: the third derivative's share is STEP^2, the rounding's 2^-53 of the sum over STEP
TOL = 1e-7


def _check(value, grads, inputs, rng):
    """value(**inputs) against the gradients in a few directions."""
    for name, g in grads.items():
        for _ in range(2):
            v = rng.standard_normal(inputs[name].shape)
            moved = [value(**{**inputs, name: inputs[name] + s * STEP * v}) for s in (1, -1)]
            want = (moved[0] - moved[1]) / (2 * STEP)
            got = float((g * v).sum())
            assert abs(got - want) <= TOL * (1 + abs(want)), (name, got, want)


@pytest.mark.parametrize("softplus", [True, False])
@pytest.mark.parametrize("G,lengths", [(1, None), (2, [4, 0, 1])])
def test_scan_gradients_are_the_forwards(G, lengths, softplus):
    r = np.random.Generator(np.random.PCG64(5))
    B, L, D, N = 3, 5, 6, 3
    i = dict(x=r.standard_normal((B, L, D)), dt=0.5 * r.standard_normal((B, L, D)), A=-r.uniform(0.2, 2, (D, N)), Bm=r.standard_normal((B, L, G, N)),
             Cm=r.standard_normal((B, L, G, N)), Dk=r.standard_normal(D), z=r.standard_normal((B, L, D)), bias=r.standard_normal(D),
             state_in=r.standard_normal((B, D, N)))
    dy, ds = r.standard_normal((B, L, D)), r.standard_normal((B, D, N))

    def value(**k):
        y, s = R.scan_fwd(lengths=lengths, softplus=softplus, **k)
        return float((y * dy).sum() + (s * ds).sum())

    g = R.scan_bwd(dy=dy, dstate_out=ds, lengths=lengths, softplus=softplus, **i)
    _check(value, dict(x=g["dx"], dt=g["ddt"], A=g["dA"], Bm=g["dBm"], Cm=g["dCm"], Dk=g["dDskip"], z=g["dz"], bias=g["ddt_bias"], state_in=g["dstate_in"]), i, r)


def test_scan_in_two_calls_is_one():
    r = np.random.Generator(np.random.PCG64(6))
    B, L, D, N = 2, 7, 4, 3
    x, dt, z = (r.standard_normal((B, L, D)) for _ in range(3))
    Bm, Cm, A = r.standard_normal((B, L, 1, N)), r.standard_normal((B, L, 1, N)), -r.uniform(0.2, 2, (D, N))
    y, s = R.scan_fwd(x, dt, A, Bm, Cm, z=z)
    y1, s1 = R.scan_fwd(x[:, :3], dt[:, :3], A, Bm[:, :3], Cm[:, :3], z=z[:, :3])
    y2, s2 = R.scan_fwd(x[:, 3:], dt[:, 3:], A, Bm[:, 3:], Cm[:, 3:], z=z[:, 3:], state_in=s1)
    assert np.allclose(np.concatenate([y1, y2], 1), y, rtol=1e-12, atol=1e-12) and np.allclose(s2, s, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("k,lengths", [(4, None), (3, [5, 0, 1]), (4, [2, 1, 0]), (1, None)])
def test_conv_gradients_are_the_forwards(k, lengths, act):
    r = np.random.Generator(np.random.PCG64(7))
    B, L, C = 3, 5, 4
    i = dict(x=r.standard_normal((B, L, C)), w=r.standard_normal((C, k)), bias=r.standard_normal(C), state_in=r.standard_normal((B, k - 1, C)))
    dy, ds = r.standard_normal((B, L, C)), r.standard_normal((B, k - 1, C))

    def value(**kw):
        y, s, _, _ = R.conv_fwd(act=act, lengths=lengths, **kw)
        return float((y * dy).sum() + (s * ds).sum())

    g = R.conv_bwd(dy=dy, dstate_out=ds, act=act, lengths=lengths, **i)
    _check(value, dict(x=g["dx"], w=g["dw"], bias=g["dbias"], **({"state_in": g["dstate_in"]} if k > 1 else {})), i, r)


def test_norm_gradients_are_the_forwards():
    r = np.random.Generator(np.random.PCG64(8))
    i = dict(h=r.standard_normal((3, 7)), w=r.standard_normal(7))
    dy, dh = r.standard_normal((3, 7)), r.standard_normal((3, 7))
    d, dw = R.rms_bwd(i["h"], dy, i["w"], dh)
    _check(lambda h, w: float((R.rms_fwd(h, w)[0] * dy).sum() + (h * dh).sum()), dict(h=d, w=dw), i, r)
