"""GELU behind the group norm keeps its relative digits in the tail, where it is a small number times the density."""
import math

import numpy as np
import pytest
import torch

from gpu_util import DEV
from paper_2604_04250_amd import binding as K

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 3])
def test_gelu_and_its_slope_relative_to_themselves(T):
    """A weight of 0 makes the bias the activation's argument, exactly.  The exponential's argument is z^2 / 2 with two roundings of 2^-24 each, 4e-6 of
    the result at |z| = 8; the rest are ten roundings or so of 2^-24."""
    z = np.concatenate([np.linspace(-8, 8, 4001), [-1e-3, -1e-6, 1e-6, -2.5, -4.9999, 30.0]]).astype(np.float32)
    C = z.size
    r = np.random.Generator(np.random.PCG64(3))
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(DEV)  # noqa: E731
    d = K.make_norm_desc(1, T, C, 1, act=2)
    x, dy, w, b = dev(r.standard_normal((1, T, C))), dev(np.ones((1, T, C))), dev(np.zeros(C)), dev(z)
    y, dx, stats, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty(1, 1, 2, device=DEV), torch.empty(C, device=DEV), torch.empty(C, device=DEV)
    ws = torch.empty(max(256, K.cawn_group_norm_workspace_bytes(d)), dtype=torch.uint8, device=DEV)
    K.check(K.cawn_group_norm_fwd(d, x, w, b, y, stats, ws))
    K.check(K.cawn_group_norm_bwd(d, x, w, b, stats, dy, dx, dw, db, ws))
    torch.cuda.synchronize()
    z = z.astype(np.float64)
    below = np.array([0.5 * math.erfc(-v / math.sqrt(2)) for v in z])
    density = np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    want, slope = z * below, below + z * density
    tol = z * z / 2 * 2 * 2.0 ** -24 + 16 * 2.0 ** -24
    assert np.all(np.abs(y[0].double().cpu().numpy() - want) <= tol * np.abs(want))
    assert np.all(np.abs(db.double().cpu().numpy() / T - slope) <= tol * (below + np.abs(z) * density))
