"""The examples' layers as their callers may call them."""
import importlib.util
import os

import pytest
import torch

from gpu_util import DEV

pytestmark = pytest.mark.gpu

_spec = importlib.util.spec_from_file_location("select_layer", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "select_layer.py"))
E = importlib.util.module_from_spec(_spec)
_spec.loader.exec_module(E)


def _layer(seed):
    torch.manual_seed(seed)
    return E.SelectLayer(48, 136, 12, groups=2, rank=5).to(DEV)


def test_lengths_that_are_a_column_of_a_table():
    layer, x, residual = _layer(1), torch.randn(4, 70, 48, device=DEV), torch.randn(4, 70, 48, device=DEV)
    table = torch.tensor([[70, 9], [0, 9], [1, 9], [33, 9]], dtype=torch.int32, device=DEV)
    results = []
    for lengths in (table[:, 0].clone(), table[:, 0]):
        layer.zero_grad()
        y, h, (conv, ssm) = layer(x, residual, lengths=lengths)
        (y.square().sum() + ssm.sum()).backward()
        results.append([y, h, conv, ssm] + [p.grad.clone() for p in layer.parameters()])
    for a, b in zip(*results):
        assert torch.equal(a, b)
