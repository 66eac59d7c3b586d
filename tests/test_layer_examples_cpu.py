"""What the examples' layers hand to the entry points (CPU only: the calls are recorded, not made)."""
import importlib.util
import os

import pytest
import torch

from paper_2604_04250_amd import binding as K

EXAMPLES = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples")


def _load(name):
    spec = importlib.util.spec_from_file_location(name, os.path.join(EXAMPLES, name + ".py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


S, D = _load("select_layer"), _load("delta_layer")


@pytest.fixture
def calls(monkeypatch):
    """Names of the entry points called, with their arguments; nothing is written."""
    made = []

    def record(name):
        def call(*args, **kw):
            made.append((name, args))
            return K.CAWN_OK
        return call

    for name in K._OPS:
        monkeypatch.setattr(K, name, record(name))
    monkeypatch.setattr(S, "_scratch", lambda n, device: torch.empty(16, dtype=torch.uint8))        # (nothing is written there)
    monkeypatch.setattr(D, "_scratch", lambda n, device: torch.empty(16, dtype=torch.uint8))
    return made


def _scan_args(grad=False, B=3, L=5, C=8, N=4, G=2):
    new = lambda *s: torch.randn(s).requires_grad_(grad)  # noqa: E731
    return [new(B, L, C), new(B, L, C), new(C, N), new(B, L, G, N), new(B, L, G, N), new(C), new(B, L, C), new(C), new(B, C, N)]


def _conv_args(grad=False, B=3, L=5, C=8, k=4):
    new = lambda *s: torch.randn(s).requires_grad_(grad)  # noqa: E731
    return [new(B, L, C), new(C, k), new(C), new(B, k - 1, C)]


def _delta_args(grad=False, B=3, L=5, H=2, W=16):
    new = lambda *s: torch.randn(s).requires_grad_(grad)  # noqa: E731
    return [new(B, L, H, W), new(B, L, H, W), new(B, L, H, W), new(B, L, H), new(B, L, H), new(B, H, W, W)]


# an autograd function, its tensors, and the place of lengths in its calls forward and backward (behind the descriptor)
OPS = [(S.ShortConv, _conv_args, 3, 3), (S.SelectiveScan, _scan_args, 8, 8), (D.DeltaRule, _delta_args, 5, 5)]


@pytest.mark.parametrize("f,args,fwd,bwd", OPS)
def test_lengths_with_a_stride_are_handed_on_as_dense_ones(calls, f, args, fwd, bwd):
    pairs = torch.tensor([[5, 100], [0, 100], [2, 100]], dtype=torch.int32)
    out, _ = f.apply(*args(True), pairs[:, 0])
    out.sum().backward()
    assert len(calls) == 2
    for (name, a), at in zip(calls, (fwd, bwd)):
        got = a[1 + at]
        assert got.is_contiguous() and got.tolist() == [5, 0, 2], name


@pytest.mark.parametrize("f,args,fwd,bwd", OPS)
def test_lengths_overwritten_before_the_backward_are_an_error(calls, f, args, fwd, bwd):
    lengths = torch.tensor([5, 0, 2], dtype=torch.int32)
    out, _ = f.apply(*args(True), lengths)
    lengths.fill_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()
    assert len(calls) == 1


LENGTHS = torch.tensor([5, 0, 2], dtype=torch.int32)
X, W = torch.randn(6, 8), torch.randn(8)
# functions, what they take as it should be, how many of it are tensors, and what nothing else has to agree with: a tensor's axis
TAKES = [(S.ShortConv, [*_conv_args(), LENGTHS], 5, (0, 1)), (S.SelectiveScan, [*_scan_args(), LENGTHS], 10, None), (S.AddNorm, [X, X, W, 1e-5], 3, None),
         (D.DeltaRule, [*_delta_args(), LENGTHS], 7, None), (D.HeadNorm, [X, W, W, 2], 3, (0, 0)), (D.DropoutAdd, [X, X, torch.zeros(2, dtype=torch.int64), 0.1], 3, None)]


@pytest.mark.parametrize("f,args,n,free", TAKES)
def test_sizes_that_do_not_agree_are_refused(calls, f, args, n, free):
    """Every tensor in turn one entry shorter along every axis: an entry point would read beyond its end, or the others would be read beyond theirs."""
    f.apply(*args)
    assert len(calls) == 1
    for i in range(n):
        for axis in range(args[i].dim()):
            if (i, axis) == free:
                continue
            with pytest.raises(ValueError):
                f.apply(*args[:i], args[i].narrow(axis, 0, args[i].shape[axis] - 1), *args[i + 1:])
    assert len(calls) == 1


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
@pytest.mark.parametrize("L", [1, 40])
def test_without_gradients_no_checkpoint_is_made(calls, mode, L):
    """The scan of a call without one goes token by token where the tokens are few, and writes no states for a backward where they are many."""
    layer = S.SelectLayer(12, 8, 4)
    x = torch.randn(2, L, 12)
    ckpt = lambda: [a[13] for name, a in calls if name == "cawn_selective_scan_fwd"]  # noqa: E731
    with mode():
        layer(x, torch.zeros_like(x))
    assert ckpt() == [None]
    layer(x, torch.zeros_like(x))
    assert ckpt()[1] is not None
    for p in layer.parameters():
        p.requires_grad_(False)
    layer(x, torch.zeros_like(x))
    assert ckpt()[2] is None
