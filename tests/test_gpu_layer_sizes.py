"""The selective scan, the short convolution and the norm at sizes whose launches go round: more work than the workgroups of one take at once."""
import pytest
import torch

from layer_util import DEV, scratch
from paper_2604_04250_amd import binding as K

pytestmark = pytest.mark.gpu


def test_parameter_sums_over_more_columns_than_a_launch_counts_threads_for():
    """Column sums of 5 x 33,554,435 columns: 5.2 million workgroups of 1,024 threads would be more than 2^32.  One token: each gradient is a product."""
    C, k = (1 << 25) + 3, 4
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, dy, state = (torch.randn(s, generator=gen, device=DEV) for s in ((1, 1, C), (1, 1, C), (1, k - 1, C)))
    w = torch.randn((C, k), generator=gen, device=DEV)
    d = K.make_conv_desc(1, 1, C, k)
    dw, db = torch.full_like(w, float("nan")), torch.full((C,), float("nan"), device=DEV)
    K.check(K.cawn_causal_conv_bwd(d, x, w, None, None, state, dy, None, None, dw, db, None, scratch(K.cawn_causal_conv_workspace_bytes(d))))
    assert torch.equal(db, dy[0, 0])
    for i in range(k):
        assert torch.equal(dw[:, i], dy[0, 0] * (state[0, i] if i < k - 1 else x[0, 0])), i
    K.check(K.cawn_causal_conv_bwd(K.make_conv_desc(0, 1, C, k), x, w, None, None, state, dy, None, None, dw, db, None, None))        # sums over nothing
    assert not bool(dw.any()) and not bool(db.any())
