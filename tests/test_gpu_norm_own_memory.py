"""GPU test of the gradients that bra_norm_backward returns: each has memory of its own, so that keeping one keeps no other, and a change of one in place does not
count as a change of the others."""
import pytest
import torch

import paper_2303_08810_amd as bra

pytestmark = pytest.mark.gpu


def test_gradients_share_nothing():
    C = 96
    X, gate, v = torch.randn(4, 9, C, device="cuda"), torch.randn(4, C, device="cuda"), torch.ones(C, device="cuda")
    g = bra.bra_norm_backward(X, v, X, dX=X, Y=X, post_gamma=v, post_beta=v, scale=v, gate=gate)
    assert len({t.untyped_storage().data_ptr() for t in g.values()}) == len(g) == 8
    assert all(t.untyped_storage().nbytes() == t.numel() * 4 for t in g.values())
    before = {k: t._version for k, t in g.items()}
    g["dgamma"].add_(1.0)
    assert [k for k, t in g.items() if t._version != before[k]] == ["dgamma"]
