"""GPU tests of the norms' gradients over no rows: zeros, whatever the vectors hold and however many groups there are."""
import pytest
import torch

import paper_2303_08810_amd as bra

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.mark.parametrize("value", [float("inf"), float("nan"), -2.0])
def test_zeros_whatever_scale_is(value):
    X, gate = torch.zeros(3, 0, 64, dtype=BF16, device="cuda"), torch.full((3, 64), value, dtype=BF16, device="cuda")
    vec = {k: torch.full((64,), value, device="cuda") for k in ("gamma", "post_gamma", "post_beta", "scale")}
    g = bra.bra_norm_backward(X, dN=X, dX=X, Y=X, gate=gate, **vec)
    for k in ("dgate", "dgamma", "dbeta", "dscale", "dpost_gamma", "dpost_beta"):
        assert (g[k] == 0).all(), k


def test_many_groups_of_no_rows():
    """2^32 values of the gate's gradient, more than a launch has threads."""
    groups, C = (1 << 21) + 5, 2048
    X, gate = torch.zeros(groups, 0, C, dtype=BF16, device="cuda"), torch.zeros(groups, C, dtype=BF16, device="cuda")
    # (what the allocator hands out for dgate has held something else)
    dirty = torch.full_like(gate, 7.0)
    del dirty
    g = bra.bra_norm_backward(X, torch.ones(C, device="cuda"), X, Y=X, gate=gate)
    assert g["dgate"].shape == gate.shape and float(g["dgate"].abs().amax()) == 0.0
    del g, gate
    torch.cuda.empty_cache()
