"""GPU tests of the norms' gates: ones behind the gate's leading dimensions wherever the map has ones too, and the gradient of a gate that is absent."""
import pytest
import torch

import paper_2303_08810_amd as bra

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


# the map's leading dimensions, and how many of them the gate has before its ones
@pytest.mark.parametrize("shape,own", [((4, 5, 1), 1), ((4, 1, 6), 1), ((4, 5, 1), 2), ((4, 1, 1), 1), ((1, 5, 1), 0), ((4, 5, 1), 0), ((2, 3, 1, 4, 1), 2), ((1, 1, 1), 0), ((4, 5, 6), 1)])
def test_ones_behind_the_leading_dimensions(shape, own):
    C = 64
    g = torch.Generator().manual_seed(len(shape) + own)
    r = lambda *s: torch.randn(*s, generator=g)
    X, Y, dN = (r(*shape, C).to(BF16).cuda() for _ in range(3))
    gate, gamma = r(*shape[:own], C).to(BF16).cuda(), r(C).cuda()
    R, N = bra.bra_norm_forward(X, gamma, Y=Y, gate=gate)
    want = bra.bra_norm_backward(R, gamma, dN, Y=Y, gate=gate)
    for ones in range(len(shape) - own + 1):
        wide = gate.view(*shape[:own], *([1] * ones), C)
        R1, N1 = bra.bra_norm_forward(X, gamma, Y=Y, gate=wide)
        assert torch.equal(R, R1) and torch.equal(N, N1), ones
        got = bra.bra_norm_backward(R, gamma, dN, Y=Y, gate=wide)
        assert got["dgate"].shape == wide.shape
        assert all(torch.equal(got[k].view(want[k].shape), want[k]) for k in want), ones


def test_gates_that_do_not_lead():
    X, gamma = torch.zeros(4, 5, 1, 64, dtype=BF16, device="cuda"), torch.ones(64, device="cuda")
    for bad in ((5,), (1, 5), (4, 6), (4, 5, 2), (4, 1, 2), (4, 5, 1, 2), (2,)):
        with pytest.raises(ValueError):
            bra.bra_norm_forward(X, gamma, Y=X, gate=torch.zeros(*bad, 64, dtype=BF16, device="cuda"))
