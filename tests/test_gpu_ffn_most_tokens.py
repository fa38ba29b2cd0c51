"""GPU test of the gated block's gradients with as many tokens as they take, 2^30 - 1: their tiles make 2^32 threads, more than a launch has."""
import pytest
import torch

import paper_2303_08810_amd as bra

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def test_most_tokens():
    """All rows but some at both ends and in the middle are 0, and so are their dY: the weights' gradients are those of the rows that are left, but for the order
    of their sums, and these rows' dX is what they have alone."""
    M, C, h, n = (1 << 30) - 1, 8, 8, 300
    g = torch.Generator().manual_seed(30)
    r = lambda *s: torch.randn(*s, generator=g)
    W1, W2, few = (r(C, 2 * h) / C ** 0.5).to(BF16).cuda(), (r(h, C) / h ** 0.5).to(BF16).cuda(), r(3 * n, C).to(BF16).cuda()
    places = torch.cat([torch.arange(n), (1 << 29) - 100 + torch.arange(n), M - n + torch.arange(n)]).cuda()
    X = torch.zeros(M, C, dtype=BF16, device="cuda")
    X[places] = few
    print("ffn gradients of 2^30 - 1 tokens", flush=True)
    dX, dW1, dW2 = bra.bra_ffn_backward(X, W1, W2, X, grad_dtype=torch.float32)
    want = bra.bra_ffn_backward(few, W1, W2, few, grad_dtype=torch.float32)
    # the same operations on the same values, one rounding to bf16
    assert float((dX[places].double() - want[0].double()).abs().max()) <= 2.0 ** -8 * float(want[0].double().abs().max())
    # each a sum of 900 products in float32, in another order: 900 2^-24 of the magnitudes, which are below 900 times the largest
    for got, w in ((dW1, want[1]), (dW2, want[2])):
        assert float((got.double() - w.double()).norm() / w.double().norm()) <= 900 * 2.0 ** -24
    zero = torch.ones(1 << 20, dtype=torch.bool, device="cuda")
    zero[:n] = False
    assert not dX[: 1 << 20][zero].any()
    del X, dX
    torch.cuda.empty_cache()
