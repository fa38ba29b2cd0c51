"""GPU tests of the norms around a residual sum and their gradients against 64 bits: every size of a row's team, rows that no piece
divides, gates for every grouping, absent parts, rows of zeros."""
import itertools

import pytest
import torch

import paper_2303_08810_amd as bra
from norm_util import check_backward, check_forward

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def make(shape, gate_dims, C, dtype, seed, post=True):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    put = lambda t, d=F32: t.to(d).cuda()
    X, Y, dN, dR = (put(r(*shape, C) + 0.5 * r(C), dtype) for _ in range(4))
    P = dict(gamma=put(1 + 0.1 * r(C)), beta=put(0.1 * r(C)), scale=put(0.5 + 0.1 * r(C)))
    if post:
        P.update(post_gamma=put(1 + 0.1 * r(C)), post_beta=put(0.1 * r(C)))
    if gate_dims is not None:
        P["gate"] = put(r(*shape[:gate_dims], C), dtype)
    return X, Y, dN, dR, P


def without_beta(P):
    return {k: v for k, v in P.items() if k != "beta"}


def run(shape, gate_dims, C, dtype, kind, post, seed, eps=1e-6):
    X, Y, dN, dR, P = make(shape, gate_dims, C, dtype, seed, post)
    print(f"norm {shape} x {C} gate {gate_dims} {dtype} {kind} post={post}", flush=True)
    R, N = bra.bra_norm_forward(X, Y=Y, kind=kind, eps=eps, **P)
    check_forward(R, N, X, Y, P, kind, eps)
    B = {k: v for k, v in P.items() if k != "beta"}
    grads = bra.bra_norm_backward(R, dN=dN, dX=dR, Y=Y, kind=kind, eps=eps, **B)
    check_backward(grads, R, Y, P, dN, dR, kind, eps)
    again = bra.bra_norm_backward(R, dN=dN, dX=dR, Y=Y, kind=kind, eps=eps, **B)
    assert all(torch.equal(grads[k], again[k]) for k in grads)


CHANNELS = [1, 3, 8, 16, 24, 40, 64, 99, 128, 192, 256, 512, 520, 768, 1000, 1024, 1032, 2048, 3000, 4096, 8192]


@pytest.mark.parametrize("C", CHANNELS)
def test_channels(C):
    for i, (kind, post) in enumerate(itertools.product(("layer", "rms"), (True, False))):
        run((3, 37), 1, C, (BF16, F32)[(C + i) % 2], kind, post, seed=C + i)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape,gate_dims", [((1,), None), ((1,), 1), ((2, 1), 0), ((5, 7), 2), ((1000, 3), 1), ((4, 5000), 1), ((3, 17, 19), 2), ((3, 17, 19), 3), ((7, 100), 1),
                                             ((20000,), None), ((700, 40), 1), ((9000, 2), 1)])
def test_groupings(shape, gate_dims, dtype):
    for C, kind, post in ((64, "layer", True), (192, "rms", False), (30, "layer", False)):
        run(shape, gate_dims, C, dtype, kind, post, seed=len(shape) + C)


def test_gate_with_ones():
    X, Y, dN, dR, P = make((4, 5, 6), 1, 64, BF16, 5)
    R, N = bra.bra_norm_forward(X, Y=Y, **P)
    P["gate"] = P["gate"].view(4, 1, 1, 64)
    R1, N1 = bra.bra_norm_forward(X, Y=Y, **P)
    assert torch.equal(R, R1) and torch.equal(N, N1)
    g = bra.bra_norm_backward(R, dN=dN, Y=Y, **without_beta(P))
    assert g["dgate"].shape == (4, 1, 1, 64)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_absent_parts(dtype):
    X, Y, dN, dR, P = make((33,), None, 96, dtype, 8)
    N = bra.bra_norm_forward(X, P["gamma"])
    check_forward(None, N, X, None, {"gamma": P["gamma"]}, "layer", 1e-6)
    R = bra.bra_norm_forward(X, Y=Y)
    check_forward(R, None, X, Y, {}, "layer", 1e-6)
    R = bra.bra_norm_forward(X, Y=Y, post_gamma=P["post_gamma"], kind="rms")
    check_forward(R, None, X, Y, {"post_gamma": P["post_gamma"]}, "rms", 1e-6)
    only = {"gamma": P["gamma"]}
    check_backward(bra.bra_norm_backward(X, dN=dN, **only), X, None, only, dN, None, "layer", 1e-6)
    check_backward(bra.bra_norm_backward(X, dN=dN, dX=dR, **only), X, None, only, dN, dR, "layer", 1e-6)
    check_backward(bra.bra_norm_backward(R, dX=dR, Y=Y), R, Y, {}, None, dR, "layer", 1e-6)
    some = {"post_gamma": P["post_gamma"], "scale": P["scale"]}
    check_backward(bra.bra_norm_backward(R, dX=dR, Y=Y, kind="rms", **some), R, Y, some, None, dR, "rms", 1e-6)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_rows_of_zeros_and_of_one_value(kind):
    X, Y, dN, dR, P = make((6,), 1, 64, F32, 9)
    X[1] = 0
    Y[1] = 0
    X[2] = 3.0
    Y[2] = -2.0
    P["post_beta"].zero_()
    R, N = bra.bra_norm_forward(X, Y=Y, kind=kind, **P)
    check_forward(R, N, X, Y, P, kind, 1e-6)
    assert torch.equal(N[1], P["beta"])
    g = bra.bra_norm_backward(R, dN=dN, dX=dR, Y=Y, kind=kind, **without_beta(P))
    check_backward(g, R, Y, P, dN, dR, kind, 1e-6)


def test_no_rows():
    X, Y, dN, dR, P = make((0, 5), 1, 64, BF16, 3)
    R, N = bra.bra_norm_forward(X, Y=Y, **P)
    assert R.shape == N.shape == X.shape
    g = bra.bra_norm_backward(R, dN=dN, dX=dR, Y=Y, **without_beta(P))
    assert all(not g[k].any() for k in ("dgamma", "dbeta", "dscale", "dpost_gamma", "dpost_beta"))
    X, Y, dN, dR, P = make((3, 0), 1, 64, BF16, 3)
    g = bra.bra_norm_backward(X, dN=dN, dX=dR, Y=Y, **without_beta(P))
    assert g["dgate"].shape == (3, 64) and not g["dgate"].any() and not g["dscale"].any()


def test_in_place():
    X, Y, dN, dR, P = make((50,), 1, 256, BF16, 4)
    R, N = bra.bra_norm_forward(X, Y=Y, **P)
    X1 = X.clone()
    R1, N1 = bra.bra_norm_forward(X1, Y=Y, out=X1, **P)
    assert R1 is X1 and torch.equal(R, R1) and torch.equal(N, N1)


def test_unaligned_views():
    C = 64
    base = torch.randn(2 * 40 * C + 8, device="cuda").to(BF16)
    X, Y = base[3:3 + 40 * C].view(40, C), base[3 + 40 * C:3 + 80 * C].view(40, C)
    P = dict(gamma=torch.randn(C + 1, device="cuda")[1:], scale=torch.randn(C + 3, device="cuda")[3:])
    R, N = bra.bra_norm_forward(X, Y=Y, **P)
    check_forward(R, N, X, Y, P, "layer", 1e-6)
    g = bra.bra_norm_backward(X, dN=Y, Y=Y, **P)
    check_backward(g, X, Y, P, Y, None, "layer", 1e-6)
