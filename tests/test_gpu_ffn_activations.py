"""GPU tests of the float32 gated block's activations by themselves, far into their tails and close to zero, on every path of the forward and in the
gradients.

The inputs make G, U and the products around the activation exact: X has g and a 1 in a row, W1 powers of two, W2 ones on a diagonal, so that
Y[m, j] = act(g_m s_j).  What is left is the activation's own error, relative to its value, with u = 2^-24:
    SiLU   the exponent log2(e) g is rounded twice (2 |g| u of the result), the power of two and the reciprocal are within 2 u each, three
           more operations within u each: (2 |g| + 8) u
    GELU   Phi(g) = erfc(-g / sqrt 2) / 2: the argument is off by 2 u of itself, which erfc takes times at most g^2 + 1; erfc itself is within 16
           units (32 u), two products 2 u: (2 g^2 + 36) u
and, where results get smaller than 2^-126, a unit of the subnormal numbers."""
import math

import pytest
import torch

import paper_2303_08810_amd as bra

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def act64(g, act):
    if act == "silu":
        f = torch.sigmoid(g)
        return g * f, f, g * f * (1 - f)
    f = 0.5 * torch.erfc(-g / math.sqrt(2.0))
    return g * f, f, g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


def units(g, act):
    return (2 * g.abs() + 8 if act == "silu" else 2 * g * g + 36) * U


# few rows, tiles, tiles whose long contraction is shared out
PATHS = [(5, 16, 24), (100, 64, 96), (300, 64, 128), (2500, 128, 128), (129, 768, 2048), (700, 331, 1401)]


def inputs(M, C, h, low):
    g = torch.linspace(-low, 4.0, M, dtype=torch.float32)
    X, W1, W2 = torch.zeros(M, C), torch.zeros(C, 2 * h), torch.zeros(h, C)
    X[:, 0], X[:, 1] = g, 1.0
    n = min(C, h)
    s = 2.0 ** -torch.arange(n).remainder(9).float()        # 1 to 2^-8
    W1[0, :n], W1[1, h:h + n] = s, 1.0
    W2[:n, :n] = torch.eye(n)
    return X.cuda(), W1.cuda(), W2.cuda(), (g[:, None] * s).double().cuda(), s.double().cuda(), n


@pytest.mark.parametrize("act,low", [("silu", 60.0), ("gelu", 12.0)])
@pytest.mark.parametrize("M,C,h", PATHS)
def test_forward(M, C, h, act, low):
    X, W1, W2, G, s, n = inputs(M, C, h, low)
    print(f"activations forward {M} x {C} x {h} {act}", flush=True)
    Y, pre = bra.bra_ffn_forward(X, W1, W2, act=act, want_pre=True)
    assert torch.equal(pre[:, :n].double(), G) and (pre[:, h:h + n] == 1).all()
    want = act64(G, act)[0]
    off = (Y[:, :n].double() - want).abs() / (units(G, act) * want.abs() + 2.0 ** -126)
    assert float(off.max()) <= 1.0, (float(off.max()), float(G.flatten()[off.argmax()]))


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("act,low", [("silu", 60.0), ("gelu", 12.0)])
@pytest.mark.parametrize("M,C,h", PATHS)
def test_gradients(M, C, h, act, low, given):
    """dY has a 1 in one column: dW2 there is the sum of A over rows, of one row where the others' dY is 0; dX[m, 0] is the slope."""
    X, W1, W2, G, s, n = inputs(M, C, h, low)
    print(f"activations gradients {M} x {C} x {h} {act} given={given}", flush=True)
    pre = bra.bra_ffn_forward(X, W1, W2, act=act, want_pre=True)[1] if given else None
    a, f, rest = act64(G, act)
    for row in (0, M // 3, M - 1):
        dY = torch.zeros_like(X)
        dY[row, 0] = 1.0
        dW2 = bra.bra_ffn_backward(X, W1, W2, dY, pre=pre, act=act)[2]
        off = (dW2[:n, 0].double() - a[row]).abs() / (units(G[row], act) * a[row].abs() + 2.0 ** -126)
        assert float(off.max()) <= 1.0, (row, float(off.max()))
    for j in (0, min(7, n - 1)):
        dY = torch.zeros_like(X)
        dY[:, j] = 1.0
        dX = bra.bra_ffn_backward(X, W1, W2, dY, pre=pre, act=act)[0]
        # dG = slope goes through W1[0] alone.  SiLU: 1 - f is off by u and f's error, of the magnitude of f where that is small; GELU: the density's exponent
        # g^2 / 2 is rounded three times (3 g^2 / 2 u); twice the units cover both
        slope, size = f + rest, f + rest.abs() + (f * f * G.abs() if act == "silu" else 0)
        off = (dX[:, 0].double() - (slope * s)[:, j]).abs() / (2 * (units(G, act) * size * s)[:, j] + 2.0 ** -126)
        assert float(off.max()) <= 1.0, (j, float(off.max()))


@pytest.mark.parametrize("small", [1.0, 0.1, 0.01])
@pytest.mark.parametrize("M,C,h", PATHS)
def test_small_pre_activations(M, C, h, small):
    """Normally distributed G of any scale.  The 2-norm of the whole error: G, U and Y are sums whose rounding errors grow like the square root of their
    terms, below sqrt(4096) = 64 of 2^-24 with the six products' own."""
    g = torch.Generator().manual_seed(M + C)
    r = lambda *s: torch.randn(*s, generator=g)
    X, W1, W2 = (small * r(M, C)).cuda(), (r(C, 2 * h) / C ** 0.5).cuda(), (r(h, C) / h ** 0.5).cuda()
    Y = bra.bra_ffn_forward(X, W1, W2, act="gelu").double()
    P = X.double() @ W1.double()
    want = (act64(P[:, :h], "gelu")[0] * P[:, h:]) @ W2.double()
    rel = float((Y - want).norm() / want.norm())
    assert rel <= 16 * U, rel / U
