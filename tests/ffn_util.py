"""The gated feed-forward block and its gradients in 64 bits, and how far a result may be off.

Bounds are worst cases by elements: a sum of products formed in float32 is off by at most (terms + 8) 2^-24 of the sum of its
terms' magnitudes, a rounding by half a step (`UNIT`) of what is rounded, and an intermediate's error goes through the next
product with that product's magnitudes.  The activations' own error (the polynomial of Phi: 7e-7 of the value for |g| > 1, 7e-7
absolute below; exp2 and rcp: a few 2^-24) is `ACT`.  The 2-norm of the whole error is held to the roundings' own size: two independent
ones of rms UNIT / sqrt(3) are below UNIT, the float32 sums' to 64 2^-24 (they grow like the square root of the terms)."""
import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
F32 = 2.0 ** -24
ACT = 1.5e-6


def make(M, C, h, dtype, bias, seed, device="cuda"):
    g = torch.Generator(device="cpu")
    g.manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    X, W1, W2, dY = r(M, C), r(C, 2 * h) / C ** 0.5, r(h, C) / h ** 0.5, r(M, C)
    b1, b2 = (r(2 * h) * 0.3, r(C) * 0.3) if bias else (None, None)
    put = lambda t, d: None if t is None else t.to(d).to(device)
    return put(X, dtype), put(W1, dtype), put(W2, dtype), put(dY, dtype), put(b1, torch.float32), put(b2, torch.float32)


def act64(g, act):
    """F, act and its slope."""
    if act == "silu":
        f = torch.sigmoid(g)
        return g * f, f + g * f * (1 - f)
    f = 0.5 * torch.erfc(-g / math.sqrt(2.0))
    return g * f, f + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


def forward64(X, W1, W2, b1, b2, act):
    """Y and G | U, each with its bound but for the last rounding."""
    X, W1, W2 = X.double(), W1.double(), W2.double()
    h = W2.shape[0]
    P, Pm = X @ W1, X.abs() @ W1.abs()
    if b1 is not None:
        P, Pm = P + b1.double(), Pm + b1.double().abs()
    eP = (X.shape[1] + 8) * F32 * Pm
    (a, slope), U = act64(P[:, :h], act), P[:, h:]
    A = a * U
    # |slope| <= 1.13 for both
    eA = 1.13 * eP[:, :h] * U.abs() + a.abs() * eP[:, h:] + ACT * (1 + a.abs()) * U.abs()
    return P, eP, A, eA, W2


def check(got, ref, bound, unit, name, norm=None):
    """Elementwise, the result's own rounding included, and the whole."""
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    got = got.double()
    assert torch.isfinite(got).all(), name
    d, most = (got - ref).abs(), bound + unit * (ref.abs() + bound) + 1e-37
    worst = float((d / most).max()) if d.numel() else 0.0
    assert worst <= 1.0, (name, worst)
    if norm is not None and d.numel() >= 64:
        rel = float(d.norm() / ref.norm())
        assert rel <= norm, (name, rel, norm)


def norm_bound(dtype):
    return UNIT[torch.bfloat16] if dtype == torch.bfloat16 else 64 * F32


def check_forward(out, X, W1, W2, b1, b2, act, pre=None):
    dt = X.dtype
    u = UNIT[dt]
    P, eP, A, eA, W = forward64(X, W1, W2, b1, b2, act)
    Y, mag = A @ W, (A.abs() + eA) @ W.abs()
    eY = (eA + u * (A.abs() + eA)) @ W.abs() + (W.shape[0] + 8) * F32 * mag
    if b2 is not None:
        Y = Y + b2.double()
        eY = eY + F32 * Y.abs()
    check(out, Y, eY, u, "Y", norm_bound(dt))
    if pre is not None:
        check(pre, P, eP, u, "pre", norm_bound(dt))


def check_backward(grads, X, W1, W2, dY, b1, act, pre=None, grad_dtype=None):
    dt = X.dtype
    u, h = UNIT[dt], W2.shape[0]
    P, eP, A, eA, W2d = forward64(X, W1, W2, b1, None, act)
    if pre is not None:
        P, eP = pre.double(), torch.zeros_like(eP)
        a, slope = act64(P[:, :h], act)
        A, eA = a * P[:, h:], ACT * (1 + a.abs()) * P[:, h:].abs()
    (a, slope), U = act64(P[:, :h], act), P[:, h:]
    Xd, W1d, dYd = X.double(), W1.double(), dY.double()
    dA, eD = dYd @ W2d.t(), (X.shape[1] + 8) * F32 * (dYd.abs() @ W2d.abs().t())
    dG, dU = dA * U * slope, dA * a
    # |act''| <= 0.8 for both
    eG = (eD * U.abs() + dA.abs() * eP[:, h:]) * slope.abs() + dA.abs() * U.abs() * (0.8 * eP[:, :h] + ACT * (1 + slope.abs()))
    eU = eD * a.abs() + dA.abs() * (1.13 * eP[:, :h] + ACT * (1 + a.abs()))
    dP, eS = torch.cat([dG, dU], 1), torch.cat([eG, eU], 1)
    eR = eS + u * (dP.abs() + eS)                       # as it goes into the next products
    M, gu = X.shape[0], UNIT[grad_dtype or dt]
    total = lambda e, ref_mag, n: e + (n + 8) * F32 * ref_mag
    n = norm_bound(dt)
    check(grads[0], dP @ W1d.t(), total(eR @ W1d.abs().t(), (dP.abs() + eR) @ W1d.abs().t(), 2 * h), u, "dX", n)
    check(grads[1], Xd.t() @ dP, total(Xd.abs().t() @ eR, Xd.abs().t() @ (dP.abs() + eR), M), gu, "dW1", n)
    eA = eA + u * (A.abs() + eA)
    check(grads[2], A.t() @ dYd, total(eA.t() @ dYd.abs(), (A.abs() + eA).t() @ dYd.abs(), M), gu, "dW2", n)
    if len(grads) > 3:
        check(grads[3], dP.sum(0), total(eR.sum(0), (dP.abs() + eR).sum(0), M), gu, "db1", n)
        check(grads[4], dYd.sum(0), (M + 8) * F32 * dYd.abs().sum(0), gu, "db2", n)
