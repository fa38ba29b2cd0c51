"""Checks of attention in float32 that notice a lost term: six products of three bf16 terms to an operand, x = hi + mid + lo, give a product to 2^-23 of itself; without the
least of them, mid mid, it is off by up to 2^-18, without hi lo or lo hi by 2^-17.

Each check takes an `att` with forward(Q, K, V, k_lens, scale) -> (O, lse) and backward(Q, K, V, O, lse, dO, k_lens, scale) -> (dQ, dK, dV) and inputs whose result has one
product in it.  Steps of 2^-24 that the bounds count: what three terms leave of a product and its sums in the matrix instruction 5 (half a step for the
operands' remainders, half for the products left out, four for the last two additions, should they cut off), a rounding 1, a constant 1, 2^x 2."""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24


def grid(*shape, g, device):
    """Values with all of their 24 bits, in +-[1, 2)."""
    x = 1 + torch.randint(0, 1 << 23, shape, generator=g).float() * 2.0 ** -23
    return (x * (2 * torch.randint(0, 2, shape, generator=g) - 1)).to(device)


def lens_of(n, B, device):
    return torch.full((B,), n, dtype=torch.int32, device=device)


def within(got, want, off, what):
    worst = float(((got.double() - want).abs() / off).max())
    assert worst <= 1, (what, worst)


def setting(B, Nq, Nk, H, d, device, seed):
    g = torch.Generator().manual_seed(seed)
    zeros = lambda n: torch.zeros(B, n, H, d, device=device)
    return g, zeros(Nq), zeros(Nk), zeros(Nk), (lambda *s: grid(*s, g=g, device=device))


def scores(att, B, Nq, Nk, H, d, device="cuda", seed=0):
    """One key, one channel: lse is the score.  Product 5, scale log2 e 2, the maximum 1, back from powers of two 2; log 2^-21."""
    g, Q, K, V, rand = setting(B, Nq, Nk, H, d, device, seed)
    Q[..., d // 3] = 4 * rand(B, Nq, H)
    K[:, 0, :, d // 3] = 4 * rand(B, H)
    _, lse = att.forward(Q, K, V, lens_of(1, B, device), 1.0)
    want = (Q.double()[..., d // 3] * K.double()[:, :1, :, d // 3]).transpose(1, 2)
    within(lse, want, 16 * U * want.abs() + 8 * U, "scores")


def values(att, B, Nq, Nk, H, d, device="cuda", seed=1):
    """One key: O is its value.  The last two additions 4, the weight in the sum that divides, its reciprocal and their product 3."""
    g, Q, K, V, rand = setting(B, Nq, Nk, H, d, device, seed)
    V[:, 0] = rand(B, H, d)
    O, _ = att.forward(Q, K, V, lens_of(1, B, device), 1.0)
    want = V.double()[:, :1].expand(-1, Nq, -1, -1)
    within(O, want, 8 * U * want.abs(), "values")


def weights(att, B, Nq, Nk, H, d, device="cuda", seed=2):
    """Two keys, scores 0 and -a of few bits, a value for the second: O = e^-a v / (1 + e^-a).  Exponents up to 3 log2 e: 5 for their rounding and the constant's; 2^x 2, product 5, sum 1,
    reciprocal and product 3."""
    g, Q, K, V, rand = setting(B, Nq, Nk, H, d, device, seed)
    a = torch.randint(8, 193, (B, Nq, H), generator=g).double().to(device) / 64
    Q[..., 0] = a.float()
    K[:, 1, :, 0] = -1.0
    V[:, 1] = rand(B, H, d)
    O, _ = att.forward(Q, K, V, lens_of(2, B, device), 1.0)
    want = (torch.exp(-a) / (1 + torch.exp(-a)))[..., None] * V.double()[:, 1:2]
    within(O, want, 24 * U * want.abs(), "weights")


def query_gradients(att, B, Nq, Nk, H, d, device="cuda", seed=3):
    """Scores and lse zero, O zero: P = 1 and dS = dO V, one channel of either; dQ = dS K.  Two products 10.  (Two keys, the second zero: a row that sees one has dS = 0.)"""
    g, Q, K, V, rand = setting(B, Nq, Nk, H, d, device, seed)
    dO = torch.zeros_like(Q)
    dO[..., d // 2] = rand(B, Nq, H)
    V[:, 0, :, d // 2] = rand(B, H)
    K[:, 0] = rand(B, H, d)
    dQ, _, _ = att.backward(Q, K, V, torch.zeros_like(Q), torch.zeros(B, H, Nq, device=device), dO, lens_of(2, B, device), 1.0)
    want = dO.double()[..., d // 2:d // 2 + 1] * V.double()[:, :1, :, d // 2:d // 2 + 1] * K.double()[:, :1]
    within(dQ, want, 16 * U * want.abs(), "dQ")


def one_row(x):
    """Of a tensor [B, Nq, H, d]: a row of each sequence and head, others zero."""
    B, N, H, _ = x.shape
    at = (torch.arange(B, device=x.device)[:, None] * 7 + torch.arange(H, device=x.device) * 3) % N
    keep = torch.zeros(B, N, H, 1, device=x.device).scatter_(1, at[:, None, :, None], 1.0)
    return x * keep, at


def row(x, at):
    return x.double().gather(1, at[:, None, :, None].expand(-1, 1, -1, x.shape[3]))


def key_gradients(att, B, Nq, Nk, H, d, device="cuda", seed=4):
    """The same with keys zero, queries that are not, and dO in one row: dK = dS Q."""
    g, Q, K, V, rand = setting(B, Nq, Nk, H, d, device, seed)
    Q = rand(B, Nq, H, d)
    dO, at = one_row(rand(B, Nq, H, d))
    dO[..., :d // 2] = 0
    dO[..., d // 2 + 1:] = 0
    V[:, :, :, d // 2] = rand(B, Nk, H)
    n = min(Nk, 5)
    _, dK, _ = att.backward(Q, K, V, torch.zeros_like(Q), torch.zeros(B, H, Nq, device=device), dO, lens_of(n, B, device), 1.0)
    want = row(dO, at)[..., d // 2:d // 2 + 1] * V.double()[:, :n, :, d // 2:d // 2 + 1] * row(Q, at)
    within(dK[:, :n], want, 16 * U * want.abs(), "dK")


def value_gradients(att, B, Nq, Nk, H, d, device="cuda", seed=5):
    """Scores 0 and -a as in weights, dO in one row: dV = P dO.  Exponents with lse 10, 2^x 2, product 5."""
    g, Q, K, V, rand = setting(B, Nq, Nk, H, d, device, seed)
    dO, at = one_row(rand(B, Nq, H, d))
    a = torch.randint(8, 193, (B, Nq, H), generator=g).double().to(device) / 64
    Q[..., 0] = a.float()
    K[:, 1, :, 0] = -1.0
    lse = torch.log(1 + torch.exp(-a)).float().transpose(1, 2).contiguous()
    _, _, dV = att.backward(Q, K, V, torch.zeros_like(Q), lse, dO, lens_of(2, B, device), 1.0)
    s = torch.stack([torch.zeros_like(a), -a], -1) - lse.double().transpose(1, 2)[..., None]      # [B, Nq, H, 2]
    p = torch.exp(row(s, at)).transpose(1, 3)                                                     # [B, 2, H, 1]
    want = p * row(dO, at)
    within(dV[:, :2], want, 24 * U * want.abs(), "dV")


def scores_again(att, B, Nq, Nk, H, d, device="cuda", seed=6):
    """One key, one channel, lse the score to 24 bits: dV = e^(S - lse) dO.  In the exponent, of |S|: product 5, scale log2 e 2, lse log2 e 2, their difference 1; 2^x 2, product 5."""
    g, Q, K, V, rand = setting(B, Nq, Nk, H, d, device, seed)
    Q[..., d // 3] = 2 * rand(B, Nq, H)
    K[:, 0, :, d // 3] = 2 * rand(B, H)
    S = Q.double()[..., d // 3] * K.double()[:, :1, :, d // 3]
    lse = S.float().transpose(1, 2).contiguous()
    dO, at = one_row(rand(B, Nq, H, d))
    _, _, dV = att.backward(Q, K, V, torch.zeros_like(Q), lse, dO, lens_of(1, B, device), 1.0)
    s = row(S[..., None], at)
    want = torch.exp(s - s.float().double()) * row(dO, at)
    within(dV[:, :1], want, (16 * s.abs() + 16) * U * want.abs(), "scores again")


def norms(att, B, Nq, Nk, H, d, device="cuda", seed=7):
    """Normal values: errors of the whole tensors in the 2-norm.  Without the three least products a score is off by 2^-18 of its terms, about 4e-6, and so is what it weighs."""
    from attention_util import Attention
    g = torch.Generator().manual_seed(seed)
    randn = lambda n: torch.randn(B, n, H, d, generator=g).to(device)
    Q, K, V, dO = randn(Nq), randn(Nk), randn(Nk), randn(Nq)
    far = lambda x, y: float((x.double() - y).norm() / y.norm())
    ref = Attention(Q, K, V)
    O_ref, lse_ref, _, _ = ref.forward()
    O, _ = att.forward(Q, K, V, None, None)
    assert far(O, O_ref) <= 1e-6, ("O", far(O, O_ref))
    O_in, lse_in = O_ref.float().contiguous(), lse_ref.float().contiguous()
    for name, x, (want, _) in zip(("dQ", "dK", "dV"), att.backward(Q, K, V, O_in, lse_in, dO, None, None), ref.backward(O_in, lse_in, dO)):
        assert far(x, want) <= 1.5e-6, (name, far(x, want))


FORWARD = (scores, values, weights)
BACKWARD = (query_gradients, key_gradients, value_gradients, scores_again)
