"""Attention between whole sequences and what goes before it in 64 bits, with bounds on how far float32 arithmetic and the roundings that the kernels
document may be off, element by element.  A rounding is off by half a step at most: 2^-8 of the value in bf16, 2^-24 in float32."""
from __future__ import annotations

import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U = 2.0 ** -24
TINY = 1e-30


def rows(x, heads):
    """[B, N, h, d] -> [B, heads, N, d] in 64 bits, heads that share a key head repeated."""
    x = x.double().transpose(1, 2)
    return x.repeat_interleave(heads // x.shape[1], 1)


def visible(B, Nq, Nk, causal, q_lens, k_lens, device):
    i, j = torch.arange(Nq, device=device)[:, None], torch.arange(Nk, device=device)
    out = torch.zeros(B, 1, Nq, Nk, dtype=torch.bool, device=device)
    for b in range(B):
        nq = Nq if q_lens is None else min(max(int(q_lens[b]), 0), Nq)
        nk = Nk if k_lens is None else min(max(int(k_lens[b]), 0), Nk)
        out[b, 0] = (i < nq) & (j < nk) & ((j <= i + nk - nq) if causal else True)
    return out


class Attention:
    """What goes in is cleaned of what the masks hide: the kernels do not read it."""

    def __init__(self, Q, K, V, causal=False, q_lens=None, k_lens=None, scale=None):
        B, Nq, H, d = Q.shape
        Nk = K.shape[1]
        self.scale, self.d, self.H, self.G, self.dtype = scale or d ** -0.5, d, H, H // K.shape[2], Q.dtype
        self.see = visible(B, Nq, Nk, causal, q_lens, k_lens, Q.device)
        some_q, some_k = self.see.any(-1, keepdim=True), self.see.any(-2).unsqueeze(-1)
        clean = lambda x, some: torch.where(some, x, 0.0)
        self.some_q = some_q
        self.q, self.k, self.v = clean(rows(Q, H), some_q), clean(rows(K, H), some_k), clean(rows(V, H), some_k)
        self.s = torch.where(self.see, self.scale * (self.q @ self.k.transpose(-1, -2)), -math.inf)
        size = self.scale * (self.q.abs() @ self.k.abs().transpose(-1, -2))
        # a product's sum of d terms, the factor in powers of two, the difference from the maximum: off by this much in an exponent
        self.delta = torch.where(self.see, (d + 8) * U * size, 0.0)
        self.n = max(Nk, 1)

    def forward(self):
        top = self.s.amax(-1, keepdim=True) if self.s.shape[-1] else torch.full_like(self.s.sum(-1, keepdim=True), -math.inf)
        top = torch.where(top == -math.inf, 0.0, top)
        p = torch.exp(self.s - top)
        total = p.sum(-1, keepdim=True)
        self.p = p / torch.where(total == 0, 1.0, total)
        O = self.p @ self.v
        lse = (top + torch.log(total)).squeeze(-1)
        worst = self.delta.amax(-1, keepdim=True) if self.s.shape[-1] else 0.0
        spread = (HALF[torch.bfloat16] if self.dtype == torch.bfloat16 else 0.0) + 2 * worst + (2 * self.n + 32) * U
        O_off = 1.01 * spread * (self.p @ self.v.abs()) + 1.01 * HALF[self.dtype] * O.abs() + TINY
        # the sum's own terms, the logarithm and the steps to and from powers of two
        lse_off = (worst.squeeze(-1) if torch.is_tensor(worst) else worst) + (self.n + 32) * U + 4 * U * lse.abs() + 8 * U * top.squeeze(-1).abs()
        return O.transpose(1, 2), lse, O_off.transpose(1, 2), torch.where(lse == -math.inf, 0.0, lse_off)

    def backward(self, O, lse, dO):
        clean = lambda x: torch.where(self.some_q, x, 0.0)
        o, g, lse = clean(rows(O, self.H)), clean(rows(dO, self.H)), torch.where(self.some_q, lse.double().unsqueeze(-1), 0.0)
        p = torch.where(self.see, torch.exp(self.s - lse), 0.0)
        dp, delta = g @ self.v.transpose(-1, -2), (g * o).sum(-1, keepdim=True)
        ds = p * (dp - delta)
        half = HALF[torch.bfloat16] if self.dtype == torch.bfloat16 else 0.0
        p_rel = self.delta + 4 * U * (torch.where(self.see, self.s, 0.0).abs() + lse.abs()) + 32 * U
        ds_off = ds.abs() * (p_rel + half + 4 * U) + p * (1 + p_rel) * (self.d + 8) * U * (g.abs() @ self.v.abs().transpose(-1, -2) + (g * o).abs().sum(-1, keepdim=True))
        t = lambda x: x.transpose(-1, -2)
        rows_n, keys_n = self.q.shape[2] * self.G + 8, self.n + 8
        dq, dk, dv = self.scale * ds @ self.k, self.scale * t(ds) @ self.q, t(p) @ g
        dq_off = self.scale * (ds_off + keys_n * U * ds.abs()) @ self.k.abs()
        dk_off = self.scale * t(ds_off + rows_n * U * ds.abs()) @ self.q.abs()
        dv_off = t(p * (p_rel + half + rows_n * U)) @ g.abs()
        shared = lambda x: x.view(x.shape[0], self.H // self.G, self.G, *x.shape[2:]).sum(2)
        out = []
        for x, off in ((dq, dq_off), (shared(dk), shared(dk_off)), (shared(dv), shared(dv_off))):
            out.append((x.transpose(1, 2), (1.02 * off + 1.01 * HALF[self.dtype] * x.abs() + TINY).transpose(1, 2)))
        return out


def heads_rule(x, gamma, cos, sin, positions, pairs, eps):
    """Norm and rotation in 64 bits, differentiable."""
    x = x.double()
    if gamma is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gamma.double()
    if cos is None:
        return x
    r = 2 * cos.shape[1]
    N = x.shape[1]
    at = torch.arange(N, device=x.device).expand(x.shape[0], N) if positions is None else positions.long().clamp(0, cos.shape[0] - 1)
    co, si = cos.double()[at].unsqueeze(2), sin.double()[at].unsqueeze(2)
    if pairs == "halves":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * co - b * si, b * co + a * si], -1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * co - b * si, b * co + a * si], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def check(got, want, off, what):
    assert got.shape == want.shape, (what, got.shape, want.shape)
    got = got.double()
    same = (got == want) | ((got - want).abs() <= off)
    if not bool(same.all()):
        worst = torch.where(same, 0.0, torch.nan_to_num((got - want).abs() / off, nan=math.inf, posinf=math.inf)).flatten()
        i = int(worst.argmax())
        raise AssertionError(f"{what}: {int((~same).sum())} of {same.numel()} off, the worst {float(worst[i]):.3g} times its bound, {float(got.flatten()[i])} for {float(want.flatten()[i])}")
