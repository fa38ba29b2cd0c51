"""Norms and rotation of queries and keys against 64-bit references, element by element."""
import pytest
import torch

import paper_2303_08810_amd as bra
from attention_util import HALF, U, check, heads_rule

pytestmark = pytest.mark.gpu

# B, N, heads, kv_heads (0: queries alone), d, rotated channels, norm, pairs, positions, packed
CASES = [
    (1, 1, 12, 12, 64, 64, True, "halves", True, False),
    (2, 3, 1, 1, 8, 8, True, "neighbours", False, False),
    (3, 37, 6, 2, 40, 40, True, "halves", False, True),
    (2, 50, 5, 1, 24, 12, True, "neighbours", True, True),
    (2, 9, 3, 3, 16, 6, True, "halves", False, False),
    (2, 9, 3, 3, 56, 14, False, "neighbours", True, False),
    (4, 600, 8, 2, 128, 64, True, "neighbours", False, True),
    (4, 600, 7, 1, 128, 128, True, "halves", True, True),
    (3, 700, 9, 0, 72, 36, True, "halves", False, False),
    (2, 33, 4, 4, 96, 0, True, "halves", False, True),
    (2, 1100, 4, 4, 64, 64, False, "halves", True, True),
    (0, 4, 2, 1, 32, 32, True, "halves", False, False),
]


def tensors(c, dtype):
    B, N, H, Hk, d, r, norm, pairs, positions, packed = c
    g = torch.Generator().manual_seed(5)
    randn = lambda *s: torch.randn(*s, generator=g).to(dtype).cuda()
    if packed:
        X = randn(B, N, H + 2 * max(Hk, 1), d)
        Q, K = X[:, :, :H], X[:, :, H:H + Hk] if Hk else None
    else:
        Q, K = randn(B, N, H, d), randn(B, N, Hk, d) if Hk else None
    dQ, dK = randn(B, N, H, d), randn(B, N, Hk, d) if Hk else None
    gamma = lambda: (1 + 0.3 * torch.randn(d, generator=g)).cuda()
    gq, gk = (gamma() if norm else None), (gamma() if norm and Hk else None)
    rule = dict(pairs=pairs, eps=1e-5, cos=None, sin=None, positions=None)
    if r:
        T = 5000 if positions else N + 3
        rule["cos"], rule["sin"] = bra.rotary_table(T, channels=r, device="cuda")
        if positions:
            rule["positions"] = torch.randint(-3, T + 3, (B, N), generator=g).to(torch.int32).cuda()      # beyond the table: its ends
    return Q, K, dQ, dK, gq, gk, rule


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("c", CASES, ids=lambda c: "x".join(map(str, c[:6])) + c[7][0])
def test_forward_and_gradients(c, dtype):
    Q, K, dQ, dK, gq, gk, rule = tensors(c, dtype)
    half, d = HALF[dtype], c[4]
    print(c, flush=True)
    outs = bra.bra_qk_norm_forward(Q, K, gq, gk, **rule)
    assert K is not None or outs[1] is None
    grads = bra.bra_qk_norm_backward(Q, K, dQ, dK, gq, gk, **rule)
    assert len(grads) == (4 if gq is not None else 2)
    for i, (x, dy, gamma) in enumerate(((Q, dQ, gq), (K, dK, gk))):
        if x is None:
            continue
        live = x.double().requires_grad_()
        g64 = None if gamma is None else gamma.double().requires_grad_()
        y = heads_rule(live, g64, rule["cos"], rule["sin"], rule["positions"], rule["pairs"], rule["eps"])
        # a rotated pair's terms are of its length at most; the mean's sum of d squares, the root and the products
        length = heads_rule(x, gamma, None, None, None, None, rule["eps"]).detach().abs()
        pair = length.amax(-1, keepdim=True) * 1.5
        steps = (d + 16) * U
        check(outs[i], y.detach(), steps * pair + half * 1.01 * y.detach().abs() + 1e-30, "out")
        want = torch.autograd.grad((y * dy.double()).sum(), [live] + ([g64] if gamma is not None else []))
        # dx = inv (g gamma - u mean(g gamma u)): terms of these sizes
        if gamma is None:
            size = dy.double().abs().amax(-1, keepdim=True) * 1.5
        else:
            inv = 1 / torch.sqrt((x.double() ** 2).mean(-1, keepdim=True) + rule["eps"])
            u, gg = (x.double() * inv).abs(), dy.double().abs().amax(-1, keepdim=True) * 1.5 * gamma.double().abs().max()
            size = inv * (gg + u * (gg * u).mean(-1, keepdim=True))
        check(grads[i], want[0], 3 * steps * size + half * 1.01 * want[0].abs() + 1e-30, "dx")
        if gamma is not None:
            u = (x.double() / torch.sqrt((x.double() ** 2).mean(-1, keepdim=True) + rule["eps"])).abs()
            terms = (u * dy.double().abs().amax(-1, keepdim=True) * 1.5).sum((0, 1, 2))
            n = x.shape[0] * x.shape[1] * x.shape[2]
            check(grads[2 + i], want[1], (min(n, 512) + 3 * d) * U * terms + 1e-30, "dgamma")
    for a, b in zip(grads, bra.bra_qk_norm_backward(Q, K, dQ, dK, gq, gk, **rule)):
        assert (a is None and b is None) or torch.equal(a, b)
    # in place
    Q2, K2 = Q.clone(), None if K is None else K.clone()
    bra.bra_qk_norm_forward(Q2, K2, gq, gk, out=(Q2, K2), **rule)
    assert torch.equal(Q2, outs[0]) and (K is None or torch.equal(K2, outs[1]))
