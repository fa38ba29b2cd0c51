"""Gradients in bf16 where a workgroup walks over many more subtiles of 32 rows than its five places in LDS hold: one share for all rows, and the most shares that there are."""
import pytest
import torch

import paper_2303_08810_amd as bra
from attention_util import Attention, check

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
PLACES = 5


def walks(B, Nq, Nk, H, Hk, d):
    """Subtiles that a workgroup of the key side walks over, at the least of the shares that the workspace's size can mean: [heads][shares][rows or 2 Nk][width] floats for either side that
    has shares, and two numbers for each row."""
    up = lambda n: (n + 255) // 256 * 256
    heads, rows, width = B * Hk, Nq * H // Hk, (d + 31) // 32 * 32
    size = bra.attention_workspace_bytes(bra.make_attention_shape(B, Nq, Nk, H, Hk, d, BF16), True) - 2 * up(4 * rows * heads)
    assert size >= 0
    part = lambda n, each: up(4 * n * each * width * heads) if n > 1 else 0
    shares = [k for q in range(1, 65) for k in range(1, 65) if part(q, rows) + part(k, 2 * Nk) == size]
    assert shares
    return ((rows + 31) // 32 + max(shares) - 1) // max(shares)


# B, Nq, Nk, heads, kv_heads, d, causal, lengths
CASES = [
    (66, 700, 130, 4, 4, 64, False, False),         # a share to a key head and tile
    (66, 700, 130, 4, 4, 64, True, True),
    (70, 500, 200, 4, 2, 128, True, False),
    (90, 450, 140, 3, 3, 72, False, True),
    (90, 450, 60, 6, 3, 32, False, True),
    (60, 240, 130, 15, 5, 128, False, True),        # three query heads to a key head: rows without a step
    (60, 240, 130, 15, 5, 104, True, False),
    (1, 6100, 300, 1, 1, 64, False, False),         # the most shares
    (1, 3100, 300, 2, 1, 128, False, False),
    (1, 2117, 300, 3, 1, 64, False, False),
    (2, 1300, 130, 5, 1, 128, False, True),
    (1, 4200, 4100, 2, 1, 64, True, False),
    (1, 4200, 4100, 2, 1, 128, True, False),
    (1, 2500, 2600, 7, 1, 72, True, False),
    (2, 1100, 900, 8, 1, 104, True, True),
    (2, 3000, 64, 2, 1, 64, True, True),            # two wavefronts
]


@pytest.mark.parametrize("c", CASES, ids=lambda c: "x".join(map(str, c[:6])) + ("c" if c[6] else "") + ("r" if c[7] else ""))
def test_long_walks(c):
    B, Nq, Nk, H, Hk, d, causal, ragged = c
    assert walks(*c[:6]) > 2 * PLACES
    g = torch.Generator().manual_seed(Nq + d)
    randn = lambda *s: torch.randn(*s, generator=g).to(BF16).cuda()
    Q, K, V, dO = randn(B, Nq, H, d), randn(B, Nk, Hk, d), randn(B, Nk, Hk, d), randn(B, Nq, H, d)
    lens = lambda n, least: torch.tensor([n - (b * 37) % (n - least + 1) for b in range(B)], dtype=torch.int32, device="cuda") if ragged else None
    q_lens, k_lens = lens(Nq, Nq - Nq // 4), lens(Nk, 1)
    print("walk", c, flush=True)
    O, lse = bra.bra_attention_forward(Q, K, V, causal=causal, q_lens=q_lens, k_lens=k_lens, want_lse=True)
    grads = bra.bra_attention_backward(Q, K, V, O, lse, dO, causal=causal, q_lens=q_lens, k_lens=k_lens)
    for x, y in zip(grads, bra.bra_attention_backward(Q, K, V, O, lse, dO, causal=causal, q_lens=q_lens, k_lens=k_lens)):
        assert torch.equal(x, y)
    for b in sorted({0, B // 2, B - 1}):
        one = slice(b, b + 1)
        ref = Attention(Q[one], K[one], V[one], causal=causal, q_lens=None if q_lens is None else q_lens[one], k_lens=None if k_lens is None else k_lens[one])
        for name, got, (want, off) in zip(("dQ", "dK", "dV"), grads, ref.backward(O[one], lse[one], dO[one])):
            check(got[one], want, off, name)
