"""Attention forward with heads of 72 to 96 channels, whose 12 pieces of 8 do not divide a workgroup: single tokens over short and long caches, many rows, keys shared out to
several workgroups and joined by 2 to 16 groups of threads."""
import pytest
import torch

import paper_2303_08810_amd as bra
from attention_util import Attention, check

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def join_bytes(Q, K, splits):
    B, Nq, H, d = Q.shape
    width, rows, up = (d + 31) // 32 * 32, Nq * H * B, lambda n: (n + 255) // 256 * 256
    return up(4 * splits * rows * width) + up(8 * splits * rows)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("d", [72, 80, 96])
@pytest.mark.parametrize("B,Nq,Nk,H,Hk,least", [(1, 1, 150, 12, 12, 1), (2, 1, 600, 4, 2, 2), (3, 1, 1300, 3, 1, 4), (1, 3, 2100, 9, 1, 8), (2, 1, 6000, 2, 2, 16), (1, 32, 5000, 2, 2, 16),
                                                (1, 33, 1600, 2, 1, 2), (2, 50, 4000, 4, 2, 4), (1, 200, 7000, 2, 2, 8)])
def test_joined_sums(B, Nq, Nk, H, Hk, least, d, dtype):
    g = torch.Generator().manual_seed(d + Nk)
    randn = lambda *s: torch.randn(*s, generator=g).to(dtype).cuda()
    Q, K, V = randn(B, Nq, H, d), randn(B, Nk, Hk, d), randn(B, Nk, Hk, d)
    lens = torch.tensor([Nk - 1 - b * (Nk // 3) for b in range(B)], dtype=torch.int32, device="cuda")
    few = Nq * H // Hk <= 32
    if least > 1 and (few or dtype == BF16):       # otherwise the terms' planes are in it too
        size = bra.attention_workspace_bytes(bra.make_attention_shape(B, Nq, Nk, H, Hk, d, dtype))
        assert any(size == join_bytes(Q, K, n) for n in range(least, 65)), (size, least)
    print("join", B, Nq, Nk, H, Hk, d, dtype, flush=True)
    for rule in (dict(), dict(k_lens=lens, causal=True)):
        O_ref, lse_ref, O_off, lse_off = Attention(Q, K, V, **rule).forward()
        O, lse = bra.bra_attention_forward(Q, K, V, want_lse=True, **rule)
        check(O, O_ref, O_off, "O")
        check(lse, lse_ref, lse_off, "lse")
        assert torch.equal(O, bra.bra_attention_forward(Q, K, V, **rule))
