"""Attention between whole sequences and its gradients against 64-bit references, element by element."""
import math

import pytest
import torch

import paper_2303_08810_amd as bra
from attention_util import Attention, check

pytestmark = pytest.mark.gpu

# B, Nq, Nk, heads, kv_heads, d, causal, q_lens, k_lens, layout
CASES = [
    (1, 1, 1, 1, 1, 8, False, None, None, "apart"),
    (1, 1, 197, 12, 12, 64, False, None, None, "cache"),
    (2, 1, 3000, 8, 2, 128, False, None, [2999, 65], "cache"),
    (3, 1, 700, 6, 1, 40, True, None, [700, 0, 1], "cache"),
    (2, 5, 260, 7, 1, 72, True, None, None, "apart"),
    (2, 49, 49, 4, 4, 32, False, None, None, "packed"),
    (1, 64, 64, 2, 2, 64, True, None, None, "packed"),
    (2, 65, 63, 2, 1, 64, True, None, None, "apart"),              # the first two queries see nothing
    (2, 127, 129, 3, 3, 96, True, None, None, "apart"),
    (3, 130, 130, 6, 2, 24, True, [130, 1, 0], [130, 1, 0], "packed"),
    (3, 70, 200, 4, 2, 128, False, [70, 64, 3], [1, 200, 129], "cache"),
    (2, 200, 90, 5, 5, 104, True, [200, 17], [90, 33], "apart"),
    (1, 333, 333, 6, 3, 64, False, None, None, "packed"),
    (1, 40, 2500, 4, 4, 64, True, None, None, "cache"),             # keys shared out, many rows
    (2, 40, 1500, 3, 3, 128, False, [40, 39], [1500, 700], "cache"),
    (2, 100, 128, 3, 3, 128, True, [100, 31], [128, 77], "apart"),     # gradients in one launch, sides of 128, 256, (float32) 128, 64 and 32
    (2, 50, 256, 4, 1, 24, True, [50, 9], [256, 1], "cache"),
    (2, 200, 250, 2, 2, 64, False, None, [250, 0], "apart"),
    (3, 30, 90, 3, 1, 16, False, None, [90, 0, 33], "apart"),
    (2, 30, 60, 2, 1, 64, True, [30, 0], [60, 7], "apart"),
    (2, 16, 32, 4, 2, 120, True, None, [32, 20], "apart"),
    (1, 3, 0, 2, 1, 32, False, None, None, "apart"),
    (2, 0, 5, 2, 1, 32, False, None, None, "apart"),
]


def tensors(c, dtype, seed=0, device="cuda"):
    B, Nq, Nk, H, Hk, d, causal, ql, kl, layout = c
    g = torch.Generator(device="cpu").manual_seed(seed)
    randn = lambda *s: torch.randn(*s, generator=g).to(dtype).to(device)
    if layout == "packed":
        X = randn(B, Nq, H + 2 * Hk, d)
        Q, K, V = X[:, :, :H], X[:, :, H:H + Hk], X[:, :, H + Hk:]
    else:
        Q = randn(B, Nq, H, d)
        K, V = (randn(B, Hk, Nk, d).transpose(1, 2) if layout == "cache" else randn(B, Nk, Hk, d) for _ in range(2))
    dO = randn(B, Nq, H, d)
    lens = lambda v: None if v is None else torch.tensor(v, dtype=torch.int32, device=device)
    return Q, K, V, dO, dict(causal=causal, q_lens=lens(ql), k_lens=lens(kl))


def spoil(c, Q, K, V, dO):
    """NaN and infinities where a sequence has nothing."""
    ql, kl = c[7], c[8]
    for b in range(c[0]):
        if ql is not None:
            Q[b, ql[b]:] = math.nan
            dO[b, ql[b]:] = math.inf
        if kl is not None:
            K[b, kl[b]:] = math.inf
            V[b, kl[b]:] = math.nan


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("c", CASES, ids=lambda c: "x".join(map(str, c[:6])) + ("c" if c[6] else ""))
def test_forward_and_gradients(c, dtype):
    Q, K, V, dO, rule = tensors(c, dtype)
    spoil(c, Q, K, V, dO)
    ref = Attention(Q, K, V, **rule)
    O_ref, lse_ref, O_off, lse_off = ref.forward()
    print("forward", c, flush=True)
    O, lse = bra.bra_attention_forward(Q, K, V, want_lse=True, **rule)
    check(O, O_ref, O_off, "O")
    check(lse, lse_ref, lse_off, "lse")
    again = bra.bra_attention_forward(Q, K, V, **rule)
    assert torch.equal(O, again)
    print("backward", c, flush=True)
    O_in, lse_in = O_ref.to(dtype), lse_ref.float()
    if c[7] is not None:
        for b in range(c[0]):
            O_in[b, c[7][b]:] = math.nan
            lse_in[b, :, c[7][b]:] = math.nan
    grads = bra.bra_attention_backward(Q, K, V, O_in, lse_in, dO, **rule)
    for name, got, (want, off) in zip(("dQ", "dK", "dV"), grads, ref.backward(O_in, lse_in, dO)):
        check(got, want, off, name)
    for x, y in zip(grads, bra.bra_attention_backward(Q, K, V, O_in, lse_in, dO, **rule)):
        assert torch.equal(x, y)
