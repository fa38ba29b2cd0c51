"""Gradients of rows that see one key: its weight is one, O is its value, and dS = dO V - dO O is zero, so that dQ, and dK of a sequence of one key, are zero too."""
import math

import pytest
import torch

import paper_2303_08810_amd as bra
from attention_util import Attention, check

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
TYPES = pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])


def make(B, Nq, Nk, H, Hk, d, dtype, seed=0):
    """Queries and keys within 0.2: a score's terms sum up to d^0.5 0.04 = 0.453 at most, and two ways to form it, each off by up to (d + 8) 2^-24 of that, differ by less than
    1.1e-5 as a power of two, 2^-16 = 1.5e-5 of which counts as the whole weight."""
    g = torch.Generator().manual_seed(seed)
    small = lambda *s: (0.4 * torch.rand(*s, generator=g) - 0.2).to(dtype).cuda()
    wide = lambda *s: torch.randn(*s, generator=g).to(dtype).cuda()
    return small(B, Nq, H, d), small(B, Nk, Hk, d), wide(B, Nk, Hk, d), wide(B, Nq, H, d)


def gradients(Q, K, V, dO, **rule):
    O, lse = bra.bra_attention_forward(Q, K, V, want_lse=True, **rule)
    ref = Attention(Q, K, V, **rule)
    got = bra.bra_attention_backward(Q, K, V, O, lse, dO, **rule)
    for name, x, (want, off) in zip(("dQ", "dK", "dV"), got, ref.backward(O, lse, dO)):
        check(x, want, off, name)
    return got


@TYPES
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,Nq,Nk,H,Hk,d", [(1, 1, 1, 1, 1, 8), (3, 1, 1, 4, 2, 128), (2, 40, 1, 4, 2, 40), (2, 9, 30, 3, 1, 96), (2, 49, 49, 4, 4, 32), (2, 100, 128, 2, 2, 64), (2, 300, 1, 6, 2, 72),
                                            (2, 700, 1, 4, 1, 128), (2, 500, 300, 2, 2, 64), (1, 1200, 40, 5, 1, 24), (40, 300, 1, 8, 4, 104)])
def test_sequences_of_one_key(B, Nq, Nk, H, Hk, d, causal, dtype):
    Q, K, V, dO = make(B, Nq, Nk, H, Hk, d, dtype)
    one = torch.ones(B, dtype=torch.int32, device="cuda") if Nk > 1 else None
    dQ, dK, dV = gradients(Q, K, V, dO, causal=causal, k_lens=one)
    assert not dQ.any() and not dK.any()
    assert bool(dV[:, 0].any())


@TYPES
@pytest.mark.parametrize("Nq", [60, 400])
def test_far_scores(Nq, dtype):
    """Whole numbers, whose scores are exact: lse keeps 2^-24 of itself, which the weight is asked in proportion to."""
    Q, K, V, dO = make(2, Nq, 1, 4, 2, 64, dtype)
    g = torch.Generator().manual_seed(9)
    Q, K = (torch.randint(-9, 10, t.shape, generator=g).to(dtype).cuda() for t in (Q, K))
    dQ, dK, _ = gradients(Q, K, V, dO)
    assert not dQ.any() and not dK.any()


@TYPES
@pytest.mark.parametrize("N,G", [(50, 1), (300, 3), (700, 2)])
def test_first_rows_of_causal_sequences(N, G, dtype):
    """One query more than keys: the first sees nothing, the second one key."""
    Q, K, V, dO = make(2, N + 1, N, 2 * G, 2, 64, dtype)
    dQ, dK, _ = gradients(Q, K, V, dO, causal=True)
    assert not dQ[:, :2].any() and bool(dQ[:, 2].any()) and bool(dK[:, 0].any())


@TYPES
@pytest.mark.parametrize("Nq", [40, 500])
def test_one_key_of_a_longer_sequence(Nq, dtype):
    """lse and O of 30 keys, one of which a call has: its weight is less than one, and its gradients are those of the formula; with the other 29's they add up to the whole."""
    Q, K, V, dO = make(2, Nq, 30, 4, 2, 64, dtype)
    O, lse = bra.bra_attention_forward(Q, K, V, want_lse=True)
    for part in (slice(0, 1), slice(1, 30)):
        k, v = K[:, part], V[:, part]
        got = bra.bra_attention_backward(Q, k, v, O, lse, dO)
        assert bool(got[0].any()) and bool(got[1].any())
        for name, x, (want, off) in zip(("dQ", "dK", "dV"), got, Attention(Q, k, v).backward(O, lse, dO)):
            check(x, want, off, name)


@TYPES
@pytest.mark.parametrize("Nq", [40, 500])
def test_what_is_not_a_number_is_kept(Nq, dtype):
    Q, K, V, dO = make(2, Nq, 1, 4, 2, 64, dtype)
    V[0, 0, 1, 5] = math.nan
    O, lse = bra.bra_attention_forward(Q, K, V, want_lse=True)
    dQ, dK, _ = bra.bra_attention_backward(Q, K, V, O, lse, dO)
    assert bool(dQ[0, :, 2:].isnan().all()) and bool(dK[0, 0, 1].isnan().all())
    assert not dQ[0, :, :2].any() and not dQ[1].any() and not dK[0, 0, 0].any() and not dK[1].any()
