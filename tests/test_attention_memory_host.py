"""Attention between whole sequences and the norms and rotation before it refuse outputs that share memory with themselves or with what else the call has (no GPU: nothing is
enqueued)."""
import ctypes

import pytest

import paper_2303_08810_amd as bra

MB = 1 << 20
OVERLAP = -10
# B, N, heads, kv_heads, d of bf16: everything in memory of its own, a packed buffer of 8 heads of 64 for tensors that share one
B, N, H, HK, D = 2, 40, 4, 2, 64
ROW = 8 * D


def at(address, batch=N * ROW, token=ROW, head=D):
    return ctypes.byref(bra.BraRows(address, batch, token, head))


def part(address, head):
    """From a head of a packed buffer on."""
    return at(address + 2 * D * head)


def attention(backward, lse=60 * MB, q_lens=61 * MB, k_lens=62 * MB, **over):
    s = ctypes.byref(bra.BraAttentionShape(B, N, N, H, HK, D, bra.BRA_BF16, 0, 0.0))
    names = ("Q", "K", "V", "O", "dO", "dQ", "dK", "dV")
    t = {n: over.get(n, at((i + 1) * MB)) for i, n in enumerate(names)}
    L = bra.lib()
    if not backward:
        return L.bra_attention_forward(s, t["Q"], t["K"], t["V"], q_lens, k_lens, t["O"], lse, 63 * MB, 1 << 40, None)
    return L.bra_attention_backward(s, t["Q"], t["K"], t["V"], t["O"], lse, t["dO"], q_lens, k_lens, t["dQ"], t["dK"], t["dV"], 63 * MB, 1 << 40, None)


def test_attention_outputs():
    for name in ("Q", "K", "V"):
        assert attention(False, **{name: at(4 * MB)}) == OVERLAP
        # heads 0..3 and, of another tensor of the buffer, from the last of them on
        assert attention(False, O=part(9 * MB, 0), **{name: part(9 * MB, 3)}) == OVERLAP
        assert attention(False, O=part(9 * MB, 2), **{name: part(9 * MB, 1)}) == OVERLAP
        # a last token of one where the other's first lies
        assert attention(False, O=at(9 * MB), **{name: at(9 * MB + 2 * ((2 * N - 1) * ROW))}) == OVERLAP
    assert attention(False, lse=4 * MB + 256) == OVERLAP and attention(False, lse=2 * MB) == OVERLAP
    assert attention(False, q_lens=4 * MB + 2 * D) == OVERLAP and attention(False, k_lens=60 * MB + 4 * (B * H * N - 1)) == OVERLAP
    for own in (dict(head=0), dict(head=D - 8), dict(token=0), dict(token=3 * D), dict(batch=0), dict(batch=(N - 1) * ROW), dict(batch=3 * D)):
        assert attention(False, O=at(4 * MB, **own)) == OVERLAP, own


def test_attention_gradients():
    for out in ("dQ", "dK", "dV"):
        for name in ("Q", "K", "V", "O", "dO"):
            assert attention(True, **{out: part(9 * MB, 1), name: part(9 * MB, 2)}) == OVERLAP, (out, name)
        for other in ("dQ", "dK", "dV"):
            if other != out:
                assert attention(True, **{out: part(9 * MB, 2), other: part(9 * MB, 3)}) == OVERLAP, (out, other)
        where = dict(dQ=6, dK=7, dV=8)[out] * MB
        assert attention(True, lse=where + 2 * D) == OVERLAP and attention(True, q_lens=where) == OVERLAP and attention(True, k_lens=where + 2 * ROW) == OVERLAP
        assert attention(True, **{out: at(9 * MB, head=8)}) == OVERLAP


def qk(backward, sums=(60 * MB, 61 * MB), vectors=None, **over):
    s = ctypes.byref(bra.BraQkNormShape(B, N, H, HK, D, D, N, 0, bra.BRA_BF16, 1e-6))
    p = {**dict(q_gamma=50 * MB, k_gamma=51 * MB, cos=52 * MB, sin=53 * MB, positions=54 * MB), **(vectors or {})}
    p = ctypes.byref(bra.BraQkNormParams(**p))
    t = {n: over.get(n, at((i + 1) * MB)) for i, n in enumerate(("Q", "K", "gQ", "gK", "dQ", "dK"))}
    L = bra.lib()
    if not backward:
        return L.bra_qk_norm_forward(s, t["Q"], t["K"], p, t["dQ"], t["dK"], None)
    return L.bra_qk_norm_backward(s, t["Q"], t["K"], p, t["gQ"], t["gK"], t["dQ"], t["dK"], *sums, 63 * MB, 1 << 40, None)


@pytest.mark.parametrize("backward", [False, True])
def test_norms_and_rotation(backward):
    ins = ("Q", "K") + (("gQ", "gK") if backward else ())
    for out in ("dQ", "dK"):
        for name in ins:
            # a head further on, of its own kind too; of the other kind also where it begins
            assert qk(backward, **{out: part(9 * MB, 2), name: part(9 * MB, 1)}) == OVERLAP, (out, name)
            if name[-1] != out[-1]:
                assert qk(backward, **{out: part(9 * MB, 2), name: part(9 * MB, 2)}) == OVERLAP, (out, name)
        where = dict(dQ=5, dK=6)[out] * MB
        for v in ("q_gamma", "k_gamma", "cos", "sin", "positions"):
            assert qk(backward, vectors={v: where}) == OVERLAP
        assert qk(backward, **{out: at(9 * MB, token=D)}) == OVERLAP
        if backward:
            assert qk(True, sums=(where, 61 * MB)) == OVERLAP and qk(True, sums=(60 * MB, where + 2 * D)) == OVERLAP
    assert qk(backward, dQ=part(9 * MB, 0), dK=part(9 * MB, 3)) == OVERLAP
    if backward:
        assert qk(True, sums=(60 * MB, 60 * MB + 4 * (D - 1))) == OVERLAP and qk(True, sums=(50 * MB, 61 * MB)) == OVERLAP


def test_places_too_far_apart():
    for stride in ("batch", "token", "head"):
        assert attention(False, K=at(2 * MB, **{stride: 1 << 56})) == -2 and attention(True, dK=at(7 * MB, **{stride: 1 << 62})) == -2
        assert qk(False, Q=at(MB, **{stride: 1 << 60})) == -2
