"""Host-side checks of attention between whole sequences and of the norms and rotation before it: invalid arguments become error codes or exceptions before
any GPU work, and the workspace queries."""
import ctypes
import math

import pytest
import torch

import paper_2303_08810_amd as bra

FAKE = 1 << 20                      # never dereferenced: a check fails first
NAN, INF = math.nan, math.inf


def rows(data=FAKE, batch=1 << 12, token=64, head=64):
    return ctypes.byref(bra.BraRows(data, batch, token, head))


def shape(B=2, Nq=40, Nk=50, heads=4, kv=2, d=64, dtype=bra.BRA_BF16, causal=0, scale=0.0):
    return bra.BraAttentionShape(B, Nq, Nk, heads, kv, d, dtype, causal, scale)


def attention(s, backward, ws=FAKE, ws_bytes=1 << 50, lse=FAKE, q_lens=None, k_lens=None, **over):
    names = ("Q", "K", "V", "O") + (("dO", "dQ", "dK", "dV") if backward else ())
    t = {n: over.get(n, rows()) for n in names}
    s = ctypes.byref(s) if s is not None else None
    L = bra.lib()
    if not backward:
        return L.bra_attention_forward(s, t["Q"], t["K"], t["V"], q_lens, k_lens, t["O"], lse, ws, ws_bytes, None)
    return L.bra_attention_backward(s, t["Q"], t["K"], t["V"], t["O"], lse, t["dO"], q_lens, k_lens, t["dQ"], t["dK"], t["dV"], ws, ws_bytes, None)


@pytest.mark.parametrize("backward", [False, True])
def test_attention_refusals(backward):
    assert attention(None, backward) == -1
    for bad in (shape(B=-1), shape(Nq=-1), shape(Nk=-1), shape(kv=0), shape(heads=3), shape(heads=0, kv=1), shape(heads=1, kv=2), shape(d=0), shape(scale=NAN), shape(scale=3e38), shape(scale=INF),
                shape(Nq=(1 << 28) + 1), shape(Nk=(1 << 28) + 1), shape(B=(1 << 28) + 1), shape(heads=65538), shape(B=1 << 28, heads=8), shape(Nq=1 << 28, heads=8),
                shape(B=1 << 14, Nk=1 << 28)):
        assert attention(bad, backward) == -2
    assert attention(shape(dtype=3), backward) == -4
    for d in (4, 65, 136, 256):
        assert attention(shape(d=d), backward) == -6
    for name in ("Q", "K", "V", "O") + (("dO", "dQ", "dK", "dV") if backward else ()):
        assert attention(shape(), backward, **{name: None}) == -1, name
        assert attention(shape(), backward, **{name: rows(data=None)}) == -1, name
        assert attention(shape(), backward, **{name: rows(data=FAKE + 8)}) == -9, name
        for stride in ("batch", "token", "head"):
            assert attention(shape(), backward, **{name: rows(**{stride: -64})}) == -2, name
            assert attention(shape(), backward, **{name: rows(**{stride: 68})}) == -9, name
            assert attention(shape(dtype=bra.BRA_F32), backward, **{name: rows(**{stride: 66})}) == -9, name
    assert attention(shape(), backward, q_lens=FAKE + 2) == -9 and attention(shape(), backward, k_lens=FAKE + 2) == -9 and attention(shape(), backward, lse=FAKE + 2) == -9
    if backward:
        assert attention(shape(), True, lse=None) == -1
    big = shape(Nq=100, Nk=100000)
    for ws, n in ((None, 1 << 50), (FAKE + 64, 1 << 50), (FAKE, 16)):
        assert attention(big, backward, ws=ws, ws_bytes=n) == -5
    # nothing to do: no tensor is looked at
    empty = {n: None for n in ("Q", "K", "V", "O", "dO", "dQ", "dK", "dV")}
    assert attention(shape(B=0), backward, ws=None, ws_bytes=0, lse=None, **empty) == 0
    assert attention(shape(Nq=0, Nk=0), backward, ws=None, ws_bytes=0, lse=None, **empty) == 0


def test_strides_of_one_entry_are_not_looked_at():
    odd = lambda: rows(batch=3, token=5, head=-7)
    # every stride is that of one entry; the workspace is what is refused
    one = dict(B=1, Nq=1, Nk=1, heads=1, kv=1)
    for name in ("Q", "K", "V", "O", "dO", "dQ", "dK", "dV"):
        assert attention(shape(B=1, Nq=1, Nk=100000, heads=1, kv=1), True, ws=None, **{n: odd() for n in ("Q", "O", "dO", "dQ")}) == -5
    assert attention(shape(**one), False, Q=odd(), K=odd(), V=odd(), O=rows(data=FAKE + 2)) == -9


def test_attention_workspaces():
    size = lambda backward=False, **k: bra.attention_workspace_bytes(shape(**k), backward)
    assert size(Nq=1, Nk=100) == 0                                           # small: none
    assert size(Nq=1, Nk=100000) > 0                                         # keys shared out
    assert size(True, Nq=49, Nk=49, heads=2) == 0                            # a short sequence's gradients
    assert size(True, Nq=4096, Nk=4096) >= 2 * 4 * 2 * 4 * 4096              # a sum and a logarithm for each query
    assert size(Nq=1000, Nk=1000, dtype=bra.BRA_F32) >= 2 * 3 * 2 * 2 * 2 * 1000 * 64      # keys and values in three bf16 terms
    for n in (size(Nq=1, Nk=100000), size(True, Nq=333, Nk=777), size(True, Nq=333, Nk=777, dtype=bra.BRA_F32)):
        assert n % 256 == 0
    assert bra.lib().bra_attention_workspace_bytes(None, None) == -1 and bra.lib().bra_attention_backward_workspace_bytes(None, None) == -1
    # no size within the limits overflows
    assert size(True, B=1 << 10, Nq=1 << 28, Nk=1 << 28, heads=4, kv=4, d=128, dtype=bra.BRA_F32) >= 12 * (1 << 40) * 128 * 2


def qk_shape(B=2, N=9, heads=4, kv=2, d=64, turned=64, table=9, pairs=0, dtype=bra.BRA_BF16, eps=1e-6):
    return bra.BraQkNormShape(B, N, heads, kv, d, turned, table, pairs, dtype, eps)


def qk(s, backward, ws=FAKE, ws_bytes=1 << 40, params=True, gammas=FAKE, vectors=None, **over):
    L = bra.lib()
    p = dict(q_gamma=FAKE, k_gamma=FAKE, cos=FAKE, sin=FAKE, positions=None)
    p.update(vectors or {})
    p = ctypes.byref(bra.BraQkNormParams(**p)) if params else None
    t = {n: over.get(n, rows()) for n in ("Q", "K", "gQ", "gK", "dQ", "dK", "Qout", "Kout")}
    s = ctypes.byref(s) if s is not None else None
    if not backward:
        return L.bra_qk_norm_forward(s, t["Q"], t["K"], p, t["Qout"], t["Kout"], None)
    return L.bra_qk_norm_backward(s, t["Q"], t["K"], p, t["gQ"], t["gK"], t["dQ"], t["dK"], gammas, gammas, ws, ws_bytes, None)


@pytest.mark.parametrize("backward", [False, True])
def test_qk_norm_refusals(backward):
    assert qk(None, backward) == -1 and qk(qk_shape(), backward, params=False) == -1
    for bad in (qk_shape(B=-1), qk_shape(N=-1), qk_shape(heads=0), qk_shape(kv=-1), qk_shape(d=0), qk_shape(turned=-2), qk_shape(turned=66), qk_shape(turned=7), qk_shape(eps=-1.0),
                qk_shape(eps=NAN), qk_shape(table=0), qk_shape(table=8), qk_shape(B=1 << 16, N=1 << 16), qk_shape(B=1 << 10, N=1 << 18, heads=7, table=1 << 18)):
        assert qk(bad, backward) == -2
    assert qk(qk_shape(table=0), backward, vectors=dict(positions=FAKE)) == -2
    assert qk(qk_shape(dtype=2), backward) == -4 and qk(qk_shape(pairs=2), backward) == -4
    for d in (12, 136):
        assert qk(qk_shape(d=d, turned=0), backward) == -6
    for name in ("cos", "sin", "k_gamma", "q_gamma"):
        assert qk(qk_shape(), backward, vectors={name: None}) == -1, name
    for name in ("cos", "sin", "k_gamma", "q_gamma", "positions"):
        assert qk(qk_shape(), backward, vectors={name: FAKE + 2}) == -9, name
    for name in ("Q", "K") + (("gQ", "gK", "dQ", "dK") if backward else ("Qout", "Kout")):
        assert qk(qk_shape(), backward, **{name: None}) == -1, name
        assert qk(qk_shape(), backward, **{name: rows(data=FAKE + 4)}) == -9, name
        assert qk(qk_shape(), backward, **{name: rows(token=60)}) == -9, name
        assert qk(qk_shape(), backward, **{name: rows(head=-64)}) == -2, name
    if backward:
        for ws, n in ((None, 1 << 40), (FAKE + 64, 1 << 40), (FAKE, 16)):
            assert qk(qk_shape(), True, ws=ws, ws_bytes=n) == -5
        assert qk(qk_shape(), True, gammas=FAKE + 2) == -9
    else:
        assert qk(qk_shape(B=0), False, Q=None, K=None, Qout=None, Kout=None) == 0


def test_binding_refuses_what_is_not_on_a_gpu():
    Q = torch.zeros(2, 5, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        bra.bra_attention_forward(Q, Q, Q)
    with pytest.raises(ValueError):
        bra.bra_attention_backward(Q, Q, Q, Q, torch.zeros(2, 4, 5), Q)
    with pytest.raises(ValueError):
        bra.bra_qk_norm_forward(Q, Q)
    with pytest.raises(ValueError):
        bra.bra_qk_norm_backward(Q, Q, Q, Q)
    with pytest.raises(ValueError):
        bra.bra_attention_forward(Q[0], Q, Q)
    with pytest.raises(ValueError):
        bra.bra_attention_forward(Q, Q[:1], Q[:1])
    with pytest.raises(TypeError):
        bra.bra_attention_forward(Q.half(), Q.half(), Q.half())
    with pytest.raises(TypeError):
        bra.bra_attention_forward(Q, Q, "x")
    with pytest.raises(bra.BraError):
        bra.bra_attention_forward(Q[..., :60], Q[..., :60], Q[..., :60])
    with pytest.raises(KeyError):
        bra.bra_qk_norm_forward(Q, Q, pairs="thirds")


def test_rotary_table():
    cos, sin = bra.rotary_table(7, channels=10, base=100.0)
    assert cos.shape == sin.shape == (7, 5) and cos.dtype == torch.float32
    for n in range(7):
        for p in range(5):
            angle = n * 100.0 ** (-2 * p / 10)
            assert abs(float(cos[n, p]) - math.cos(angle)) <= 2.0 ** -24 and abs(float(sin[n, p]) - math.sin(angle)) <= 2.0 ** -24
    cos, sin = bra.rotary_table(3, 5, channels=8)
    for y in range(3):
        for x in range(5):
            for p in range(4):
                angle = (y if p < 2 else x) * 10000.0 ** (-2 * (p % 2) / 4)
                assert abs(float(cos[5 * y + x, p]) - math.cos(angle)) <= 2.0 ** -24 and abs(float(sin[5 * y + x, p]) - math.sin(angle)) <= 2.0 ** -24
    # a far position: formed in 64 bits
    far = bra.rotary_table(1 << 20, channels=2)
    assert abs(float(far[0][-1, 0]) - math.cos((1 << 20) - 1)) <= 2.0 ** -24
    for bad in (dict(H=4, channels=5), dict(H=4, W=4, channels=6), dict(H=4, channels=-2)):
        with pytest.raises(ValueError):
            bra.rotary_table(**bad)
