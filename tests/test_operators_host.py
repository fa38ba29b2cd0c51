"""Host-side checks of the gated feed-forward block, the norms around a residual sum and the AdamW step: invalid arguments become
error codes or exceptions before any GPU work (none of these calls reaches a launch), and the workspace queries."""
import ctypes

import pytest
import torch

import paper_2303_08810_amd as bra

FAKE = 1 << 20                      # never dereferenced: a check fails first


def ptr(v):
    return ctypes.c_void_p(v)


def ffn(shape, backward=False, ws=ptr(FAKE), ws_bytes=1 << 40, grad=0, **over):
    L = bra.lib()
    p = dict(X=FAKE, W1=FAKE, b1=None, W2=FAKE, b2=None, Y=FAKE, pre=None, dY=FAKE, dX=FAKE, dW1=FAKE, dW2=FAKE, db1=None, db2=None)
    p.update(over)
    p = {k: ptr(v) for k, v in p.items()}
    s = ctypes.byref(shape) if shape is not None else None
    if not backward:
        return L.bra_ffn_forward(s, p["X"], p["W1"], p["b1"], p["W2"], p["b2"], p["Y"], p["pre"], ws, ws_bytes, None)
    return L.bra_ffn_backward(s, p["X"], p["W1"], p["b1"], p["W2"], p["pre"], p["dY"], p["dX"], p["dW1"], p["dW2"], p["db1"], p["db2"], grad, ws, ws_bytes, None)


@pytest.mark.parametrize("backward", [False, True])
def test_ffn_refusals(backward):
    S = lambda M=5, C=64, h=128, dtype=bra.BRA_BF16, act=0: bra.BraFfnShape(M, C, h, dtype, act)
    assert ffn(None, backward) == -1
    for bad in (S(M=-1), S(C=0), S(h=0), S(M=(1 << 30) + 1), S(C=(1 << 20) + 1), S(h=(1 << 20) + 1)):
        assert ffn(bad, backward) == -2
    assert ffn(S(dtype=7), backward) == -4
    assert ffn(S(act=2), backward) == -4
    for name in ("X", "W1", "W2") + (("dY", "dX", "dW1", "dW2") if backward else ("Y",)):
        assert ffn(S(), backward, **{name: None}) == -1, name
        assert ffn(S(), backward, **{name: FAKE + 8}) == -9, name
    assert ffn(S(), backward, b1=FAKE + 2) == -9
    assert ffn(S(), backward, pre=FAKE + 4) == -9
    assert ffn(S(C=63), backward, X=FAKE + 1) == -9                         # odd rows: elements' size
    assert ffn(S(C=63, dtype=bra.BRA_F32), backward, X=FAKE + 2) == -9
    assert ffn(S(C=63), backward, X=FAKE + 2, ws=None) == -5                # that alignment was fine
    for ws, n in ((None, 1 << 40), (ptr(FAKE + 64), 1 << 40), (ptr(FAKE), 16)):
        assert ffn(S(), backward, ws=ws, ws_bytes=n) == -5
    if backward:
        assert ffn(S(), True, grad=3) == -4
        assert ffn(S(), True, grad=bra.BRA_F32, db1=FAKE + 2) == -9
    else:
        assert ffn(S(M=0), False, X=None) == 0                              # nothing to do


def test_ffn_workspaces():
    for backward in (False, True):
        last = 0
        for M in (1, 64, 1000, 40000):
            n = bra.ffn_workspace_bytes(bra.make_ffn_shape(M, 256, 512, torch.bfloat16), backward)
            assert n % 256 == 0 and n >= last
            last = n
        # operands are laid out anew in float32 and where rows are no multiple of 8
        assert bra.ffn_workspace_bytes(bra.make_ffn_shape(1000, 256, 512, torch.float32), backward) > bra.ffn_workspace_bytes(bra.make_ffn_shape(1000, 256, 512, torch.bfloat16), backward)
        assert bra.ffn_workspace_bytes(bra.make_ffn_shape(1000, 255, 512, torch.bfloat16), backward) > bra.ffn_workspace_bytes(bra.make_ffn_shape(1000, 256, 512, torch.bfloat16), backward)
    assert bra.lib().bra_ffn_workspace_bytes(None, None) == -1
    # no size within the limits overflows
    assert bra.ffn_workspace_bytes(bra.make_ffn_shape(1 << 30, 1 << 20, 1 << 20, torch.bfloat16)) >= (1 << 51)


def norm_shape(rows=6, groups=1, C=64, dtype=bra.BRA_BF16, kind=0, eps=1e-6):
    return bra.BraNormShape(rows, groups, C, dtype, kind, eps)


def norm(shape, X=FAKE, Y=FAKE, R=FAKE, N=FAKE, params=True, **vec):
    p = bra.BraNormParams(**{k: v for k, v in dict(dict(gamma=FAKE), **vec).items()})
    return bra.lib().bra_norm_forward(ctypes.byref(shape) if shape is not None else None, ptr(X), ptr(Y), ctypes.byref(p) if params else None, ptr(R), ptr(N), None)


def test_norm_refusals():
    assert norm(None) == -1 and norm(norm_shape(), params=False) == -1
    for bad in (norm_shape(rows=-1), norm_shape(C=0), norm_shape(groups=0), norm_shape(groups=4), norm_shape(eps=-1.0), norm_shape(eps=float("nan")),
                norm_shape(rows=(1 << 30) + 1)):
        assert norm(bad) == -2
    assert norm(norm_shape(dtype=5)) == -4 and norm(norm_shape(kind=3)) == -4
    assert norm(norm_shape(C=8193)) == -6
    assert norm(norm_shape(), X=None) == -1
    assert norm(norm_shape(), R=None) == -1 and norm(norm_shape(), Y=None) == -1           # the sum goes with Y
    assert norm(norm_shape(), N=None) == -1 and norm(norm_shape(), gamma=None) == -1       # N goes with gamma
    assert norm(norm_shape(), Y=None, R=None, N=None, gamma=None) == -1                    # nothing to do
    assert norm(norm_shape(), X=FAKE + 1) == -9 and norm(norm_shape(dtype=0), Y=FAKE + 2) == -9 and norm(norm_shape(), scale=FAKE + 2) == -9
    assert norm(norm_shape(rows=0), X=None) == 0


def norm_backward(shape, R=FAKE, Y=FAKE, dN=FAKE, dR=None, ws=ptr(FAKE), ws_bytes=1 << 40, gamma=FAKE, **g):
    p = bra.BraNormParams(gamma=gamma)
    out = bra.BraNormGrads(**dict(dict(dX=FAKE, dY=FAKE), **g))
    return bra.lib().bra_norm_backward(ctypes.byref(shape), ptr(R), ptr(Y), ctypes.byref(p), ptr(dN), ptr(dR), ctypes.byref(out), ws, ws_bytes, None)


def test_norm_backward_refusals():
    S = norm_shape()
    assert norm_backward(S, R=None) == -1 and norm_backward(S, dX=None) == -1 and norm_backward(S, dY=None) == -1
    assert norm_backward(S, dN=None) == -1                                  # nothing came back
    assert norm_backward(S, gamma=None) == -1                               # dN goes with gamma
    assert norm_backward(S, dgamma=FAKE + 2) == -9 and norm_backward(S, dN=FAKE + 1) == -9
    for ws, n in ((None, 1 << 40), (ptr(FAKE + 16), 1 << 40), (ptr(FAKE), 8)):
        assert norm_backward(S, ws=ws, ws_bytes=n) == -5
    assert norm_backward(norm_shape(groups=5)) == -2 and norm_backward(norm_shape(C=9000)) == -6
    n = ctypes.c_size_t()
    assert bra.lib().bra_norm_backward_workspace_bytes(ctypes.byref(S), 1, None) == -1
    assert bra.lib().bra_norm_backward_workspace_bytes(ctypes.byref(S), 1, ctypes.byref(n)) == 0 and n.value > 0


def adamw(tensors, count=None, **over):
    a = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, bits=32, exp_avg=FAKE, exp_avg_sq=FAKE, exp_avg_scale=FAKE, exp_avg_sq_scale=FAKE)
    a.update(over)
    args = bra.BraAdamwArgs(**a)
    arr = (bra.BraAdamwTensor * max(1, len(tensors)))(*tensors)
    return bra.lib().bra_adamw_step(arr, len(tensors) if count is None else count, ctypes.byref(args), None)


def one(param=FAKE, grad=FAKE, copy=None, n=64, wd=0.0, p=0, g=0):
    return bra.BraAdamwTensor(param, grad, copy, n, wd, p, g)


def test_adamw_refusals():
    assert bra.lib().bra_adamw_step(None, 0, None, None) == -1
    assert adamw([one()], count=-1) == -2
    nan, inf = float("nan"), float("inf")
    for bad in (dict(lr=-1.0), dict(lr=nan), dict(lr=inf), dict(eps=-1e-8), dict(eps=nan), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=nan), dict(step=0)):
        assert adamw([one()], **bad) == -2, bad
    assert adamw([one(n=-1)]) == -2 and adamw([one(n=(1 << 34) + 1)]) == -2 and adamw([one(wd=-0.1)]) == -2 and adamw([one(wd=nan)]) == -2
    assert adamw([one()], bits=16) == -4 and adamw([one(p=2)]) == -4 and adamw([one(g=-1)]) == -4
    assert adamw([one(p=1, copy=FAKE)]) == -4                               # a copy of a bf16 parameter
    assert adamw([one(param=None)]) == -1
    assert adamw([one()], exp_avg=None) == -1 and adamw([one()], exp_avg_sq=None) == -1
    assert adamw([one()], bits=8, exp_avg_scale=None) == -1 and adamw([one()], bits=8, exp_avg_sq_scale=None) == -1
    assert adamw([one()], step_device=FAKE) == -1                           # no room for the scalars
    assert adamw([one(param=FAKE + 2)]) == -9 and adamw([one(grad=FAKE + 1, g=1)]) == -9 and adamw([one()], exp_avg=FAKE + 16) == -9
    assert adamw([one(), one()]) == -10                                     # the same parameter twice
    assert adamw([one(n=100), one(param=FAKE + 396)]) == -10                # one's end in the other
    assert adamw([one(copy=FAKE + 128)]) == -10
    assert adamw([]) == 0 and adamw([one(n=0)]) == 0 and adamw([one(grad=None)]) == 0


def test_strings():
    for code in (-9, -10):
        assert bra.strerror(code) != "unknown error code"


def test_python_refusals():
    X, W1, W2 = torch.zeros(4, 8), torch.zeros(8, 32), torch.zeros(16, 8)
    with pytest.raises(ValueError):
        bra.bra_ffn_forward(X, W1, W2)                                      # not on a GPU
    with pytest.raises(ValueError):
        bra.bra_ffn_forward(None, W1, W2)
    with pytest.raises(KeyError):
        bra.bra_ffn_forward(X, W1, W2, act="tanh")
    with pytest.raises(TypeError):
        bra.bra_ffn_forward("X", W1, W2)
    with pytest.raises(ValueError):
        bra.bra_ffn_backward(X, W1, W2, X)
    with pytest.raises(KeyError):
        bra.bra_ffn_backward(X, W1, W2, X, grad_dtype=torch.float16)
    g = torch.ones(8)
    with pytest.raises(ValueError):
        bra.bra_norm_forward(X, g)
    with pytest.raises(KeyError):
        bra.bra_norm_forward(X, g, kind="batch")
    with pytest.raises(ValueError):
        bra.bra_norm_backward(X, g, X)
    with pytest.raises(ValueError):
        bra.bra_adamw_step([X], [X], bra.adamw_state([X]), step=1)
    with pytest.raises(ValueError):
        bra.bra_adamw_step([X], [], {}, step=1)
    with pytest.raises(ValueError):
        bra.adamw_state([X], bits=4)
    assert bra.bra_adamw_step([], [], {}, step=1) is None


def test_adamw_state_layout():
    params = [torch.zeros(5, 7), torch.zeros(0), torch.zeros(64), torch.zeros(1)]
    s = bra.adamw_state(params)
    assert {k: (v.numel(), v.dtype) for k, v in s.items()} == {"exp_avg": (160, torch.float32), "exp_avg_sq": (160, torch.float32)}
    s = bra.adamw_state(params, 8)
    assert {k: (v.numel(), v.dtype) for k, v in s.items()} == {
        "exp_avg": (160, torch.float8_e4m3fn), "exp_avg_scale": (5, torch.float8_e8m0fnu), "exp_avg_root": (160, torch.float8_e4m3fn),
        "exp_avg_root_scale": (5, torch.float8_e8m0fnu)}
    assert not any(v.view(torch.uint8).any() for v in s.values())


def test_ffn_most_tokens():
    shape = bra.BraFfnShape(1 << 30, 8, 8, bra.BRA_BF16, 0)
    assert ffn(shape, True) == -2                           # 2^32 threads cannot be launched
    assert ffn(bra.BraFfnShape((1 << 30) - 1, 8, 8, bra.BRA_BF16, 0), True, ws=None) == -5
    assert ffn(shape, False, ws=None) == -5


@pytest.mark.parametrize("backward", [False, True])
def test_ffn_workspace_is_that_of_the_shape(backward):
    """A byte less than what a shape asks for is refused, whatever more tokens would ask for."""
    for M in (1, 130, 442, 519, 2045, 2052):
        n = bra.ffn_workspace_bytes(bra.make_ffn_shape(M, 768, 2048, torch.bfloat16), backward)
        assert ffn(bra.BraFfnShape(M, 768, 2048, bra.BRA_BF16, 0), backward, ws_bytes=n - 1) == -5
