"""GPU tests of the gated feed-forward block and its gradients against 64 bits: sizes below, at and beyond the tiles' edges, sizes that
nothing divides, one token, both activations, with and without biases and given pre-activations."""
import pytest
import torch

import paper_2303_08810_amd as bra
from ffn_util import check_backward, check_forward, make

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32

SIZES = [  # (M, C, hidden)
    (1, 8, 8), (1, 64, 128), (1, 768, 2048), (2, 1, 1), (3, 5, 7), (5, 64, 64), (16, 256, 512), (17, 128, 344), (33, 96, 200), (64, 64, 64),
    (65, 72, 136), (100, 99, 261), (129, 128, 256), (200, 40, 1000), (257, 264, 520), (640, 512, 1365), (1000, 256, 512), (2049, 64, 176),
    (4100, 192, 384),
]
LARGE = [(9000, 768, 2048), (12544, 256, 512), (6000, 1000, 2730)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,C,h", SIZES)
def test_forward(M, C, h, dtype):
    act, bias = ("silu", "gelu")[(M + h) % 2], C % 3 != 0
    X, W1, W2, _, b1, b2 = make(M, C, h, dtype, bias, seed=M + 7 * C + h)
    print(f"ffn forward {M} x {C} x {h} {dtype} {act} bias={bias}", flush=True)
    Y, pre = bra.bra_ffn_forward(X, W1, W2, b1=b1, b2=b2, act=act, want_pre=True)
    Y2 = bra.bra_ffn_forward(X, W1, W2, b1=b1, b2=b2, act=act)
    assert torch.equal(Y, Y2)
    check_forward(Y, X, W1, W2, b1, b2, act, pre)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,C,h", SIZES)
def test_backward(M, C, h, dtype):
    act, bias, given = ("silu", "gelu")[(M + h) % 2], C % 3 != 0, M % 2 == 0
    X, W1, W2, dY, b1, b2 = make(M, C, h, dtype, bias, seed=M + 7 * C + h + 1)
    print(f"ffn backward {M} x {C} x {h} {dtype} {act} bias={bias} given={given}", flush=True)
    pre = bra.bra_ffn_forward(X, W1, W2, b1=b1, b2=b2, act=act, want_pre=True)[1] if given else None
    wide = torch.float32 if h % 2 else None
    grads = bra.bra_ffn_backward(X, W1, W2, dY, b1=b1, pre=pre, act=act, bias_grads=bias, grad_dtype=wide)
    assert len(grads) == (5 if bias else 3) and all(g.dtype == (wide or dtype) for g in grads[1:]) and grads[0].dtype == dtype
    check_backward(grads, X, W1, W2, dY, b1, act, pre, wide)
    again = bra.bra_ffn_backward(X, W1, W2, dY, b1=b1, pre=pre, act=act, bias_grads=bias, grad_dtype=wide)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))


@pytest.mark.parametrize("M,C,h", LARGE)
def test_large_tiles(M, C, h):
    X, W1, W2, dY, b1, b2 = make(M, C, h, BF16, True, seed=M)
    print(f"ffn large {M} x {C} x {h}", flush=True)
    Y, pre = bra.bra_ffn_forward(X, W1, W2, b1=b1, b2=b2, want_pre=True)
    check_forward(Y, X, W1, W2, b1, b2, "silu", pre)
    for given in (None, pre):
        check_backward(bra.bra_ffn_backward(X, W1, W2, dY, b1=b1, pre=given, bias_grads=True), X, W1, W2, dY, b1, "silu", given)


# Few rows of wide channels: contractions that are shared out and joined, in the forward, in dX and in the weights' gradients.
SHARED = [(33, 768, 2048), (40, 1001, 3900), (65, 1024, 2816), (129, 771, 2051), (257, 1024, 4096), (700, 331, 1401)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,C,h", SHARED)
def test_shared_contractions(M, C, h, dtype):
    act = ("silu", "gelu")[M % 2]
    X, W1, W2, dY, b1, b2 = make(M, C, h, dtype, C % 2 == 1, seed=M + C + h)
    print(f"ffn shared {M} x {C} x {h} {dtype} {act}", flush=True)
    shape = bra.make_ffn_shape(M, C, h, dtype, act)
    ws = torch.full((bra.ffn_workspace_bytes(shape),), 0xFF, dtype=torch.uint8, device="cuda")
    Y, pre = bra.bra_ffn_forward(X, W1, W2, b1=b1, b2=b2, act=act, want_pre=True, ws=ws)
    assert torch.equal(Y, bra.bra_ffn_forward(X, W1, W2, b1=b1, b2=b2, act=act))
    check_forward(Y, X, W1, W2, b1, b2, act, pre)
    for given in (None, pre):
        ws = torch.full((bra.ffn_workspace_bytes(shape, backward=True),), 0xFF, dtype=torch.uint8, device="cuda")
        grads = bra.bra_ffn_backward(X, W1, W2, dY, b1=b1, pre=given, act=act, bias_grads=True, ws=ws)
        check_backward(grads, X, W1, W2, dY, b1, act, given)
        again = bra.bra_ffn_backward(X, W1, W2, dY, b1=b1, pre=given, act=act, bias_grads=True)
        assert all(torch.equal(a, b) for a, b in zip(grads, again))
