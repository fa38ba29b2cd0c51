"""GPU tests of the gated block, the norms and AdamW at the widest and longest that their header allows: 2^20 channels or hidden units, 2^30 rows, a gate for every row,
a list of one-value tensors."""
import pytest
import torch

import paper_2303_08810_amd as bra
from ffn_util import F32 as U, UNIT, act64, make
from norm_util import check_backward, check_forward

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,C,h", [(1, 1 << 20, 8), (1, 8, 1 << 20), (3, 1, 1 << 20), (150, 1 << 20, 16), (150, 9, (1 << 20) - 1)])
def test_widest_blocks(M, C, h, dtype):
    """The 2-norm of the error: the results' own rounding and, in bf16, those of A, dG and dU, each below UNIT; float32 sums of up to 2^20 terms in partial sums of at most 2^16 grow like
    the square root of the terms, 256 2^-24, through two products."""
    X, W1, W2, dY, b1, b2 = make(M, C, h, dtype, True, seed=M)
    print(f"ffn {M} x {C} x {h} {dtype}", flush=True)
    limit = 2 * UNIT[BF16] if dtype == BF16 else 512 * U
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())
    Y = bra.bra_ffn_forward(X, W1, W2, b1=b1, b2=b2, act="gelu")
    P = X.double() @ W1.double() + b1.double()
    a, slope = act64(P[:, :h], "gelu")
    A = a * P[:, h:]
    assert rel(Y, A @ W2.double() + b2.double()) <= limit
    got = bra.bra_ffn_backward(X, W1, W2, dY, b1=b1, act="gelu", bias_grads=True, grad_dtype=F32)
    dA = dY.double() @ W2.double().t()
    dP = torch.cat([dA * P[:, h:] * slope, dA * a], 1)
    want = (dP @ W1.double().t(), X.double().t() @ dP, A.t() @ dY.double(), dP.sum(0), dY.double().sum(0))
    for name, g, w in zip(("dX", "dW1", "dW2", "db1", "db2"), got, want):
        assert rel(g, w) <= limit, name


@pytest.mark.parametrize("gated", [False, True])
def test_most_rows(gated):
    """2^30 rows of one channel, of which the first, middle and last ones are looked at; RMSNorm, for LayerNorm of one channel is 0."""
    rows = 1 << 30
    g = torch.Generator(device="cuda").manual_seed(4)
    X = torch.randn(rows, 1, generator=g, device="cuda", dtype=BF16)
    Y = X.roll(1, 0)
    P = dict(gamma=torch.tensor([1.5], device="cuda"), scale=torch.tensor([0.5], device="cuda"))
    if gated:
        P["gate"] = X.roll(-1, 0)
    print(f"norm 2^30 rows gated={gated}", flush=True)
    R, N = bra.bra_norm_forward(X, Y=Y, kind="rms", **P)
    grads = bra.bra_norm_backward(R, dN=X, dX=Y, Y=Y, kind="rms", **P)
    for at in (slice(0, 999), slice((1 << 29) - 500, (1 << 29) + 500), slice(rows - 777, rows)):
        few = {k: v[at].contiguous() if k == "gate" else v for k, v in P.items()}
        check_forward(R[at], N[at], X[at], Y[at], few, "rms", 1e-6)
        alone = bra.bra_norm_backward(R[at].contiguous(), dN=X[at].contiguous(), dX=Y[at].contiguous(), Y=Y[at].contiguous(), kind="rms", **few)
        check_backward(alone, R[at], Y[at], few, X[at], Y[at], "rms", 1e-6)
        for k in ("dX", "dY") + (("dgate",) if gated else ()):
            assert torch.equal(grads[k][at], alone[k]), k
    # sums over 2^30 rows; in float32, by threads of at most 2^13 rows, whose errors grow like the square root of their number
    total = sum(part.double().sum() for part in X.flatten().split(1 << 26))
    size = sum(part.double().abs().sum() for part in X.flatten().split(1 << 26))
    assert abs(float(grads["dbeta"]) - float(total)) <= 2.0 ** -24 * 128 * float(size)
    del X, Y, R, N, grads, P
    torch.cuda.empty_cache()


def test_many_tensors_of_one_value():
    n = 5000
    g = torch.Generator().manual_seed(6)
    w, d = torch.randn(n, generator=g).cuda(), torch.randn(n, generator=g).cuda()
    for bits in (32, 8):
        many, one = list(w.clone().split(1)), [w.clone()]
        state, flat = bra.adamw_state(many, bits), bra.adamw_state(one, 32)
        assert state["exp_avg"].numel() == 32 * n
        bra.bra_adamw_step(many, list(d.split(1)), state, step=1, lr=1e-2)
        bra.bra_adamw_step(one, [d], flat, step=1, lr=1e-2)
        assert torch.equal(torch.cat(many), one[0])
