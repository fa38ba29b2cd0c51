"""GPU tests of bra_ffn_backward at the C ABI: either bias's gradient asked for alone, in both types, with and without pre-activations, into memory that
holds something else."""
import ctypes

import pytest
import torch

import paper_2303_08810_amd as bra
from ffn_util import make

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("M,C,h", [(1, 8, 8), (300, 64, 128), (129, 99, 261), (5000, 128, 344), (0, 16, 24)])
def test_each_bias_alone(M, C, h, given, dtype):
    X, W1, W2, dY, b1, b2 = make(M, C, h, dtype, True, seed=M + h)
    print(f"ffn requests {M} x {C} x {h} {dtype} given={given}", flush=True)
    pre = bra.bra_ffn_forward(X, W1, W2, b1=b1, want_pre=True)[1] if given else None
    shape = bra.make_ffn_shape(M, C, h, dtype)
    ptr = lambda t: ctypes.c_void_p(t.data_ptr() if t is not None else None)
    for grad in (BF16, F32):
        def backward(asked):
            ws = torch.full((bra.ffn_workspace_bytes(shape, backward=True),), 0xFF, dtype=torch.uint8, device="cuda")
            new = lambda *s, t=grad: torch.full(s, 77.0, dtype=t, device="cuda")
            out = dict(dX=new(M, C, t=dtype), dW1=new(C, 2 * h), dW2=new(h, C))
            out.update({k: new(2 * h if k == "db1" else C) for k in asked})
            rc = bra.lib().bra_ffn_backward(ctypes.byref(shape), ptr(X), ptr(W1), ptr(b1), ptr(W2), ptr(pre), ptr(dY), ptr(out["dX"]), ptr(out["dW1"]), ptr(out["dW2"]),
                                            ptr(out.get("db1")), ptr(out.get("db2")), bra.BRA_F32 if grad == F32 else bra.BRA_BF16, ptr(ws), ws.numel(),
                                            ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
            assert rc == 0, rc
            torch.cuda.synchronize()
            return out
        want = dict(zip(("dX", "dW1", "dW2", "db1", "db2"), bra.bra_ffn_backward(X, W1, W2, dY, b1=b1, pre=pre, bias_grads=True, grad_dtype=grad)))
        for asked in ((), ("db1",), ("db2",), ("db1", "db2")):
            got = backward(asked)
            assert all(torch.equal(got[k], want[k]) for k in got), asked
