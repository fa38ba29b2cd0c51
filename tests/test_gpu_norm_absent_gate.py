"""GPU test of bra_norm_backward at the C ABI: what a gate of ones has for its gradient, asked for without a gate, and without a scale."""
import ctypes

import pytest
import torch

import paper_2303_08810_amd as bra

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("groups,per,C", [(1, 100, 64), (3, 500, 40), (900, 40, 64), (5000, 2, 64), (1, 8, 192)])
def test_gradients_of_factors_that_are_absent(groups, per, C, post, dtype):
    g = torch.Generator().manual_seed(groups + C)
    r = lambda *s: torch.randn(*s, generator=g)
    R, Y, dN = (r(groups * per, C).to(dtype).cuda() for _ in range(3))
    vec = {k: (1 + 0.1 * r(C)).cuda() for k in ("gamma",) + (("post_gamma", "post_beta") if post else ())}
    shape = bra.BraNormShape(groups * per, groups, C, bra.BRA_F32 if dtype == F32 else bra.BRA_BF16, 0, 1e-6)
    need = ctypes.c_size_t()
    assert bra.lib().bra_norm_backward_workspace_bytes(ctypes.byref(shape), int(post), ctypes.byref(need)) == 0

    def backward(factors):
        ws = torch.empty(max(256, need.value), dtype=torch.uint8, device="cuda")
        out = {k: torch.full_like(R, 77.0) for k in ("dX", "dY")}
        out.update(dgate=torch.full((groups, C), 77.0, dtype=dtype, device="cuda"), dscale=torch.full((C,), 77.0, device="cuda"))
        p = bra.BraNormParams(**{k: v.data_ptr() for k, v in {**vec, **factors}.items()})
        grads = bra.BraNormGrads(**{k: v.data_ptr() for k, v in out.items()})
        ptr = lambda t: ctypes.c_void_p(t.data_ptr())
        rc = bra.lib().bra_norm_backward(ctypes.byref(shape), ptr(R), ptr(Y), ctypes.byref(p), ptr(dN), None, ctypes.byref(grads), ptr(ws), ws.numel(),
                                         ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
        assert rc == 0, rc
        torch.cuda.synchronize()
        return out

    gate, scale = torch.ones(groups, C, dtype=dtype, device="cuda"), torch.ones(C, device="cuda")
    want = backward(dict(gate=gate, scale=scale))
    for factors in (dict(), dict(gate=gate), dict(scale=scale)):
        got = backward(factors)
        assert all(torch.equal(got[k], want[k]) for k in want), (list(factors), [k for k in want if not torch.equal(got[k], want[k])])
