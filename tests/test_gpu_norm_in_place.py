"""GPU tests of the norms' gradients in the place of what they are formed from: dX in R's, dN's or dR's, dY in Y's, with rows that
leave teams of threads without one."""
import ctypes

import pytest
import torch

import paper_2303_08810_amd as bra

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


def backward(T, vec, gate, groups, dX, dY, kind, eps):
    rows, C = T["R"].shape
    shape = bra.BraNormShape(rows, groups, C, bra.BRA_F32 if T["R"].dtype == F32 else bra.BRA_BF16, kind, eps)
    need = ctypes.c_size_t()
    assert bra.lib().bra_norm_backward_workspace_bytes(ctypes.byref(shape), 1, ctypes.byref(need)) == 0
    ws = torch.empty(max(256, need.value), dtype=torch.uint8, device="cuda")
    out = {k: torch.empty(C, device="cuda") for k in ("dgamma", "dbeta", "dpost_gamma", "dpost_beta", "dscale")}
    out.update(dX=dX, dY=dY, dgate=torch.empty_like(gate))
    p = bra.BraNormParams(**{k: v.data_ptr() for k, v in vec.items()}, gate=gate.data_ptr())
    g = bra.BraNormGrads(**{k: v.data_ptr() for k, v in out.items()})
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())
    rc = bra.lib().bra_norm_backward(ctypes.byref(shape), ptr(T["R"]), ptr(T["Y"]), ctypes.byref(p), ptr(T["dN"]), ptr(T["dR"]), ctypes.byref(g), ptr(ws), ws.numel(),
                                     ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert rc == 0, rc
    torch.cuda.synchronize()
    return out


# a row more than the teams of a workgroup; parts of groups; many groups of few rows; teams of several wavefronts
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("groups,per,C", [(1, 33, 64), (1, 1000, 64), (3, 65, 40), (1700, 3, 64), (2, 7, 1024), (1, 3, 4096), (5, 9, 192)])
def test_in_place(groups, per, C, dtype):
    """eps = 0 and gradients of 0 in a group's last row: overwritten, that row's deviation is 0 and its normalised values are not numbers."""
    g = torch.Generator().manual_seed(groups + C)
    r = lambda *s: torch.randn(*s, generator=g)
    rows = groups * per
    T = {k: r(rows, C).to(dtype).cuda() for k in ("R", "Y", "dN", "dR")}
    for k in ("dN", "dR"):
        T[k][per - 1::per] = 0
    vec = {k: (1 + 0.1 * r(C)).cuda() for k in ("gamma", "post_gamma", "post_beta", "scale")}
    gate = r(groups, C).to(dtype).cuda()
    for kind in (bra.LAYERNORM, bra.RMSNORM):
        print(f"norm in place {groups} x {per} x {C} {dtype} {kind}", flush=True)
        want = backward(T, vec, gate, groups, torch.empty_like(T["R"]), torch.empty_like(T["R"]), kind, 0.0)
        assert all(torch.isfinite(v).all() for v in want.values())
        for x in ("R", "dN", "dR"):
            for _ in range(5):
                own = {k: v.clone() for k, v in T.items()}
                got = backward(own, vec, gate, groups, own[x], own["Y"], kind, 0.0)
                assert all(torch.equal(got[k], want[k]) for k in want), x
