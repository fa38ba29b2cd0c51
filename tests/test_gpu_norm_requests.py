"""GPU tests of bra_norm_backward at the C ABI: each gradient of a vector or of the gate asked for alone, into memory that holds something else."""
import ctypes

import pytest
import torch

import paper_2303_08810_amd as bra

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
VECTORS = ("dgamma", "dbeta", "dpost_gamma", "dpost_beta", "dscale")


def make(groups, per, C, dtype, seed, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)
    maps = {k: r(groups * per, C).to(dtype).to(device) for k in ("R", "Y", "dN", "dR")}
    vec = {k: (1 + 0.1 * r(C)).to(device) for k in ("gamma", "post_gamma", "post_beta", "scale")}
    return maps, vec, r(groups, C).to(dtype).to(device)


def backward(maps, vec, gate, groups, asked, kind=0, eps=1e-6):
    """The gradients of the maps and those `asked` for, every buffer poisoned before the call."""
    rows, C = maps["R"].shape
    dtype = maps["R"].dtype
    shape = bra.BraNormShape(rows, groups, C, bra.BRA_F32 if dtype == F32 else bra.BRA_BF16, kind, eps)
    need = ctypes.c_size_t()
    post = vec.get("post_gamma") is not None
    assert bra.lib().bra_norm_backward_workspace_bytes(ctypes.byref(shape), int(post), ctypes.byref(need)) == 0
    ws = torch.full((max(256, need.value),), 0xFF, dtype=torch.uint8, device="cuda")
    out = {k: torch.full_like(maps["R"], 77.0) for k in ("dX", "dY")}
    for k in asked:
        out[k] = torch.full((groups, C), 77.0, dtype=dtype, device="cuda") if k == "dgate" else torch.full((C,), 77.0, device="cuda")
    p = bra.BraNormParams(**{k: v.data_ptr() for k, v in vec.items()}, gate=None if gate is None else gate.data_ptr())
    g = bra.BraNormGrads(**{k: v.data_ptr() for k, v in out.items()})
    ptr = lambda t: ctypes.c_void_p(t.data_ptr())
    rc = bra.lib().bra_norm_backward(ctypes.byref(shape), ptr(maps["R"]), ptr(maps["Y"]), ctypes.byref(p), ptr(maps["dN"]), ptr(maps["dR"]), ctypes.byref(g), ptr(ws),
                                     ws.numel(), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert rc == 0, rc
    torch.cuda.synchronize()
    return out


# groups that come in parts; a group to a workgroup; several groups to a workgroup's teams; one workgroup for everything
CASES = [(1, 100, 64), (32, 1024, 192), (3, 500, 40), (900, 40, 64), (5000, 2, 64), (1, 8, 192)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("groups,per,C", CASES)
def test_each_alone(groups, per, C, dtype):
    maps, vec, gate = make(groups, per, C, dtype, seed=groups + C)
    print(f"norm requests {groups} x {per} x {C} {dtype}", flush=True)
    everything = backward(maps, vec, gate, groups, VECTORS + ("dgate",))
    for k in VECTORS + ("dgate",):
        alone = backward(maps, vec, gate, groups, (k,))
        for name in ("dX", "dY", k):
            assert torch.equal(alone[name], everything[name]), (k, name)
