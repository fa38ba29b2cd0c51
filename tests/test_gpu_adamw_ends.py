"""GPU test of the AdamW states behind a tensor's last value, which stay zero whatever the gradients and their scale are."""
import pytest
import torch

import paper_2303_08810_amd as bra

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("scale", [float("inf"), float("nan"), 0.5])
def test_zeros_behind_the_ends(bits, scale):
    sizes = [1, 7, 33, 2049, 64, 100]
    g = torch.Generator().manual_seed(1)
    p, grads = [torch.zeros(n, device="cuda") for n in sizes], [torch.randn(n, generator=g).cuda() for n in sizes]
    state = bra.adamw_state(p, bits)
    for t in (1, 2):
        bra.bra_adamw_step(p, grads, state, step=t, grad_scale=torch.tensor([scale], device="cuda"))
    at = 0
    for n in sizes:
        end = at + (n + 31) // 32 * 32
        for k in state:
            if not k.endswith("_scale"):
                assert not state[k][at + n:end].contiguous().view(torch.uint8).any(), (k, n)
        assert torch.isfinite(state["exp_avg"][at:at + n].float()).all() == (scale == 0.5)
        at = end
