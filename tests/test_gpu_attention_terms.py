"""float32 attention keeps every product of terms: planes in memory, terms formed on the way to LDS, few rows on the float32 instruction; gradients over the planes and in one
launch (attention_terms_util.py has the checks, test_attention_terms_host.py what they notice)."""
import pytest

import torch

import paper_2303_08810_amd as bra
import attention_terms_util as terms
from test_gpu_attention_use import layer64

pytestmark = pytest.mark.gpu


class Kernels:
    @staticmethod
    def forward(Q, K, V, k_lens, scale):
        return bra.bra_attention_forward(Q, K, V, k_lens=k_lens, scale=scale, want_lse=True)

    @staticmethod
    def backward(Q, K, V, O, lse, dO, k_lens, scale):
        return bra.bra_attention_backward(Q, K, V, O, lse, dO, k_lens=k_lens, scale=scale)


# few rows; up to 256, 128 and 64 keys in LDS; planes, shared out or not
@pytest.mark.parametrize("check", terms.FORWARD, ids=lambda f: f.__name__)
@pytest.mark.parametrize("B,Nq,Nk,H,d", [(40, 8, 100, 3, 64), (5, 20, 3000, 3, 104), (8, 70, 60, 3, 64), (8, 70, 130, 3, 32), (8, 130, 250, 3, 24), (8, 70, 64, 3, 128), (8, 70, 300, 3, 64), (8, 140, 257, 3, 32),
                                         (8, 70, 65, 3, 72), (8, 200, 100, 3, 128), (4, 150, 3000, 2, 40), (2, 600, 2000, 2, 120)])
def test_forward(B, Nq, Nk, H, d, check):
    check(Kernels, B, Nq, Nk, H, d)


# one launch with sides of 32, 64 and 128; planes, two and four wavefronts, shared out or not
@pytest.mark.parametrize("check", terms.BACKWARD, ids=lambda f: f.__name__)
@pytest.mark.parametrize("B,Nq,Nk,H,d", [(40, 20, 30, 4, 64), (40, 30, 30, 4, 120), (40, 60, 50, 4, 64), (40, 100, 128, 4, 24), (40, 200, 60, 4, 64), (40, 60, 200, 4, 40), (40, 300, 300, 4, 32), (40, 130, 140, 4, 96),
                                         (40, 70, 40, 4, 128), (30, 1500, 700, 2, 72), (30, 900, 1100, 1, 128)])
def test_gradients(B, Nq, Nk, H, d, check):
    check(Kernels, B, Nq, Nk, H, d)


@pytest.mark.parametrize("B,Nq,Nk,H,d", [(2, 49, 49, 4, 32), (2, 60, 150, 3, 64), (1, 300, 300, 2, 128), (2, 700, 900, 2, 40), (1, 1300, 1300, 2, 72), (1, 3000, 2000, 1, 96), (3, 20, 500, 2, 64)])
def test_norms_of_the_errors(B, Nq, Nk, H, d):
    terms.norms(Kernels, B, Nq, Nk, H, d)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("N", [49, 150, 400])
def test_errors_of_a_layer(N, causal):
    """Norms and rotation, attention and back, whose errors in the 2-norm are attention's own, 1e-6 and 1.5e-6, and those of what the norms and the rotation round, some steps of 2^-24 of
    every value, forward and back: below 3e-6 together."""
    B, H, Hk, d = 2, 4, 2, 64
    g = torch.Generator().manual_seed(N)
    X, dO = torch.randn(B, N, H + 2 * Hk, d, generator=g).cuda(), torch.randn(B, N, H, d, generator=g).cuda()
    gq, gk = ((1 + 0.2 * torch.randn(d, generator=g)).cuda() for _ in range(2))
    cos, sin = bra.rotary_table(N, channels=d, device="cuda")
    Q, K = bra.bra_qk_norm_forward(X[:, :, :H], X[:, :, H:H + Hk], gq, gk, cos=cos, sin=sin)
    O, lse = bra.bra_attention_forward(Q, K, X[:, :, H + Hk:], causal=causal, want_lse=True)
    dQ, dK, dV = bra.bra_attention_backward(Q, K, X[:, :, H + Hk:], O, lse, dO, causal=causal)
    dXq, dXk, dgq, dgk = bra.bra_qk_norm_backward(X[:, :, :H], X[:, :, H:H + Hk], dQ, dK, gq, gk, cos=cos, sin=sin)
    live = [t.double().requires_grad_() for t in (X, gq, gk)]
    out = layer64(live[0], H, Hk, live[1], live[2], cos, sin, causal)
    want = torch.autograd.grad((out * dO.double()).sum(), live)
    for a, b in ((O, out.detach()), (torch.cat([dXq, dXk, dV], 2), want[0]), (dgq, want[1]), (dgk, want[2])):
        assert float((a.double() - b).norm() / b.norm()) <= 3e-6
