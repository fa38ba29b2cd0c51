"""Outputs of attention between whole sequences and of the norms and rotation before it that share memory are refused; those that lie between other tensors of a buffer are not."""
import pytest
import torch

import paper_2303_08810_amd as bra

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_parts_of_one_buffer(dtype):
    B, N, H, Hk, d = 2, 50, 4, 2, 64
    X = torch.randn(B, N, 3 * H + 6 * Hk, d, generator=torch.Generator().manual_seed(0)).to(dtype).cuda()
    Q, K, V = X[:, :, :H], X[:, :, H:H + Hk], X[:, :, H + Hk:H + 2 * Hk]
    start, rest = H + 2 * Hk, X[:, :, H + 2 * Hk:]
    kept = X[:, :, :start].clone()
    O, lse = bra.bra_attention_forward(Q, K, V, want_lse=True)
    dO = torch.randn(B, N, H, d, generator=torch.Generator().manual_seed(1)).to(dtype).cuda()
    for first in range(start):          # H heads from one of the inputs' on
        with pytest.raises(ValueError):
            bra.bra_attention_forward(Q, K, V, out=X[:, :, first:first + H])
        with pytest.raises(ValueError):
            bra.bra_attention_backward(Q, K, V, O, lse, dO, out=(X[:, :, first:first + H], torch.empty_like(K), torch.empty_like(V)))
    for a, b in ((0, 1), (H - 1, H), (1, 0)):      # gradients that share a head
        with pytest.raises(ValueError):
            bra.bra_attention_backward(Q, K, V, O, lse, dO, out=(rest[:, :, :H], rest[:, :, H + a:H + a + Hk], rest[:, :, H + b:H + b + Hk]))
    if dtype == torch.float32:          # lse within a gradient
        wide = torch.zeros(B * N * H * d, device="cuda")
        inner = wide[:lse.numel()].view_as(lse).copy_(lse)
        with pytest.raises(ValueError):
            bra.bra_attention_backward(Q, K, V, O, inner, dO, out=(wide.view(B, N, H, d), torch.empty_like(K), torch.empty_like(V)))
    with pytest.raises(ValueError):
        bra.bra_qk_norm_forward(Q, K, out=(X[:, :, 1:H + 1], X[:, :, H:H + Hk]))
    with pytest.raises(ValueError):
        bra.bra_qk_norm_backward(Q, K, dO, K, out=(dO, X[:, :, H + 1:H + 1 + Hk]))
    # next to the inputs, every other head, in place
    got = bra.bra_attention_forward(Q, K, V, out=rest[:, :, :H])
    assert torch.equal(got, O) and torch.equal(X[:, :, :start], kept)
    got = bra.bra_attention_forward(Q, K, V, out=rest[:, :, 1:2 * H + 1:2])
    assert torch.equal(got, O) and torch.equal(X[:, :, :start], kept)
    want = bra.bra_attention_backward(Q, K, V, O, lse, dO)
    parts = rest[:, :, :H], rest[:, :, H:H + Hk], rest[:, :, H + Hk:H + 2 * Hk]
    for a, b in zip(bra.bra_attention_backward(Q, K, V, O, lse, dO, out=parts), want):
        assert torch.equal(a, b)
    assert torch.equal(X[:, :, :start], kept)
    cos, sin = bra.rotary_table(N, channels=d, device="cuda")
    want = bra.bra_qk_norm_forward(Q, K, cos=cos, sin=sin)
    got = bra.bra_qk_norm_forward(Q, K, cos=cos, sin=sin, out=(Q, K))
    assert got[0] is Q and got[1] is K and torch.equal(Q, want[0]) and torch.equal(K, want[1]) and torch.equal(V, kept[:, :, H + Hk:])
