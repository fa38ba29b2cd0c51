"""Flags of the binding: what has no truth value raises its own exception, before anything else is looked at (no GPU)."""
import pytest
import torch

import paper_2303_08810_amd as bra


class NoTruth:
    def __bool__(self):
        raise ZeroDivisionError("no truth value")


@pytest.mark.parametrize("flag", [NoTruth(), torch.zeros(2)], ids=["object", "tensor"])
def test_what_has_no_truth_value(flag):
    error = ZeroDivisionError if isinstance(flag, NoTruth) else RuntimeError
    X, Q = torch.zeros(1, 8, 8, 32), torch.zeros(1, 5, 2, 32)
    W, Wo, Wl = torch.zeros(32, 96), torch.zeros(32, 32), torch.zeros(32, 5, 5)
    params = {n: torch.zeros(1) for n in bra.BraBlockParams.FIELDS}
    params["W1"] = torch.zeros(32, 64)
    for call in (lambda: bra.bra_route(X, W, 2, 1, 1, want_Ar=flag),
                 lambda: bra.bra_forward(X, W, Wo, Wl, 2, 1, 1, want_Ir=flag),
                 lambda: bra.bra_forward_padded(X, W, Wo, Wl, 2, 1, 1, want_Ir=flag),
                 lambda: bra.bra_block_forward(X, params, 2, 1, 1, want_Ir=flag),
                 lambda: bra.bra_ffn_forward(X, W, Wo, want_pre=flag),
                 lambda: bra.bra_ffn_backward(X, W, Wo, X, bias_grads=flag),
                 lambda: bra.bra_attention_forward(Q, Q, Q, want_lse=flag),
                 lambda: bra.bra_attention_forward(Q, Q, Q, causal=flag),
                 lambda: bra.bra_attention_backward(Q, Q, Q, Q, Q, Q, causal=flag)):
        with pytest.raises(error) as info:
            call()
        assert type(info.value) is error
    with pytest.raises(ValueError):
        bra.bra_attention_forward(Q, Q, Q, want_lse=1, causal=[])          # what `if` takes; refused for its place in memory
