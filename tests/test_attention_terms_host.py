"""The checks of attention_terms_util.py on an emulation of attention in three bf16 terms (CPU): six products pass them, and with any one left out anywhere they fail."""
import pytest
import torch

import attention_terms_util as terms

SIX = ((2, 0), (0, 2), (1, 1), (1, 0), (0, 1), (0, 0))
SIZE = dict(B=6, Nq=40, Nk=9, H=3, d=16, device="cpu")


def split3(x):
    out = []
    for _ in range(3):
        out.append(x.bfloat16().float())
        x = x - out[-1]
    return out


class Emulated:
    """`lost`: (which product, pair of terms) that is left out, or the pairs left out everywhere."""

    def __init__(self, lost=()):
        self.lost = lost

    def mm(self, name, a, b):
        a, b = split3(a), split3(b)
        out = torch.zeros(*a[0].shape[:-1], b[0].shape[-1])
        for pair in SIX:
            if pair not in self.lost and (name, pair) not in self.lost:
                out = out + a[pair[0]] @ b[pair[1]]
        return out

    def _scores(self, Q, K, k_lens, scale):
        self.scale = Q.shape[-1] ** -0.5 if scale is None else scale
        q, k = (x.transpose(1, 2) for x in (Q, K))
        s = self.mm("S", q, k.transpose(-1, -2)) * self.scale
        if k_lens is not None:
            s = s.masked_fill(torch.arange(K.shape[1]) >= k_lens.view(-1, 1, 1, 1), -torch.inf)
        return s

    def forward(self, Q, K, V, k_lens, scale):
        s = self._scores(Q, K, k_lens, scale)
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(-1, keepdim=True)
        return (self.mm("PV", p, V.transpose(1, 2)) / total).transpose(1, 2), (top + torch.log(total)).squeeze(-1)

    def backward(self, Q, K, V, O, lse, dO, k_lens, scale):
        q, k, v, o, g = (x.transpose(1, 2) for x in (Q, K, V, O, dO))
        p = torch.exp(self._scores(Q, K, k_lens, scale) - lse.unsqueeze(-1))
        ds = p * (self.mm("dP", g, v.transpose(-1, -2)) - (g * o).sum(-1, keepdim=True))
        out = self.mm("dQ", ds, k) * self.scale, self.mm("dK", ds.transpose(-1, -2), q) * self.scale, self.mm("dV", p.transpose(-1, -2), g)
        return [x.transpose(1, 2) for x in out]


def fails(lost):
    found = []
    for check in terms.FORWARD + terms.BACKWARD:
        try:
            check(Emulated(lost), **SIZE)
        except AssertionError:
            found.append(check.__name__)
    return found


def test_six_products_pass():
    assert fails(()) == []
    terms.norms(Emulated(), B=2, Nq=60, Nk=150, H=3, d=64, device="cpu")


@pytest.mark.parametrize("pair", SIX[:5], ids=lambda p: "%d%d" % p)
@pytest.mark.parametrize("where,check", [("S", "scores"), ("S", "scores_again"), ("PV", "weights"), ("dP", "query_gradients"), ("dP", "key_gradients"), ("dQ", "query_gradients"),
                                         ("dK", "key_gradients"), ("dV", "value_gradients")])
def test_five_do_not(where, pair, check):
    assert check in fails([(where, pair)])


def test_three_do_not():
    for size in (dict(B=2, Nq=60, Nk=150, H=3, d=64), dict(B=1, Nq=300, Nk=300, H=2, d=128)):
        with pytest.raises(AssertionError):
            terms.norms(Emulated(SIX[:3]), device="cpu", **size)
    assert "values" in fails(SIX[:2])
