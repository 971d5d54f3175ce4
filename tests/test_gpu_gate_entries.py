"""The logits' gradient where `chosen` names experts that are not there, beside ones that are, against 64 bits.

An entry outside [0, experts) has no weight and no gradient, whatever its dweights. Tolerance as for the whole gradient: an exponential of a
logit difference of at most 40 carries 40 roundings of 2^-24, and 60 more cover the sums and products, relative to the sum of
the terms' magnitudes.
"""
import math

import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu

REL = 100 * 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


@pytest.mark.parametrize("E,k,T", [(5, 3, 700), (33, 4, 701), (128, 8, 700), (500, 32, 90)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True])
def test_entries_that_name_no_expert(E, k, T, score, renorm):
    g = torch.Generator(device="cuda").manual_seed(E + T)
    x = torch.randn((T, E), device="cuda", generator=g) * 2
    chosen = torch.rand((T, E), device="cuda", generator=g).argsort(dim=1)[:, :k].int()
    outside = torch.tensor([E, E + 1, 2 * E, 1 << 20, (1 << 31) - 1, -1, -2, -E, -(1 << 31)], device="cuda").int()
    bad = torch.rand((T, k), device="cuda", generator=g) < 0.4
    bad[:10] = True                                    # none that is there
    bad[10:20, 1:] = True
    bad[10:20, 0] = False                              # one
    chosen[bad] = outside[torch.randint(0, len(outside), (int(bad.sum()),), device="cuda", generator=g)]
    dw = torch.randn((T, k), device="cuda", generator=g)
    dw[bad] = math.inf
    dx = S.Router(E, k, score=score, renorm=renorm, scale=1.5).grad(x, chosen, dw)
    # the formula, over those that are there
    at = chosen.long().masked_fill(bad, 0)
    s = torch.softmax(x.double(), 1) if score == "softmax" else torch.sigmoid(x.double())
    rest = torch.ones_like(s) if score == "softmax" else 1 - s
    p, d = s.gather(1, at).masked_fill(bad, 0.0), (dw.double() * 1.5).masked_fill(bad, 0.0)
    if renorm:
        q = p / p.sum(1, keepdim=True).clamp(min=1e-300)
        v, size = q * (d - (d * q).sum(1, keepdim=True)), q * (d.abs() + (d * q).abs().sum(1, keepdim=True))
        v, size = v * rest.gather(1, at), size
    elif score == "sigmoid":
        v = size = d * p * rest.gather(1, at)
    if renorm or score == "sigmoid":
        want = torch.zeros_like(s).scatter_add_(1, at, v.masked_fill(bad, 0.0))
        size = torch.zeros_like(s).scatter_add_(1, at, size.abs().masked_fill(bad, 0.0))
    else:
        ds = torch.zeros_like(s).scatter_add_(1, at, d)
        dot = (ds * s).sum(1, keepdim=True)
        want, size = s * (ds - dot), s * (ds.abs() + (ds * s).abs().sum(1, keepdim=True))
    assert dx.isfinite().all() and (dx[:10] == 0).all()
    assert ((dx.double() - want).abs() <= REL * size + 1e-38).all()
    assert renorm or int((want != 0).sum()) > T  # there is something to be wrong
