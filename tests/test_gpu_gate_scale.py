"""Renormalised weights of tokens whose chosen scores are tiny, or whose scale is large, against 64 bits.

A weight is at most the scale, whatever the scores: score / sum is at most 1. Tolerance, relative, in roundings of
2^-24: a score takes an exponential (4, by its documented bound), a sum, a quotient, and, below 2^-126, a spacing of 2^-149
(half of it at exp(-88.7) = 3.0e-39 is 4): 10 at most. A sum of such scores has the same 10 and at most 31 of its own, the
quotient and the product with the scale two more: 53.
"""
import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu

REL = 53 * 2.0 ** -24


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# a thread to a token; a warp to a token by the logits, and by scores plus a bias; the general way (few lanes to large groups)
@pytest.mark.parametrize("E,groups,T,biased", [(8, 1, 5000, False), (24, 3, 15000, True), (128, 1, 300, False), (256, 8, 300, True), (510, 3, 300, True)])
@pytest.mark.parametrize("k", [1, 8])
@pytest.mark.parametrize("scale,low,high", [(2.5, -88.7, -87.0), (1e30, -30.0, -20.0), (-3e38, -2.0, -1.0)])
def test_weights_of_tiny_scores(E, groups, T, biased, k, scale, low, high):
    x = low + (high - low) * torch.rand((T, E), device="cuda", generator=_gen(E + k))
    bias = None
    choice = x.double()
    if biased:  # it settles the choice: its steps are far above the scores, which are below 2^-2 (high > -10) or 1e-8
        order = torch.randperm(E, device="cuda", generator=_gen(k))
        bias = order.float() * (2.0 if high > -10 else 1e-3)
        choice = bias.double().expand(T, E)
    if groups > 1:
        best = choice.view(T, groups, -1).amax(2)
        kept = torch.zeros((T, groups), dtype=torch.bool, device="cuda").scatter_(1, best.argmax(1, keepdim=True), True)
        choice = choice.masked_fill(~kept.repeat_interleave(E // groups, dim=1), float("-inf"))
    want = torch.sort(choice, dim=1, descending=True, stable=True).indices[:, :k]
    s = torch.sigmoid(x.double()).gather(1, want)
    w = s / s.sum(1, keepdim=True) * scale
    chosen, got, _ = S.Router(E, k, score="sigmoid", groups=groups, top_groups=1, scale=scale).route(x, bias=bias)
    assert torch.equal(chosen.long(), want)
    assert ((got.double() - w).abs() <= REL * w.abs()).all()
    if k == 1:
        assert torch.equal(got, torch.full_like(got, scale))
