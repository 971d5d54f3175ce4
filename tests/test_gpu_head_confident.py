"""The head's gradients where the target is nearly certain, on the GPU, against 64 bits.

There p - 1 is a small difference, so that the gradient's logits have to be the loss's: with one way of summing for both, a sum's error e is in lse and in the
logit alike, and leaves the softmax of logits off by e: 2 e of each p, and of 1 - p. A sum of d products, added up anew every 1024 of them: at most
64 additions (of 16 products) of 2^-23 of the magnitudes, and d / 1024 of 2^-24. Of a largest logit l, five factors and sums are rounded on the way to lse and back (2^-24 of l
each, the two constants' own rounding among them by halves), and an exponential to 2^-22: eta. A logit's gradient is rounded to bf16 (2^-8 of it); dh and dW are sums of
K of them, K / 16 additions of 2^-23 of the magnitudes, rounded to bf16.
"""
import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


def _check(T, V, d, low, high, lay=lambda t: t):
    gen = torch.Generator(device="cuda").manual_seed(5)
    w = (torch.randn((V, d), device="cuda", generator=gen) * 0.05).to(BF16)
    targets = torch.randint(0, V, (T,), device="cuda", generator=gen)
    size = torch.linspace(low, high, T, device="cuda")[:, None]
    mine = w[targets].float()
    h = lay((mine * (size / (mine * mine).sum(1, keepdim=True))).to(BF16))  # the target's logit is `size`, of products that are not negative
    op = S.HeadLoss(V, d)
    _, lse = op.loss(h, w, targets)
    dh, dw = op.grad(h, w, targets, lse, torch.ones(T, device="cuda"))
    H, W, at = h.double(), w.double(), targets[:, None]
    x = H @ W.t()
    e = (64 * 2.0 ** -23 + (d / 1024 + 1) * 2.0 ** -24) * (H.abs() @ W.abs().t()).amax(1, keepdim=True)
    eta = 6 * 2.0 ** -24 * x.abs().amax(1, keepdim=True) + 2.0 ** -22
    p = torch.softmax(x, 1)
    q = p.clone().scatter_(1, at, 0.0).sum(1, keepdim=True)  # 1 - p of the target, without the difference
    near = p * (eta + 2 * e + 2.0 ** -8 * 1.01)
    near.scatter_(1, at, q * (2 * e + 2.0 ** -8 * 1.01) + eta * 1.01)
    p.scatter_(1, at, -q)
    for got, ref, terms, noise, K in ((dh, p @ W, p.abs() @ W.abs(), near @ W.abs(), V), (dw, p.t() @ H, p.t().abs() @ H.abs(), near.t() @ H.abs(), T)):
        allow = noise + (K / 16 + 1) * 2.0 ** -23 * (terms + noise) + 2.0 ** -8 * (ref.abs() + noise)
        bad = (got.double() - ref).abs() > allow + 1e-38
        assert not bad.any(), (int(bad.sum()), torch.nonzero(bad)[:4].tolist(), float(((got.double() - ref).abs() / (allow + 1e-38)).max()))
    op.sync_status()


def _apart(t):
    big = torch.empty((t.shape[0], t.shape[1] + 3), dtype=t.dtype, device="cuda")
    big[:, 1:1 + t.shape[1]] = t
    return big[:, 1:1 + t.shape[1]]


@pytest.mark.parametrize("T,V,d", [(64, 256, 8192), (300, 1000, 4096), (5, 130, 16384), (40, 300, 4099), (33, 64, 200)])
@pytest.mark.parametrize("low,high", [(60.0, 60.0), (4.0, 40.0)])
def test_targets_that_are_nearly_certain(T, V, d, low, high):
    _check(T, V, d, low, high)


def test_activations_off_16_byte_boundaries():
    _check(64, 256, 8192, 60.0, 60.0, lay=_apart)
