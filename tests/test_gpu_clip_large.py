"""Norm and clipping of sets over 2 GiB, which are cut into larger tiles, with dense gradients, against 64 bits.

A thread adds at most 32 squares in fp32 to each of two sums a tile of 32 KiB (16384 bf16 or 8192 fp32 elements, 256 threads),
whose own rounding and joining add three: the sum of squares is within 67 * 2^-24 with room to spare, the norm, rounded once, within half
of that and 2^-24, the factor within three more. A clipped element is one product and one rounding: bit for bit.
"""
import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu

NORM = 35 * 2.0 ** -24
GAMMA = NORM + 3 * 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
PIECE = 1 << 27


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


def _normal(n, dtype, skew, seed):
    t = torch.empty(n + skew, dtype=dtype, device="cuda")
    return t.normal_(0, 1e-3, generator=torch.Generator(device="cuda").manual_seed(seed))[skew:]


def _norm64(ts):
    return sum(float(p.double().square().sum()) for t in ts for p in t.split(PIECE)) ** 0.5


def _holds(out, g, gamma):
    return all(torch.equal(o, (p.float() * gamma).to(o.dtype)) for o, p in zip(out.split(PIECE), g.split(PIECE)))


def test_a_large_set_of_both_types():
    """Off a 16-byte boundary alike on both sides, on one side, and aligned; odd ends; into tensors of its own, and to bf16."""
    gs = [_normal((1 << 30) + 12345, BF16, 3, 1), _normal((1 << 26) + 5, F32, 1, 2), _normal((1 << 25) + 3, F32, 0, 3), _normal((1 << 24) + 9, BF16, 7, 4),
          _normal(5, BF16, 1, 5), _normal(1, F32, 0, 6)]
    assert sum(g.numel() * g.element_size() for g in gs) > 1 << 31
    bufs = [torch.full((g.numel() + 8,), 7.0, dtype=t, device="cuda") for g, t in zip(gs, (BF16, BF16, F32, BF16, BF16, F32))]
    skews = (3, 2, 4, 0, 5, 0)
    outs = [b[s: s + g.numel()] for b, s, g in zip(bufs, skews, gs)]
    want = _norm64(gs)
    c = S.GradClip(gs, out=outs)
    norm, gamma = c.clip(1.0).tolist()
    assert abs(norm - want) <= NORM * want
    factor = min(1.0, 1.0 / (want + 1e-6))
    assert abs(gamma - factor) <= GAMMA * factor and gamma < 1.0
    for b, s, g, o in zip(bufs, skews, gs, outs):
        assert _holds(o, g, gamma)
        assert (b[:s] == 7).all() and (b[s + g.numel():] == 7).all()
    assert c.norm(1.0).tolist() == [norm, gamma]
    assert abs(_norm64(gs) - want) == 0.0


def test_a_large_set_in_place():
    gs = [_normal((1 << 30) + 77, BF16, 1, 7), _normal((1 << 20) + 1, F32, 2, 8)]
    keep = [g.clone() for g in gs]
    want = _norm64(gs)
    norm, gamma = S.GradClip(gs).clip(0.5).tolist()
    assert abs(norm - want) <= NORM * want
    for g, k in zip(gs, keep):
        assert _holds(g, k, gamma)
