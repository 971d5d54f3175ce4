"""The embedding's gradient onto a base, where the base and the output start at different places of a 16-byte unit."""
import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


@pytest.mark.parametrize("V,d,T", [(2000, 33, 100), (1500, 64, 300), (700, 257, 40), (40, 1000, 5)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("base_at,out_at", [(0, 1), (1, 0), (3, 5), (2, 6), (1, 9), (5, 5), (0, 4)])
def test_base_and_output_apart(V, d, T, dtype, base_at, out_at):
    """Rows without tokens are the base's bits; the others have the bits of a call on aligned tensors (the terms' order does not hang on
    alignment); what lies around the output stays."""
    g = torch.Generator(device="cuda").manual_seed(V + d)
    ids = torch.randint(-1, V, (T,), device="cuda", generator=g)
    dy = torch.randn((T, d), device="cuda", generator=g).to(dtype)
    whole = torch.randn(V * d + 16, device="cuda", generator=g).to(dtype)
    base = whole[base_at: base_at + V * d].view(V, d)
    around = torch.full((V * d + 32,), 7.0, dtype=dtype, device="cuda")
    out = around[out_at: out_at + V * d].view(V, d)
    e = S.Embedding(V, d, dtype, dtype, scale=0.5)
    want = e.grad(ids, dy, base=base.clone())
    keep = whole.clone()
    assert e.grad(ids, dy, base=base, out=out) is out
    assert torch.equal(out, want) and torch.equal(whole, keep)
    assert (around[:out_at] == 7).all() and (around[out_at + V * d:] == 7).all()
    empty = torch.ones(V, dtype=torch.bool, device="cuda")
    empty[ids[ids >= 0]] = False
    assert int(empty.sum()) > V // 2 and torch.equal(out[empty], base[empty])
    e.grad(ids, dy, base=base, out=base)      # in place, off a boundary
    assert torch.equal(base, want) and torch.equal(whole[:base_at], keep[:base_at]) and torch.equal(whole[base_at + V * d:], keep[base_at + V * d:])
