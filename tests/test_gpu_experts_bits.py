"""The matrices' gradient onto a base where tiles are cut along the rows: experts without rows keep the base's bits."""
import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


@pytest.mark.parametrize("grad", [BF16, F32])
@pytest.mark.parametrize("n,m", [(256, 256), (130, 391)])
def test_few_tiles_of_many_rows_keep_the_base_of_experts_without_rows(grad, n, m):
    """Bit for bit, NaN with its payload and signed zeros among it, into another tensor and in place."""
    E, R = 3, 30000  # few matrices, many rows: shares of the rows to several tiles, which a second launch adds
    gen = torch.Generator(device="cuda").manual_seed(1)
    make = lambda shape, dtype=BF16: torch.randn(shape, device="cuda", generator=gen).to(dtype)  # noqa: E731
    x, dy, base = make((R, n)), make((R, m)), make((E, n, m), grad)
    bits = torch.int16 if grad == BF16 else torch.int32
    base[0, ::7], base[2, 5], base[2, n - 1, m - 1] = -0.0, float("nan"), float("inf")
    base.view(bits)[2, 6] = 0x7F91 if grad == BF16 else 0x7F800001  # NaN of other bits
    offsets = torch.tensor([0, 0, R, R], dtype=torch.int32, device="cuda")
    op = S.Experts(E, n, m, grad_dtype=grad)
    want, keep = base[1].double() + x.double().t() @ dy.double(), base.clone()
    for out in (None, base):
        dw = op.grad(x, dy, offsets, base=base, out=out)
        for e in (0, 2):
            assert torch.equal(dw[e].view(bits), keep[e].view(bits))
        assert (dw[1].double() - want).norm() <= 2.0 ** -8 * want.norm()


def _at(shape, dtype, skew, seed=None, value=0.0):
    """A tensor that starts `skew` elements behind a 16-byte boundary, and what it lies in."""
    size = torch.Size(shape).numel()
    store = torch.full((size + 64,), value, dtype=dtype, device="cuda")
    t = store[skew:skew + size].view(shape)
    if seed is not None:
        t.copy_(torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype))
    return t, store


@pytest.mark.parametrize("grad", [BF16, F32])
@pytest.mark.parametrize("E,n,m", [(3, 1, 1), (4, 3, 5), (5, 129, 257), (2, 2000, 1031), (1024, 8, 9), (300, 40, 56)])
@pytest.mark.parametrize("base_at,out_at", [(0, 0), (3, 3), (1, 0), (0, 5), (2, 7)])
def test_matrices_of_experts_without_rows_are_the_bases(grad, E, n, m, base_at, out_at):
    """Wherever the two start; the others get their sums, and nothing behind or before the result is written."""
    bits = torch.int16 if grad == BF16 else torch.int32
    base = _at((E, n, m), grad, base_at, 3)[0]
    base.view(-1)[::11] = -0.0
    base.view(bits).view(-1)[5::1003] = 0x7F91 if grad == BF16 else 0x7F800001
    out, store = _at((E, n, m), grad, out_at, value=7.0)
    filled = sorted({E // 2, E - 1 if E % 2 else E // 2, *range(7, E, 100)})
    loads = [5 if e in filled else 0 for e in range(E)]
    R = sum(loads)
    offsets = torch.tensor([0, *torch.tensor(loads).cumsum(0).tolist()], dtype=torch.int32, device="cuda")
    x, dy = _at((R, n), BF16, 0, 1)[0], _at((R, m), BF16, 0, 2)[0]
    dw = S.Experts(E, n, m, grad_dtype=grad).grad(x, dy, offsets, base=base, out=out)
    assert dw is out and (store[:out_at] == 7).all() and (store[out_at + E * n * m:] == 7).all()
    still = torch.tensor([e for e in range(E) if e not in filled], device="cuda")
    assert torch.equal(out.view(bits)[still], base.view(bits)[still])
    o = offsets.tolist()
    for e in filled:
        i = slice(o[e], o[e + 1])
        want = base[e].double() + x[i].double().t() @ dy[i].double()
        ok = want.isfinite()
        # at most 5 products and a base, sums in fp32, one rounding
        size = base[e].double().abs() + x[i].double().abs().t() @ dy[i].double().abs()
        near = 6 * 2.0 ** -23 * size + (2.0 ** -8 if grad == BF16 else 2.0 ** -24) * want.abs()
        assert ((out[e].double() - want).abs() <= near)[ok].all() and out[e][~ok].isnan().all()


def test_no_tokens_leave_the_tables_base():
    """The head's gradient of no tokens, onto a base that holds NaN of any bits."""
    V, d = 1000, 72
    w, base = _at((V, d), BF16, 0, 1)[0], _at((V, d), BF16, 1, 2)[0]
    base.view(torch.int16).view(-1)[::13] = 0x7F91
    op = S.HeadLoss(V, d)
    h, ids, none = torch.empty((0, d), dtype=BF16, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    dw = op.grad(h, w, ids, none, none, base=base)[1]
    assert torch.equal(dw.view(torch.int16), base.view(torch.int16))
