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
