"""A product that takes longer than a wait on the device may last without progress (some four seconds)."""
import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


def test_the_last_row_of_a_gradient_of_some_seconds():
    """The warp that clears what lies behind a group's last row waits for the first group that ends within a stage: here for one row
    behind some seconds of whole stages (384,000 rows of 65,536 columns; dy's lines are off 16-byte boundaries, which takes four times as long:
    5.2 s)."""
    n, R = 65536, 384000
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("100 GB of memory")
    big = torch.empty((R + 1, n + 8), dtype=BF16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    x, dy = big[:, :n], big[:, 1:n + 1]
    offsets = torch.tensor([0, R, R + 1], dtype=torch.int32, device="cuda")
    op = S.Experts(2, n, n)
    out = torch.empty((2, n, n), dtype=BF16, device="cuda")
    op.grad(x, dy, offsets, out=out)
    op.sync_status()
    a, b = x[R].float(), dy[R].float()
    for i in range(0, n, 4096):  # a product each, rounded once
        assert torch.equal(out[1, i:i + 4096], (a[i:i + 4096, None] * b).to(BF16))
    i = torch.tensor([0, 1, 127, 128, 255, 256, 33333, n - 257, n - 1], device="cuda")
    want = x[:R].index_select(1, i).double().t() @ dy[:R].index_select(1, i).double()
    # the sum's rounding to bf16, and additions on the tensor cores: 8192 products at a time of 2^-23 of sums of up to sqrt(R) in size (x dy's spread is 1), linear in their number
    size = R ** 0.5
    assert ((out[0][i][:, i].double() - want).abs() <= 2.0 ** -8 * want.abs() + (8192 / 16 * 2.0 ** -23 + (R / 8192 + 1) * 2.0 ** -24) * 6 * size).all()
