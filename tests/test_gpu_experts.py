"""Products grouped by expert on the GPU, against 64 bits.

Products of two bf16 numbers are exact in fp32. A sum of K of them on the tensor cores, in whatever order, with every addition off by at most
2^-23 (fp32, truncated) of the magnitudes: K * 2^-23 of the sum of magnitudes; then one rounding to the result's type (half a step: 2^-8 in bf16,
2^-24 in fp32), and one of 2^-24 where a base is added. That bound is wide where K is large, so that the 2-norm of
all errors is held to K / 16 additions (16 products enter at a time) of 2^-23 of the result's, beside the last rounding.
"""
import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
STEP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


def _randn(shape, seed, dtype=BF16):
    return torch.randn(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


def _offsets(loads, first=0):
    return torch.tensor([first] + [first + sum(loads[:i + 1]) for i in range(len(loads))], dtype=torch.int32, device="cuda")


def _near(got, want, terms, K, dtype, what):
    assert got.dtype == dtype and got.shape == want.shape
    err = (got.double() - want).abs()
    bad = err > K * 2.0 ** -23 * terms + STEP[dtype] * want.abs() * 1.001 + 1e-38
    assert not bad.any(), (what, int(bad.sum()), torch.nonzero(bad)[:4].tolist(), float(err.max()))
    assert float(err.norm()) <= (K / 16 * 2.0 ** -23 + STEP[dtype] + 2.0 ** -24) * float(want.norm()) * 2 + 1e-30, what


def _check(loads, n, m, row=BF16, grad=BF16, first=0, behind=0, lay=None, base=False, garbage=float("nan")):
    E, used = len(loads), sum(loads)
    R = first + used + behind
    lay = lay or (lambda t: t)
    op = S.Experts(E, n, m, row_dtype=row, grad_dtype=grad)
    x, dy, w, offsets = lay(_randn((R, n), 1)), lay(_randn((R, m), 2)), _randn((E, n, m), 3), _offsets(loads, first)
    for t in (x, dy):  # rows of no expert enter nothing
        t[:first], t[first + used:] = garbage, garbage
    y, dx = op.product(x, w, offsets), op.grad_rows(dy, w, offsets)
    b = _randn((E, n, m), 4, grad) if base else None
    dw = op.grad(x, dy, offsets, base=b)
    want = [torch.zeros(s, dtype=torch.float64, device="cuda") for s in ((R, m), (R, n), (E, n, m))]
    terms = [t.clone() for t in want]
    o = offsets.tolist()
    for e in range(E):
        i = slice(o[e], o[e + 1])
        X, D, W = x[i].double(), dy[i].double(), w[e].double()
        for at, k, a, c in ((i, 0, X, W), (i, 1, D, W.t()), (e, 2, X.t(), D)):
            want[k][at], terms[k][at] = a @ c, a.abs() @ c.abs()
    if base:
        want[2] += b.double()
        terms[2] += b.double().abs()
    _near(y, want[0], terms[0], n, row, "product")
    _near(dx, want[1], terms[1], m, row, "grad_rows")
    _near(dw, want[2], terms[2], max(loads + [1]), grad, "grad")
    for t in (y, dx):
        assert (t[:first] == 0).all() and (t[first + used:] == 0).all()
    assert torch.equal(y, op.product(x, w, offsets)) and torch.equal(dw, op.grad(x, dy, offsets, base=b))  # the same bits again
    if base:
        keep = b.clone()
        op.grad(x, dy, offsets, base=b, out=b)
        assert torch.equal(b, dw)
        for e in range(E):
            if not loads[e]:
                assert torch.equal(b[e], keep[e])
    op.sync_status()


LOADS = [[1], [0, 1, 0], [900, 3, 0, 700], [127, 128, 129], [64, 0, 0, 300, 5], [1] * 40, [255, 256, 257, 1, 0], [700]]


@pytest.mark.parametrize("loads", LOADS, ids=lambda v: "-".join(map(str, v[:5])))
@pytest.mark.parametrize("n,m", [(64, 64), (8, 8), (256, 128), (200, 328), (1, 1), (65, 130), (127, 64), (136, 71)])
def test_products(loads, n, m):
    _check(loads, n, m)
    _check(loads, n, m, F32, F32, first=3, behind=5, base=True)


@pytest.mark.parametrize("loads", [[300, 0, 200], [5, 1]], ids=str)
@pytest.mark.parametrize("n,m", [(1024, 512), (4096, 264), (520, 2000), (1000, 511), (2049, 384)])
def test_wider_matrices(loads, n, m):
    _check(loads, n, m, base=True, behind=1)


def test_no_rows():
    op = S.Experts(3, 16, 24)
    x, dy = torch.empty((0, 16), dtype=BF16, device="cuda"), torch.empty((0, 24), dtype=BF16, device="cuda")
    w, o = _randn((3, 16, 24), 1), torch.zeros(4, dtype=torch.int32, device="cuda")
    assert op.product(x, w, o).shape == (0, 24) and op.grad_rows(dy, w, o).shape == (0, 16)
    assert (op.grad(x, dy, o) == 0).all()
    b = _randn((3, 16, 24), 2)
    assert torch.equal(op.grad(x, dy, o, base=b), b)
    # rows, but none of any expert
    x, dy = _randn((50, 16), 1), _randn((50, 24), 2)
    assert (op.product(x, w, o) == 0).all() and (op.grad_rows(dy, w, o) == 0).all() and (op.grad(x, dy, o) == 0).all()


def test_many_experts():
    _check([(i * 7) % 5 for i in range(1024)], 72, 40)
    _check([0] * 1023 + [33], 40, 72)


def test_strides_and_alignment():
    def apart(t):
        big = torch.full((t.shape[0], t.shape[1] + 40), float("nan"), dtype=t.dtype, device="cuda")
        big[:, 16:16 + t.shape[1]] = t
        return big[:, 16:16 + t.shape[1]]

    def off(t):
        big = torch.full((t.shape[0], t.shape[1] + 5), float("nan"), dtype=t.dtype, device="cuda")
        big[:, 1:1 + t.shape[1]] = t
        return big[:, 1:1 + t.shape[1]]
    for lay in (apart, off):
        _check([100, 0, 31], 192, 320, lay=lay, behind=2)
        _check([3], 200, 72, lay=lay)


def test_matrices_off_16_bytes():
    """W, base and dW that start off a 16-byte boundary."""
    E, n, m, loads = 2, 64, 128, [70, 60]
    def off(t):
        big = torch.empty(t.numel() + 1, dtype=t.dtype, device="cuda")
        big[1:] = t.reshape(-1)
        return big[1:].view(t.shape)
    op, x, dy, o = S.Experts(E, n, m), _randn((130, n), 1), _randn((130, m), 2), _offsets(loads)
    w = _randn((E, n, m), 3)
    y, dx, dw = op.product(x, w, o), op.grad_rows(dy, w, o), op.grad(x, dy, o, base=w)
    assert torch.equal(op.product(x, off(w), o), y) and torch.equal(op.grad_rows(dy, off(w), o), dx)
    assert torch.equal(op.grad(x, dy, o, base=off(w), out=off(torch.zeros_like(w))), dw)


@pytest.mark.parametrize("grad", [BF16, F32])
@pytest.mark.parametrize("m", [384, 392, 391, 130, 3])
def test_the_base_of_experts_without_rows_stays_as_it_is(grad, m):
    """Bit for bit, NaN and signed zeros among it, into another tensor, wherever the two start."""
    E, n = 5, 300
    loads = [0, 40, 0, 0, 7]
    op, x, dy, o = S.Experts(E, n, m, grad_dtype=grad), _randn((47, n), 1), _randn((47, m), 2), _offsets(loads)
    for skew in (0, 1):
        store = torch.zeros(E * n * m + 1, dtype=grad, device="cuda")
        base = store[skew:skew + E * n * m].view(E, n, m)
        base.copy_(_randn((E, n, m), 3, grad))
        base[0, ::7], base[2, 5], base[3, 299, m - 1] = -0.0, float("nan"), float("inf")
        dw = op.grad(x, dy, o, base=base)
        bits = torch.int16 if grad == BF16 else torch.int32
        for e in (0, 2, 3):
            assert torch.equal(dw[e].view(bits), base[e].view(bits))
        want = base[1].double() + x[:40].double().t() @ dy[:40].double()
        assert (dw[1].double() - want).norm() <= 2.0 ** -8 * want.norm()


def test_infinities_and_nan_stay_in_their_rows():
    E, n, m = 2, 128, 96
    x, w, o = _randn((200, n), 1), _randn((E, n, m), 2), _offsets([90, 110])
    op = S.Experts(E, n, m)
    plain = op.product(x, w, o)
    x[10, 3], x[89, 0] = float("nan"), float("inf")
    y = op.product(x, w, o)
    rest = torch.ones(200, dtype=torch.bool, device="cuda")
    rest[[10, 89]] = False
    assert torch.equal(y[rest], plain[rest]) and y[10].isnan().all() and not y[89].isfinite().any()
    dy = _randn((200, m), 3)
    dw = op.grad(x, dy, o)
    assert dw[1].isfinite().all() and dw[0, 3].isnan().all() and dw[0, 5].isfinite().all()


@pytest.mark.parametrize("offsets", [[0, 50, 30, 60], [-5, 20, 20, 70], [10, 40, 1000, 2000], [0, 0, 0, 0], [90, 95, 99, 10**9]])
def test_offsets_that_no_order_made(offsets):
    """Taken as they come: within the rows, and none below the one before."""
    R, n, m = 64, 40, 48
    op, x, w, dy = S.Experts(3, n, m), _randn((R, n), 1), _randn((3, n, m), 2), _randn((R, m), 3)
    o = torch.tensor(offsets, dtype=torch.int32, device="cuda")
    clean, last = [], 0
    for v in offsets:
        last = max(last, min(max(v, 0), R))
        clean.append(last)
    c = torch.tensor(clean, dtype=torch.int32, device="cuda")
    assert torch.equal(op.product(x, w, o), op.product(x, w, c)) and torch.equal(op.grad(x, dy, o), op.grad(x, dy, c))
    want = torch.zeros((R, m), dtype=torch.float64, device="cuda")
    for e in range(3):
        want[clean[e]:clean[e + 1]] = x[clean[e]:clean[e + 1]].double() @ w[e].double()
    assert (op.product(x, w, o).double() - want).norm() <= 2.0 ** -8 * want.norm()


def test_matrices_past_2_31_elements():
    E, n, m = 160, 4096, 4096  # 2.7e9 elements
    loads = [0] * E
    loads[0], loads[77], loads[E - 1] = 3, 200, 5
    x, dy, o = _randn((208, n), 1), _randn((208, m), 2), _offsets(loads)
    w = torch.zeros((E, n, m), dtype=BF16, device="cuda")
    for e in (0, 77, E - 1):
        w[e] = _randn((n, m), e)
    op = S.Experts(E, n, m)
    y, dx, dw = op.product(x, w, o), op.grad_rows(dy, w, o), op.grad(x, dy, o)
    for e in (0, 77, E - 1):
        a, b = int(o[e]), int(o[e + 1])
        for got, want in ((y[a:b], x[a:b].double() @ w[e].double()), (dx[a:b], dy[a:b].double() @ w[e].double().t()), (dw[e], x[a:b].double().t() @ dy[a:b].double())):
            assert (got.double() - want).norm() <= 2.0 ** -8 * want.norm()
    assert not dw[1].any() and not dw[E - 2].any()


def test_a_long_sum():
    """One expert of many rows: the matrices' gradient sums over all of them."""
    _check([70001], 72, 136)


@pytest.mark.parametrize("loads,n,m", [([70001], 73, 137), ([9000, 0, 20001], 264, 520), ([300, 0, 7], 3001, 40), ([500], 41, 5000), ([3], 9000, 24)])
def test_long_sums_in_fp32(loads, n, m):
    """Sums that are taken out of the tensor cores several times, of lines on 16-byte boundaries and off them: as near as fp32 is, however long."""
    _check(loads, n, m, F32, F32, base=True, behind=1)
    x, w, o = _randn((sum(loads), n), 1).abs(), _randn((len(loads), n, m), 2).abs(), _offsets(loads)
    y = S.Experts(len(loads), n, m, row_dtype=F32).product(x, w, o)
    want = torch.cat([x[o[e]:o[e + 1]].double() @ w[e].double() for e in range(len(loads))])
    # 32 additions of 16 products each, rounded down by at most 2^-23 of a sum that grows to its size, so by half of that on average; then n / 512 of 2^-24
    assert float((y.double() - want).norm()) <= (32 * 2.0 ** -24 + n / 512 * 2.0 ** -24) * float(want.norm())


def test_a_wait_that_gives_up_is_reported_once():
    op = S.Experts(2, 64, 64)
    x, w, o = _randn((100, 64), 1), _randn((2, 64, 64), 2), _offsets([40, 60])
    y = op.product(x, w, o)
    op.sync_status()
    S.skew_ops_selftest_wait_timeout(torch.cuda.current_stream().cuda_stream)
    with pytest.raises(S.SkewError) as e:
        op.sync_status()
    assert e.value.code == S.SKEW_ETIMEOUT
    op.sync_status()
    assert torch.equal(op.product(x, w, o), y)


def test_gradients_are_the_products_by_differences():
    """<dy, y(x + t u)> changes by t <dx, u>, and likewise in w: y is linear in both."""
    E, n, m, loads = 3, 48, 80, [10, 0, 25]
    o, op = _offsets(loads), S.Experts(E, n, m, row_dtype=F32, grad_dtype=F32)
    x, w, dy = _randn((35, n), 1), _randn((E, n, m), 2), _randn((35, m), 3)
    u, v = _randn((35, n), 4), _randn((E, n, m), 5)
    dot = lambda a, b: float((a.double() * b.double()).sum())  # noqa: E731
    sizes = lambda a, b: float((a.double() * b.double()).abs().sum())  # noqa: E731
    for got, want, scale in ((dot(op.product(u, w, o), dy), dot(op.grad_rows(dy, w, o), u), sizes(op.product(u, w, o), dy)),
                             (dot(op.product(x, v, o), dy), dot(op.grad(x, dy, o), v), sizes(op.product(x, v, o), dy))):
        assert abs(got - want) <= 80 * 2.0 ** -23 * 10 * scale  # (sums of up to 80 products; magnitudes exceed the sums' by less than 10)
