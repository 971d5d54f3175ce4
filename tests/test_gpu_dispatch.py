"""Rows by expert and back on the GPU, against an order by sorting and against 64 bits.

Places and offsets are whole numbers: equal. A spread row is a cast: bit for bit. A combined element is a sum of top_k products in fp32, each
addition fused: at most top_k roundings of 2^-24 of the terms' magnitudes, then one to the result's type (half a step: 2^-8 in bf16, 2^-24 in fp32).
A row's gradient is one product in fp32, then that rounding. A weight's gradient is a sum of `width` products, up to width / 32 + 8 of them in
a row, then five sums across lanes: at most width / 32 + 13 roundings of 2^-24 of the magnitudes.
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


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(shape, dtype, seed):
    return torch.randn(shape, device="cuda", generator=_gen(seed)).to(dtype)


def _chosen(kind, T, k, E, seed=1):
    g = _gen(seed)
    if kind == "even":
        c = torch.randint(0, E, (T, k), device="cuda", generator=g)
    elif kind == "skewed":
        c = (torch.rand((T, k), device="cuda", generator=g) ** 6 * E).long()
    elif kind == "one":
        c = torch.full((T, k), E - 1, device="cuda")
    elif kind == "outside":
        c = torch.randint(-2, E + 2, (T, k), device="cuda", generator=g)
    else:  # "none"
        c = torch.full((T, k), -1, device="cuda")
    return c.int()


def _want_order(chosen, E):
    key = chosen.long().reshape(-1).clone()
    key[(key < 0) | (key >= E)] = E
    by = torch.sort(key, stable=True).indices
    place = torch.empty_like(by)
    place[by] = torch.arange(len(by), device="cuda")
    place[key == E] = -1
    offsets = torch.zeros(E + 1, dtype=torch.long, device="cuda")
    offsets[1:] = torch.bincount(key, minlength=E + 1)[:E].cumsum(0)
    return offsets.int(), place.view(chosen.shape).int()


ORDERS = [(1, 1, 1), (1, 3, 7), (5, 2, 1024), (1024, 2, 8), (4096, 1, 3), (2048, 2, 128), (2049, 2, 127), (700, 6, 513), (33333, 3, 65), (30000, 8, 256),
          (200001, 8, 64)]


@pytest.mark.parametrize("T,k,E", ORDERS)
@pytest.mark.parametrize("kind", ["even", "skewed", "one", "outside", "none"])
def test_order(T, k, E, kind):
    chosen = _chosen(kind, T, k, E, T)
    d = S.Dispatch(E, k)
    offsets, places = d.order(chosen)
    want = _want_order(chosen, E)
    assert torch.equal(offsets, want[0]) and torch.equal(places, want[1])


def test_order_of_runs_longer_than_a_cta_takes_at_once():
    T, k, E = 700001, 2, 31  # over 304 CTAs' first runs of 4096 entries
    chosen = _chosen("skewed", T, k, E)
    got, want = S.Dispatch(E, k).order(chosen), _want_order(chosen, E)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def _check(T, k, E, d, tok, row, kind, lay=None):
    chosen = _chosen(kind, T, k, E, d)
    op = S.Dispatch(E, k, token_dtype=tok, row_dtype=row)
    order = op.order(chosen)
    p = order[1].long()
    there, at = p >= 0, p.clamp(min=0)
    kept = int(there.sum())
    lay = lay or (lambda t: t)
    # spread
    x = lay(_randn((T, d), tok, 2))
    rows = op.spread(x, order)
    want = torch.zeros((T * k, d), dtype=row, device="cuda")
    want[p[there]] = x[:, None, :].expand(T, k, d)[there].to(row)
    assert rows.dtype == row and torch.equal(rows, want)
    # combine, with weights and without
    y = _randn((T * k, d), row, 3)
    y[kept:] = float("nan")  # rows of no entry: not read
    w = torch.rand((T, k), device="cuda", generator=_gen(4)) - 0.3
    w[~there] = float("nan")
    mine = torch.where(there[..., None], y[at].double(), 0.0)
    for ws in (w, None):
        terms = mine * (1.0 if ws is None else torch.where(there, ws, 0.0).double()[..., None])
        got, ref = op.combine(y, ws, order), terms.sum(1)
        allow = k * 2.0 ** -24 * terms.abs().sum(1) + STEP[tok] * ref.abs() + 1e-40
        assert got.dtype == tok and got.shape == (T, d) and ((got.double() - ref).abs() <= allow).all()
    # its gradient
    dy = lay(_randn((T, d), tok, 5))
    drows, dw = op.combine_grad(dy, y, w, order)
    ref = torch.zeros((T * k, d), dtype=torch.float64, device="cuda")
    ref[p[there]] = (w.double()[..., None] * dy.double()[:, None, :])[there]
    assert drows.dtype == row and ((drows.double() - ref).abs() <= (2.0 ** -24 + STEP[row]) * ref.abs() * 1.001 + 1e-40).all()
    terms = mine * dy.double()[:, None, :]
    assert ((dw.double() - terms.sum(-1)).abs() <= (d / 32 + 13) * 2.0 ** -24 * terms.abs().sum(-1) + 1e-40).all()
    assert (dw[~there] == 0).all()


@pytest.mark.parametrize("T,k,E,d", [(1, 1, 1, 1), (1, 2, 8, 64), (7, 3, 5, 5), (1000, 2, 8, 64), (129, 4, 127, 1001), (300, 8, 256, 512), (64, 64, 100, 24),
                                     (50, 2, 128, 4096), (9, 5, 3, 8200), (5000, 1, 16, 9), (3000, 2, 4, 8), (2, 10, 16, 5197), (400, 2, 9, 1000)])
@pytest.mark.parametrize("tok,row", [(BF16, BF16), (F32, BF16), (BF16, F32), (F32, F32)])
def test_rows(T, k, E, d, tok, row):
    _check(T, k, E, d, tok, row, "even")
    _check(T, k, E, d, tok, row, "outside")


@pytest.mark.parametrize("kind", ["one", "none", "skewed"])
def test_rows_of_lopsided_choices(kind):
    _check(777, 3, 40, 72, BF16, BF16, kind)
    _check(777, 3, 40, 73, F32, BF16, kind)


def test_tokens_that_lie_apart_or_off_16_bytes():
    def apart(t):
        big = torch.full((t.shape[0], t.shape[1] + 24), float("nan"), dtype=t.dtype, device="cuda")
        big[:, 8:8 + t.shape[1]] = t
        return big[:, 8:8 + t.shape[1]]

    def off(t):
        big = torch.full((t.shape[0], t.shape[1] + 3), float("nan"), dtype=t.dtype, device="cuda")
        big[:, 1:1 + t.shape[1]] = t
        return big[:, 1:1 + t.shape[1]]
    for lay in (apart, off):
        for tok in (BF16, F32):
            _check(200, 2, 9, 256, tok, BF16, "outside", lay)


def test_no_tokens():
    d = S.Dispatch(7, 2)
    order = d.order(torch.empty((0, 2), dtype=torch.int32, device="cuda"))
    assert order[0].tolist() == [0] * 8 and order[1].shape == (0, 2)
    x = torch.empty((0, 16), dtype=BF16, device="cuda")
    assert d.spread(x, order).shape == (0, 16) and d.combine(x, None, order).shape == (0, 16)
    w = torch.empty((0, 2), device="cuda")
    assert [t.shape for t in d.combine_grad(x, x, w, order)] == [(0, 16), (0, 2)]


def test_places_that_no_order_made():
    """Places outside the rows are none; offsets that say more rows than there are clear none."""
    d = S.Dispatch(4, 2)
    places = torch.tensor([[0, 99], [-7, 1]], dtype=torch.int32, device="cuda")
    order = torch.full((5,), 1000, dtype=torch.int32, device="cuda"), places
    y = _randn((4, 8), BF16, 1)
    assert torch.equal(d.combine(y, None, order), y[:2])
    drows, dw = d.combine_grad(y[:2].contiguous(), y, torch.ones((2, 2), device="cuda"), order)
    assert torch.equal(drows[:2], y[:2]) and dw[0, 1] == 0 and dw[1, 0] == 0


def test_rows_past_2_31_elements():
    T, k, E, d = 300000, 2, 16, 4096  # 2.4e9 elements of rows
    op = S.Dispatch(E, k)
    order = op.order(_chosen("even", T, k, E))
    x = _randn((T, d), BF16, 1)
    rows = op.spread(x, order)
    for t in (0, 1, T // 2, T - 2, T - 1):
        for j in range(k):
            assert torch.equal(rows[int(order[1][t, j])], x[t])
    y = op.combine(rows, None, order)
    assert torch.equal(y, (2 * x.float()).to(BF16))


def test_gradients_by_differences():
    """spread and combine are linear in each argument, so that a difference along a direction is the result for the direction: what it
    makes of dy is what the gradient makes of the direction, within the roundings of 2^-24 that either takes of the terms' magnitudes (fewer than 100)."""
    T, k, E, d = 90, 3, 7, 50
    op = S.Dispatch(E, k, token_dtype=F32, row_dtype=F32)
    order = op.order(_chosen("outside", T, k, E))
    x, u, dy = (_randn((T, d), F32, s) for s in (1, 2, 3))
    rows, r, drows = (_randn((T * k, d), F32, s) for s in (4, 5, 6))
    w, v = (torch.rand((T, k), device="cuda", generator=_gen(s)) for s in (7, 8))
    kept = int(order[0][-1])
    for t in (r, drows):
        t[kept:] = 0
    dr, dw = op.combine_grad(dy, rows, w, order)
    dot = lambda a, b: (a.double() * b.double()).sum()  # noqa: E731
    size = lambda a, b: (a.double() * b.double()).abs().sum()  # noqa: E731
    there = order[1] >= 0
    for a, b in (((op.spread(u, order), drows), (u, op.combine(drows, None, order))), ((op.combine(r, w, order), dy), (dr, r)),
                 ((op.combine(rows, v, order), dy), (dw, torch.where(there, v, 0.0)))):
        assert abs(float(dot(*a) - dot(*b))) <= 100 * 2.0 ** -24 * float(size(*a) + size(*b)) * k
