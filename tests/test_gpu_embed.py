"""Embedding lookup and its gradient on the GPU against 64 bits.

A looked-up element is one product, rounded once: compared bit for bit. An element of the gradient is a sum
of n terms in fp32, in runs of at most 32 whose sums are then added: at most 32 + n / 32 + 2 roundings of 2^-24
of the terms' magnitudes, two more for scale and base, and for bf16 one of 2^-8 (half a spacing) of the result.
"""
import math

import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _ids(kind, T, V, seed, dtype):
    g = _gen(seed)
    if kind == "even":
        ids = torch.randint(0, V, (T,), device="cuda", generator=g)
    elif kind == "zipf":
        u = torch.rand(T, device="cuda", dtype=torch.float64, generator=g)
        ids = (torch.exp(u * math.log(V + 1.0)) - 1).long().clamp(0, V - 1)
    elif kind == "one":
        ids = torch.full((T,), V - 1, device="cuda")
    elif kind == "pad":  # ids outside the table among the others
        ids = torch.randint(-3, V + 3, (T,), device="cuda", generator=g)
    else:  # "none": padding alone
        ids = torch.full((T,), -1, device="cuda")
    return ids.to(dtype)


def _randn(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, device="cuda", generator=_gen(seed)) * scale).to(dtype)


def _check_lookup(V, d, ids, tt, at, scale):
    table = _randn((V, d), tt, 1)
    y = S.Embedding(V, d, tt, at, scale=scale).lookup(table, ids)
    ok = (ids >= 0) & (ids < V)
    want = (table[ids.clamp(0, V - 1).long()].float() * scale).masked_fill(~ok[..., None], 0.0).to(at)
    assert y.shape == (*ids.shape, d) and torch.equal(y, want)


def _grad64(V, d, ids, dy, scale, base):
    ok = (ids >= 0) & (ids < V)
    at, v = ids[ok].long(), dy.reshape(-1, d)[ok].double()
    n = torch.bincount(at, minlength=V).double()[:, None]
    s = torch.zeros((V, d), dtype=torch.float64, device="cuda").index_add_(0, at, v)
    a = torch.zeros((V, d), dtype=torch.float64, device="cuda").index_add_(0, at, v.abs())
    b = 0.0 if base is None else base.double()
    return s * scale + b, (a * abs(scale)) * (32 + n / 32 + 4) + (0.0 if base is None else 2 * b.abs())


def _check_grad(V, d, ids, tt, at, scale=1.0, with_base=False, dy=None):
    dy = _randn((ids.numel(), d), at, 2) if dy is None else dy
    base = _randn((V, d), tt, 3) if with_base else None
    e = S.Embedding(V, d, tt, at, scale=scale)
    want, terms = _grad64(V, d, ids, dy, scale, base)
    allow = 2.0 ** -24 * terms + (2.0 ** -8 if tt == BF16 else 2.0 ** -24) * want.abs() + 1e-40
    keep = None if base is None else base.clone()
    got = e.grad(ids, dy, base=base)
    assert got.dtype == tt and ((got.double() - want).abs() <= allow).all()
    assert torch.equal(got, e.grad(ids, dy, base=base))          # the same bits again
    if with_base:
        assert torch.equal(base, keep)
        e.grad(ids, dy, base=base, out=base)                     # in place
        assert torch.equal(base, got)
    return got


@pytest.mark.parametrize("V,d,T", [(1, 1, 1), (3, 5, 7), (512, 64, 1024), (300, 8, 33), (1000, 255, 500), (777, 257, 64), (50257, 768, 300), (257, 1000, 129),
                                   (100, 4096, 70), (64, 8200, 9), (33, 31, 5000)])
@pytest.mark.parametrize("tt,at", [(BF16, BF16), (BF16, F32), (F32, BF16), (F32, F32)])
def test_lookup(V, d, T, tt, at):
    for kind, dt, scale in (("even", torch.int64, 1.0), ("pad", torch.int32, math.sqrt(d))):
        _check_lookup(V, d, _ids(kind, T, V, T, dt), tt, at, scale)
    _check_lookup(V, d, _ids("even", 6, V, 1, torch.int64).view(2, 3), tt, at, 0.5)


@pytest.mark.parametrize("V,d,T", [(1, 1, 1), (3, 5, 7), (512, 64, 1024), (300, 8, 33), (1000, 255, 500), (777, 257, 64), (50257, 768, 300), (257, 1000, 1290),
                                   (100, 4096, 700), (64, 8200, 9), (33, 31, 5000), (2048, 16, 40000), (200000, 24, 3001)])
@pytest.mark.parametrize("kind", ["even", "zipf", "one", "pad", "none"])
def test_gradient(V, d, T, kind):
    for k, (tt, at) in enumerate(((BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16))):
        ids = _ids(kind, T, V, T, (torch.int64, torch.int32)[k % 2])
        _check_grad(V, d, ids, tt, at, (1.0, 0.5, math.sqrt(d), -2.0)[k], with_base=k % 2 == 1)
        _check_grad(V, d, ids, tt, at, (1.0, 0.5, math.sqrt(d), -2.0)[k], with_base=k % 2 == 0)


@pytest.mark.parametrize("n", [1, 31, 32, 33, 63, 64, 65, 96, 1000])
@pytest.mark.parametrize("lead", [0, 1, 31, 32])
def test_runs_around_the_chunks(n, lead):
    """Runs of n equal ids after `lead` other tokens, and more runs behind them: cut, uncut, whole chunks."""
    ids = torch.cat([torch.arange(lead), torch.full((n,), 40), torch.full((33,), 41), torch.full((70,), 42), torch.tensor([43, 44, 44])])
    ids = ids[torch.randperm(len(ids), generator=torch.Generator().manual_seed(n))].cuda()
    _check_grad(50, 72, ids, F32, F32, with_base=True)
    _check_grad(50, 300, ids, BF16, BF16)


def test_no_tokens():
    e = S.Embedding(10, 16)
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    assert e.lookup(torch.ones((10, 16), dtype=BF16, device="cuda"), ids).shape == (0, 16)
    dy = torch.empty((0, 16), dtype=BF16, device="cuda")
    assert (e.grad(ids, dy) == 0).all()
    base = _randn((10, 16), BF16, 1)
    assert torch.equal(e.grad(ids, dy, base=base), base)


def test_order_of_terms_is_the_tokens():
    """1e8 + 1 - 1e8 differs with the order: the tokens' own, wherever they stand."""
    big = 1e8
    for gap in (1, 40, 3000):
        T = 2 * gap + 1
        ids = torch.arange(5, 5 + T, device="cuda")
        ids[0] = ids[gap] = ids[2 * gap] = 2
        dy = torch.zeros((T, 8), device="cuda")
        for vals, want in (((big, 1.0, -big), 0.0), ((big, -big, 1.0), 1.0)):
            for at, v in zip((0, gap, 2 * gap), vals):
                dy[at] = v
            got = S.Embedding(T + 10, 8, F32, F32).grad(ids, dy)
            assert (got[2] == want).all()


def test_strided_and_unaligned_rows():
    ids = _ids("zipf", 500, 90, 4, torch.int64)
    for dt in (BF16, F32):
        wide = _randn((500, 96), dt, 5)
        for at in (0, 1, 4, 8):
            dy = wide[:, at: at + 64]
            e = S.Embedding(90, 64, dt, dt)
            assert torch.equal(e.grad(ids, dy), e.grad(ids, dy.contiguous()))
        flat = _randn(90 * 64 + 3, dt, 6)
        table = flat[3:].view(90, 64)
        assert torch.equal(S.Embedding(90, 64, dt, dt).lookup(table, ids), table[ids])
    # rows of `out` apart: what lies between them stays
    out = torch.full((500, 80), 7.0, dtype=BF16, device="cuda")
    table = _randn((90, 64), BF16, 7)
    c = S.EmbedConfig(90, 64, 1.0, S.EMBED_IDS_64)
    S.skew_embed_lookup(c, table.data_ptr(), ids.data_ptr(), 500, out.data_ptr(), 80, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(out[:, :64], table[ids]) and (out[:, 64:] == 7).all()


def test_nan_and_inf_stay_in_their_rows():
    ids = torch.tensor([3, 3, 5, -1, 9], device="cuda")
    dy = torch.ones((5, 40), device="cuda")
    dy[0, 7], dy[2, 8], dy[3] = math.nan, math.inf, math.nan
    got = S.Embedding(10, 40, F32, F32).grad(ids, dy)
    assert got.isnan().sum() == 1 and got[3, 7].isnan() and got.isinf().sum() == 1 and got[5, 8] == math.inf
    table = torch.full((10, 40), math.nan, device="cuda")
    assert (S.Embedding(10, 40, F32, F32).lookup(table, torch.tensor([-1, 10], device="cuda")) == 0).all()


def test_a_table_past_2_31_elements():
    V, d = (1 << 20) + 3, 2056
    table = torch.zeros((V, d), dtype=BF16, device="cuda")
    rows = torch.tensor([0, 1 << 19, (1 << 20) + 2, (1 << 20) - 1, 1 << 19], device="cuda")
    table[rows] = _randn((5, d), BF16, 8)
    e = S.Embedding(V, d)
    assert torch.equal(e.lookup(table, rows), table[rows])
    dy = _randn((5, d), BF16, 9)
    got = e.grad(rows, dy)
    assert torch.equal(got[rows[[0, 2, 3]]], dy[[0, 2, 3]])
    assert torch.equal(got[1 << 19], (dy[1].float() + dy[4].float()).to(BF16))
    got[rows] = 0
    assert int(torch.count_nonzero(got)) == 0


def test_gradient_against_differences():
    """The lookup is linear: <dW, P> is the loss's difference along P, exactly."""
    V, d, T = 200, 24, 600
    ids = _ids("zipf", T, V, 10, torch.int64)
    W, P, dy = _randn((V, d), F32, 11), _randn((V, d), F32, 12), _randn((T, d), F32, 13)
    e = S.Embedding(V, d, F32, F32, scale=3.0)
    dW = e.grad(ids, dy)
    loss = lambda w: (e.lookup(w, ids).double() * dy.double()).sum()  # noqa: E731
    diff = loss(W + P) - loss(W - P)
    along = 2 * (dW.double() * P.double()).sum()
    size = 2 * (e.lookup(P.abs(), ids).double() * dy.double().abs()).sum() + (e.lookup(W.abs(), ids).double() * dy.double().abs()).sum()
    assert abs(float(diff - along)) <= 60 * 2.0 ** -24 * float(size)


def test_on_a_side_stream_and_captured():
    V, d, T = 1000, 128, 4000
    ids, table, dy = _ids("zipf", T, V, 14, torch.int32), _randn((V, d), BF16, 15), _randn((T, d), BF16, 16)
    e = S.Embedding(V, d)
    want = [e.lookup(table, ids), e.grad(ids, dy)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = [e.lookup(table, ids), e.grad(ids, dy)]
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
