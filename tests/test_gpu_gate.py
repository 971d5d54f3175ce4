"""Routing and its gradient on the GPU against 64 bits.

Without a bias experts are chosen by the logits themselves, so choices are compared exactly, ties too. With
one they are chosen by fp32 scores: tokens whose 64-bit choice hangs on less than MARGIN (a score, at most 1, is
within about 10 roundings of 2^-24) are left out of the inputs.

Tolerances (2^-24 relative to a rounding). An exponential of a logit difference of at most 40 carries 40
roundings of its argument and 4 of its own, a sum of n terms n at most, and a few products and divisions
follow: REL with n <= 40 (lanes add 16 terms, then 5 times two; top_k is at most 32). Gradients subtract two such
terms: the same, relative to the sum of the terms' magnitudes, and bf16 ones round by half a spacing, 2^-8, besides.
"""
import math

import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu

REL = 100 * 2.0 ** -24
MARGIN = 1e-5
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


def _logits(T, E, seed, dtype=F32, scale=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn((T, E), device="cuda", generator=g) * scale).to(dtype)


def _best(v, k):
    """Values and indices of the k largest, the lowest index first among equals."""
    v, i = torch.sort(v, dim=-1, descending=True, stable=True)
    return v[..., :k], i[..., :k]


def reference(x, bias, E, k, score="softmax", renorm=True, groups=1, top_groups=1, group_top=1, scale=1.0):
    """(chosen, weights, counts, margin): margin is what each token's choices hang on."""
    x = x.double()
    T = x.shape[0]
    nan = x.isnan().any(1)
    out = x.isnan() | (x == -math.inf)
    xs = x.masked_fill(out, -math.inf)
    if score == "softmax":
        m = xs.amax(1, keepdim=True)
        e = torch.exp(xs - m.masked_fill(m == -math.inf, 0.0))
        s = e / e.sum(1, keepdim=True).clamp(min=1e-300)
    else:
        s = 1 / (1 + torch.exp(-xs))
    c = xs if bias is None else s + bias.double()
    shown = s if bias is None else c
    out = out | c.isnan() | (c == -math.inf)
    c = c.masked_fill(out, -math.inf)
    margin = torch.full((T,), math.inf, dtype=torch.float64, device=x.device)

    def gap(v, n):  # between what is taken and what is not
        if n >= v.shape[1]:
            return margin
        d = torch.sort(v, dim=1, descending=True).values
        g = d[:, n - 1] - d[:, n]
        return torch.minimum(margin, torch.where(g.isnan(), math.inf, g))

    if groups > 1:
        v = (c if group_top == 1 else shown.masked_fill(out, -math.inf)).view(T, groups, -1)
        b = _best(v, group_top)[0]
        v = b[..., 0] if group_top == 1 else b[..., 0] + torch.where(b[..., -1] == -math.inf, 0.0, b[..., -1]) * (v.shape[2] > 1)
        if bias is not None or group_top == 2:
            margin = gap(v, top_groups)
        kept = torch.zeros_like(v, dtype=torch.bool).scatter_(1, _best(v, top_groups)[1], True)
        c = c.masked_fill(~kept.repeat_interleave(E // groups, dim=1), -math.inf)
    if bias is not None:
        d = torch.sort(c, dim=1, descending=True).values[:, :k + 1]
        g = (d[:, :-1] - d[:, 1:]).amin(1) if d.shape[1] > 1 else margin
        margin = torch.minimum(margin, torch.where(g.isnan(), math.inf, g))
    v, chosen = _best(c, k)
    none = v == -math.inf
    w = s.gather(1, chosen).masked_fill(none, 0.0)
    if renorm:
        total = w.sum(1, keepdim=True)
        w = torch.where(total == 0, 0.0, w / total)
    w = (w * scale).masked_fill(nan[:, None], math.nan)
    chosen = chosen.masked_fill(none, -1)
    counts = torch.bincount(chosen[chosen >= 0], minlength=E)
    return chosen, w, counts, margin


def _check(x, bias, E, k, **kw):
    chosen, w, counts, margin = reference(x, bias, E, k, **kw)
    if not bool((margin > MARGIN).all()):  # inputs, not results: only tokens whose choice 64 bits settles
        x = x[margin > MARGIN]
        chosen, w, counts, margin = reference(x, bias, E, k, **kw)
    r = S.Router(E, k, **kw)
    for _ in range(2):  # the second call finds the workspace as the first left it
        got, gw, gc = r.route(x, bias=bias)
        assert torch.equal(got.long(), chosen)
        assert torch.equal(gc.long(), counts)
        assert torch.equal(gw.isnan(), w.isnan())
        assert ((gw - w).abs() <= REL * w.abs() + 1e-37)[~w.isnan()].all()
    return r, x


@pytest.mark.parametrize("E,k", [(1, 1), (2, 1), (3, 3), (8, 2), (16, 16), (17, 4), (32, 32), (33, 5), (64, 6), (100, 32), (127, 4),
                                 (128, 2), (129, 8), (200, 8), (256, 8), (257, 3), (500, 31), (512, 10)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_experts_and_scores(E, k, score, dtype):
    for T in (1, 31, 700):
        x = _logits(T, E, E * 1000 + T, dtype)
        for renorm in (True, False):
            _check(x, None, E, k, score=score, renorm=renorm, scale=2.5)
    bias = 0.2 * torch.randn(E, device="cuda", generator=torch.Generator(device="cuda").manual_seed(E))
    _check(_logits(700, E, E, F32), bias, E, k, score=score)


@pytest.mark.parametrize("E,groups,top_groups,k", [(8, 4, 2, 3), (16, 4, 2, 8), (64, 8, 3, 6), (60, 4, 2, 7), (96, 3, 1, 8), (128, 32, 8, 8), (128, 8, 4, 2),
                                                   (256, 8, 4, 8), (256, 16, 16, 32), (240, 16, 5, 9), (512, 8, 4, 16), (512, 2, 1, 8), (90, 30, 7, 12), (5, 5, 2, 2)])
@pytest.mark.parametrize("group_top", [1, 2])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_groups(E, groups, top_groups, k, group_top, score):
    x = _logits(900, E, E + groups, F32, 1.0)
    bias = 0.1 * torch.randn(E, device="cuda", generator=torch.Generator(device="cuda").manual_seed(groups))
    for b in (None, bias):
        _check(x, b, E, k, score=score, groups=groups, top_groups=top_groups, group_top=group_top)
    x[::7, : E // 2] = -math.inf  # groups with nothing, or one expert, left
    x[::5, 1::2] = -math.inf
    x[::35] = -math.inf
    for b in (None, bias):
        _check(x, b, E, k, score=score, groups=groups, top_groups=top_groups, group_top=group_top)


@pytest.mark.parametrize("E,k", [(8, 4), (40, 6), (128, 8), (256, 8), (512, 32)])
def test_ties_go_to_the_lowest_index(E, k):
    for dtype in (F32, BF16):
        x = _logits(600, E, E, dtype).round()  # few distinct values, -0 among them
        _check(x, None, E, k)
        _check(torch.zeros_like(x), None, E, k)
        _check(x, None, E, min(k, E // 4), groups=4, top_groups=1, group_top=1)
    for score in ("softmax", "sigmoid"):  # equal scores, equal bias: 64 bits sees the same ties
        r = S.Router(E, k, score=score)
        chosen, w, _ = r.route(torch.zeros((50, E), device="cuda"), bias=torch.full((E,), 0.25, device="cuda"))
        assert torch.equal(chosen, torch.arange(k, device="cuda", dtype=torch.int32).expand(50, k))
        assert ((w - 1 / k).abs() <= REL / k).all()


@pytest.mark.parametrize("E,k", [(8, 2), (127, 4), (256, 8)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
def test_masks_nan_and_extremes(E, k, score, renorm):
    x = _logits(400, E, E, F32)
    x[0] = -math.inf                       # nothing to choose
    x[1, 1:] = -math.inf                   # fewer than k
    x[2, : E // 2] = -math.inf
    x[3, 0] = math.nan                     # poisons its token's weights, and no other
    x[4] = math.nan
    x[5] = -1e30
    x[6] = torch.finfo(F32).min            # a mask by the type's lowest value
    x[6, 1] = 0.0
    x[7] = 1e30
    x[8] = torch.linspace(-300, 300, E, device="cuda")
    x[9] = torch.linspace(-3e-39, 3e-39, E, device="cuda")
    if score == "softmax" and not renorm:
        x[8] = torch.linspace(-30, 30, E, device="cuda")
    if score == "sigmoid":
        x[8] = torch.linspace(-30, 30, E, device="cuda")
        x[5] = -30.0
        x[6] = -30.0
    _check(x, None, E, k, score=score, renorm=renorm)
    bias = torch.zeros(E, device="cuda")
    bias[0], bias[1] = -math.inf, math.nan  # experts that no token may take
    r = S.Router(E, k, score=score, renorm=renorm)
    chosen, w, counts = r.route(_logits(300, E, 1), bias=bias)
    assert int(counts[0]) == 0 and int(counts[1]) == 0 and (chosen >= 2).all() and int(counts.sum()) == 300 * k
    assert not w.isnan().any()


def test_sigmoid_scores_that_all_underflow():
    x = torch.full((3, 16), -200.0, device="cuda")
    chosen, w, _ = S.Router(16, 4, score="sigmoid").route(x)
    assert torch.equal(chosen, torch.arange(4, device="cuda", dtype=torch.int32).expand(3, 4)) and (w == 0).all()
    dx = S.Router(16, 4, score="sigmoid").grad(x, chosen, torch.ones((3, 4), device="cuda"))
    assert (dx == 0).all()


@pytest.mark.parametrize("E,k", [(8, 2), (128, 2), (256, 8)])
def test_many_tokens_and_none(E, k):
    _check(_logits(70001, E, 5, BF16), None, E, k)
    r = S.Router(E, k)
    chosen, w, counts = r.route(torch.empty((0, E), device="cuda"))
    assert chosen.shape == (0, k) and w.shape == (0, k) and (counts == 0).all()
    assert r.grad(torch.empty((0, E), device="cuda"), chosen, w).shape == (0, E)


@pytest.mark.parametrize("E", [8, 12, 128, 130, 256])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strided_and_unaligned_rows(E, dtype):
    wide = _logits(333, E + 9, E, dtype)
    for at in (0, 1, 3, 8):
        x = wide[:, at: at + E]
        r, _ = _check(x, None, E, 2)
        chosen, w, _ = r.route(x)
        dw = torch.randn((333, 2), device="cuda")
        assert torch.equal(r.grad(x, chosen, dw), r.grad(x.contiguous(), chosen, dw))


def _loss(x, chosen, dw, score, renorm, scale):
    ok = chosen >= 0
    s = torch.softmax(x, 1) if score == "softmax" else torch.sigmoid(x)
    w = s.gather(1, chosen.clamp(min=0)).masked_fill(~ok, 0.0)
    if renorm:
        w = w / w.sum(1, keepdim=True)
    return (w * dw).sum(1) * scale


@pytest.mark.parametrize("E,k", [(2, 1), (8, 2), (8, 8), (33, 5), (127, 4), (128, 2), (200, 32), (256, 8), (512, 10)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradient(E, k, score, renorm, dtype):
    for T in (1, 5, 1003):
        x = _logits(T, E, T + E, dtype)
        r = S.Router(E, k, score=score, renorm=renorm, scale=1.5)
        chosen, _, _ = r.route(x)
        chosen[::3, 0] = -1 if k > 1 else chosen[::3, 0]   # a slot without an expert
        dw = torch.randn((T, k), device="cuda", generator=torch.Generator(device="cuda").manual_seed(T))
        keep = (x.clone(), chosen.clone(), dw.clone())
        dx = r.grad(x, chosen, dw)
        assert dx.dtype == dtype and dx.shape == x.shape
        assert torch.equal(keep[0], x) and torch.equal(keep[1], chosen) and torch.equal(keep[2], dw)
        # the formula
        x64, at, ok = x.double(), chosen.long().clamp(min=0), chosen >= 0
        s = torch.softmax(x64, 1) if score == "softmax" else torch.sigmoid(x64)
        p = s.gather(1, at).masked_fill(~ok, 0.0)
        g = dw.double().masked_fill(~ok, 0.0) * 1.5
        if renorm:
            q = p / p.sum(1, keepdim=True)
            rest = 1.0 if score == "softmax" else 1 - s.gather(1, at)
            v = q * (g - (g * q).sum(1, keepdim=True)) * rest
            size = q * (g.abs() + (g * q).abs().sum(1, keepdim=True))
            want = torch.zeros_like(x64).scatter_add_(1, at, v.masked_fill(~ok, 0.0))
            size = torch.zeros_like(x64).scatter_add_(1, at, size.masked_fill(~ok, 0.0))
        elif score == "sigmoid":
            want = torch.zeros_like(x64).scatter_add_(1, at, g * p * (1 - p))
            size = want.abs()
        else:
            ds = torch.zeros_like(x64).scatter_add_(1, at, g)
            want = s * (ds - (ds * s).sum(1, keepdim=True))
            size = s * (ds.abs() + (ds * s).abs().sum(1, keepdim=True))
        off = (dx.double() - want).abs()
        assert (off <= REL * size + (2.0 ** -8 * want.abs() if dtype == BF16 else 0) + 1e-38).all()
        # differences, in 64 bits, along a random direction
        v = torch.randn(x64.shape, device="cuda", dtype=torch.float64, generator=torch.Generator(device="cuda").manual_seed(1))
        h = 1e-5
        d = (_loss(x64 + h * v, chosen.long(), dw.double(), score, renorm, 1.5) -
             _loss(x64 - h * v, chosen.long(), dw.double(), score, renorm, 1.5)) / (2 * h)
        along = (dx.double() * v).sum(1)
        allow = ((REL * size + (2.0 ** -8 * want.abs() if dtype == BF16 else 0)) * v.abs()).sum(1) + 1e-6
        if not (renorm and k == 1):  # then a slot without an expert leaves 0 / 0 in the plain form
            assert ((along - d).abs() <= allow).all()


def test_gradient_of_masked_rows():
    x = _logits(6, 128, 3)
    x[0] = -math.inf
    x[1, 2:] = -math.inf
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            r = S.Router(128, 4, score=score, renorm=renorm)
            chosen, _, _ = r.route(x)
            dx = r.grad(x, chosen, torch.ones((6, 4), device="cuda"))
            assert dx.isfinite().all() and (dx[0] == 0).all() and (dx[1, 2:] == 0).all()
    chosen = torch.tensor([[1000, -7, 128, 5]], dtype=torch.int32, device="cuda").expand(6, 4).contiguous()
    for score in ("softmax", "sigmoid"):     # entries that name no expert have no gradient
        dx = S.Router(128, 4, score=score).grad(x[2:3], chosen[2:3], torch.ones((1, 4), device="cuda"))
        assert int((dx != 0).sum()) == (0 if score == "softmax" else 0) and dx.isfinite().all()


def test_on_a_side_stream_and_captured():
    x = _logits(5000, 128, 9)
    r = S.Router(128, 2)
    want = [t.clone() for t in r.route(x)]
    dw = torch.randn((5000, 2), device="cuda")
    want.append(r.grad(x, want[0], dw))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = list(r.route(x))
        got.append(r.grad(x, got[0], dw))
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("E,k,groups,top_groups", [(1, 1, 1, 1), (2, 2, 1, 1), (6, 1, 2, 1), (8, 2, 1, 1), (8, 8, 1, 1), (15, 4, 3, 2), (24, 3, 8, 4), (33, 20, 1, 1), (47, 4, 1, 1),
                                                   (48, 16, 16, 6), (64, 6, 1, 1), (64, 32, 2, 2), (64, 8, 32, 5)])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_few_experts_and_many_tokens(E, k, groups, top_groups, score):
    """Enough tokens for a thread to each: every score, bias, group rule, masks, ties and strides."""
    T = 601 * E + 77
    wide = _logits(T, E + 3, E + k, F32, 1.5)
    bias = 0.2 * torch.randn(E, device="cuda", generator=_gen_of(E))
    for x in (wide[:, :E].contiguous(), wide[:, 1: E + 1], wide[:, :E].to(BF16)):
        for group_top in (1, 2) if groups > 1 else (1,):
            kw = dict(score=score, groups=groups, top_groups=top_groups, group_top=group_top, scale=1.5)
            _check(x, None, E, k, renorm=False, **kw)
            _check(x, bias, E, k, renorm=True, **kw)
    x = wide[:, :E].clone()
    x[::7, E // 2:] = -math.inf
    x[::5, ::2] = -math.inf
    x[::11] = -math.inf
    for b in (bias, None):
        if b is None or score == "sigmoid":  # (a softmax with a NaN logit is NaN throughout: then its scores choose nothing)
            x[3, 0], x[40] = math.nan, math.nan
        _check(x, b, E, k, score=score, groups=groups, top_groups=top_groups, group_top=1)
        _check(x, b, E, k, score=score, renorm=False, groups=groups, top_groups=top_groups, group_top=2 if groups > 1 else 1)
    _check(x.round(), None, E, k, score=score, groups=groups, top_groups=top_groups, group_top=1)  # ties
    r = S.Router(E, k, score=score)
    chosen, w, counts = r.route(torch.zeros((T, E), device="cuda"))
    assert torch.equal(chosen, torch.arange(k, device="cuda", dtype=torch.int32).expand(T, k)) and int(counts.sum()) == T * k


def _gen_of(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


@pytest.mark.parametrize("E,groups,top_groups,k", [(65, 5, 2, 9), (96, 8, 4, 5), (352, 8, 4, 6), (396, 4, 2, 15), (480, 32, 9, 12), (510, 3, 2, 8), (300, 12, 12, 32), (511, 7, 3, 4)])
@pytest.mark.parametrize("group_top", [1, 2])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_groups_of_any_size(E, groups, top_groups, k, group_top, score):
    """Groups that fill their lanes unevenly, and some that only the general way serves."""
    x = _logits(800, E, E, F32, 1.0)
    x[::9, : E // 3] = -math.inf
    bias = 0.1 * torch.randn(E, device="cuda", generator=_gen_of(groups))
    for b in (None, bias):
        for renorm in (True, False):
            _check(x, b, E, k, score=score, renorm=renorm, groups=groups, top_groups=top_groups, group_top=group_top)


@pytest.mark.parametrize("E,k", [(96, 4), (128, 8), (256, 8), (500, 16)])
def test_near_ties_are_settled_by_fp32_scores(E, k):
    """Scores that differ by less than quick ones may be off: what is chosen is the largest of the fp32 scores plus bias,
    the lowest index first, as a plain fp32 evaluation orders them."""
    x = torch.zeros((400, E), device="cuda") + _logits(1, E, 1, F32, 1e-6) + _logits(400, 1, 2, F32, 1.0)
    bias = 1e-7 * torch.randn(E, device="cuda", generator=_gen_of(E))
    s = 1.0 / (1.0 + torch.exp(-x)) + bias
    chosen, w, _ = S.Router(E, k, score="sigmoid").route(x, bias=bias)
    assert torch.equal(chosen.long(), _best(s, k)[1])
    if E % 4 == 0:
        by = s.view(400, 4, -1)
        by = _best(by, 2)[0]
        kept = torch.zeros((400, 4), dtype=torch.bool, device="cuda").scatter_(1, _best(by[..., 0] + by[..., 1], 2)[1], True)
        want = _best(s.masked_fill(~kept.repeat_interleave(E // 4, dim=1), -math.inf), k)[1]
        chosen, w, _ = S.Router(E, k, score="sigmoid", groups=4, top_groups=2, group_top=2).route(x, bias=bias)
        assert torch.equal(chosen.long(), want)
