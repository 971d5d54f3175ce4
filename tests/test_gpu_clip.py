"""Global gradient norm and clipping on the GPU against 64 bits.

Tolerances. A thread adds at most 64 squares in fp32 to each of two sums before joining them by
compensated or fp64 sums, so the sum of squares is within 67 * 2^-24 and the norm, rounded once, within
half of that and 2^-24: NORM. The factor takes three more roundings: GAMMA. A clipped element is one product of
the factor that was used and one rounding, so it is compared bit for bit.
"""
import math

import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu

NORM = 35 * 2.0 ** -24
GAMMA = NORM + 3 * 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


def _rand(n, dtype, seed, scale=1e-3, skew=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(n + skew, dtype=torch.float32, device="cuda").normal_(0, scale, generator=g).to(dtype)[skew:]


def _norm64(ts):
    return math.sqrt(sum(float(t.double().square().sum()) for t in ts))


def _check(ts, outs=None, max_norm=1.0):
    want = _norm64(ts)
    copies = [t.clone() for t in ts]
    c = S.GradClip(ts, out=outs)
    norm, gamma = (float(x) for x in c.norm(max_norm))
    assert abs(norm - want) <= NORM * want
    g64 = min(1.0, max_norm / (want + 1e-6))
    assert abs(gamma - g64) <= GAMMA * g64
    for t, u in zip(ts, copies):
        assert torch.equal(t, u)                              # norm reads only
    again = c.clip(max_norm)
    assert [float(x) for x in again] == [norm, gamma]         # the same bits from the same gradients
    for u, o in zip(copies, c.out):
        assert torch.equal(o, (u.float() * gamma).to(o.dtype))
    if outs is not None:
        for t, u in zip(ts, copies):
            assert torch.equal(t, u)
    return norm, gamma


@pytest.mark.parametrize("n", [1, 7, 8, 9, 255, 2048, 2049, 8191, 8192, 8193, 100003, 1 << 21])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_one_tensor(n, dtype):
    _check([_rand(n, dtype, n, 1.0)])
    _check([_rand(n, dtype, n + 1, 1.0)], [torch.empty(n, dtype=dtype, device="cuda")])


@pytest.mark.parametrize("skew,out_skew", [(1, 1), (3, 3), (1, 0), (0, 5), (7, 2), (4, 4)])
@pytest.mark.parametrize("types", [(BF16, BF16), (F32, F32), (F32, BF16)])
def test_off_alignment(skew, out_skew, types):
    """Tensors that start off a 16-byte boundary, alike or not on both sides; what lies around `out` stays."""
    for n in (1, 5, 31, 9001, 70003):
        buf = torch.full((n + 16,), 7.0, dtype=types[1], device="cuda")
        _check([_rand(n, types[0], n, 1.0, skew)], [buf[out_skew: out_skew + n]])
        assert (buf[:out_skew] == 7).all() and (buf[out_skew + n:] == 7).all()


def test_many_tensors_of_both_types():
    ts = [_rand(1 + (k * 7919) % 30011, (BF16, F32)[k % 3 == 0], k, 1e-2, k % 4) for k in range(600)]
    _check(ts, [torch.empty_like(t) for t in ts])
    _check(ts)


def test_a_set_of_large_tiles():
    """Over 39 MB of gradient the tiles are larger; an fp32 accumulator beside bf16 gradients."""
    ts = [_rand((1 << 24) + 13, BF16, 1), _rand((1 << 22) + 5, F32, 2, 1e-3, 1)]
    _check(ts, [torch.empty_like(ts[0]), torch.empty(ts[1].numel(), dtype=BF16, device="cuda")])


def test_no_tensors_and_empty_tensors():
    c = S.GradClip([])
    assert c.clip(1.0).tolist() == [0.0, 1.0]
    ts = [torch.empty(0, device="cuda", dtype=BF16), _rand(10, BF16, 3, 1.0), torch.empty((4, 0), device="cuda")]
    _check(ts)
    assert S.GradClip(ts[:1]).norm(2.0).tolist() == [0.0, 1.0]


def test_zero_gradients_and_a_factor_of_one():
    z = torch.zeros(70000, dtype=BF16, device="cuda")
    assert S.GradClip([z]).clip(1.0).tolist() == [0.0, 1.0]
    t = _rand(70000, BF16, 4, 1e-4)
    o = torch.empty_like(t)
    assert _check([t], [o])[1] == 1.0 and torch.equal(o, t)
    assert S.GradClip([t]).norm(0.0)[1] == 0.0


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-22, 1e-15, 1e15, 1e19, 1e30])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_squares_outside_fp32(scale, dtype):
    """Norms of gradients whose squares fp32 does not hold, and of ordinary ones beside them. (Below 1e-37 the
    inputs are subnormal, which changes nothing: 64 bits see the same inputs.)"""
    big = _rand(50001, dtype, 5, scale)
    want = _norm64([big])
    for ts in ([big], [big, _rand(3000, dtype, 6)], [torch.cat([big, _rand(999, dtype, 7)])]):
        want = _norm64(ts)
        got = float(S.GradClip(ts).norm(1.0)[0])
        assert abs(got - want) <= NORM * want + 2.0 ** -149


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_nan_and_inf(dtype):
    for bad, norm, gamma in ((math.nan, math.isnan, math.isnan), (math.inf, math.isinf, lambda x: x == 0),
                             (-math.inf, math.isinf, lambda x: x == 0)):
        for at in (0, 777, 49999):
            t = _rand(50000, dtype, 8)
            t[at] = bad
            r = S.GradClip([t]).norm(1.0).tolist()
            assert norm(r[0]) and gamma(r[1])
    t = _rand(100, dtype, 9)
    t[3] = math.inf
    out = torch.empty_like(t)
    S.GradClip([t], out=[out]).clip(1.0)
    assert torch.isnan(out[3]) and (out.isnan().sum() == 1) and out.nan_to_num().abs().max() == 0
    # a finite gradient whose norm exceeds fp32
    t = torch.full((1000,), 3e38, device="cuda").to(dtype)
    r = S.GradClip([t]).norm(1.0).tolist()
    assert math.isinf(r[0]) and r[1] == 0


def test_past_2_31_elements():
    n = (1 << 31) + 24
    t = torch.zeros(n, dtype=BF16, device="cuda")
    for k, at in enumerate((0, (1 << 31) - 1, 1 << 31, n - 1)):
        t[at] = 3.0 + k
    c = S.GradClip([t])
    r = c.clip(0.5)
    want = math.sqrt(9 + 16 + 25 + 36)
    assert abs(float(r[0]) - want) <= NORM * want
    assert float(t[n - 1]) == float((torch.tensor(6.0) * r[1].cpu()).to(BF16))
    assert int(torch.count_nonzero(t)) == 4


def test_on_a_side_stream_and_captured():
    ts = [_rand(30000, BF16, 10, 1.0), _rand(5000, F32, 11, 1.0)]
    outs = [torch.empty_like(t) for t in ts]
    c = S.GradClip(ts, out=outs)
    want = c.clip(1.0).clone()
    want_out = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.result.zero_()
        got = c.clip(1.0)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.clip(1.0)
    for t in ts:
        t.mul_(2.0)
    for _ in range(3):
        for o in outs:
            o.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert float(c.result[0]) == 2 * float(want[0])
    for t, o, w in zip(ts, outs, want_out):
        assert torch.equal(o, (t.float() * c.gamma).to(t.dtype))


def test_factor_feeds_the_step():
    """The gamma view is the step's grad_scale: the same step as with the factor from elsewhere."""
    def make():
        ps = [(_rand((300 * 64), BF16, 12, 0.02).view(300, 64), _rand(300 * 64, BF16, 13, 1.0).view(300, 64), 0),
              (_rand(500, F32, 14, 0.02), _rand(500, F32, 15, 1.0), 0)]
        return ps, S.SkewAdam(ps, S.hparams())
    pa, a = make()
    pb, b = make()
    c = S.GradClip([p[1] for p in pa])
    c.norm(1.0)
    a.step(1, 1e-3, 5, grad_scale=c.gamma)
    b.step(1, 1e-3, 5, grad_scale=c.gamma.clone())
    for (w, _, _), (v, _, _) in zip(pa, pb):
        assert torch.equal(w, v)
    assert torch.equal(a.state, b.state)
