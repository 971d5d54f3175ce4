"""The output head's loss and gradients on the GPU, against 64 bits.

A logit is a sum of d products (exact in fp32) off by at most d * 2^-23 of the magnitudes, called e here, times the scale. An exponential is
off by e, by 2^-22 (its approximation) and by 2^-22 of the logits' size (what powers of two are made of); a row's sum adds at most 128 + 64
roundings of 2^-24. lse and loss add a few roundings of their sizes. A logit's gradient is rounded to bf16: 2^-8 of it; dh and dW are sums of
such terms on the tensor cores, at most K * 2^-23 of the magnitudes, rounded to bf16: 2^-8 of the result.
"""
import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _inputs(T, V, d, sigma, dtype, seed=1):
    g = _gen(seed)
    h = torch.randn((T, d), device="cuda", generator=g).to(BF16)
    w = (torch.randn((V, d), device="cuda", generator=g) * sigma).to(BF16)
    t = torch.randint(-1, V + 1, (T,), device="cuda", generator=g).to(dtype)  # some outside
    return h, w, t, torch.randn(T, device="cuda", generator=g)


def _check(T, V, d, sigma=0.1, scale=1.0, dtype=torch.int64, base=False, lay=None):
    h, w, targets, dloss = _inputs(T, V, d, sigma, dtype)
    if lay:
        h = lay(h)
    op = S.HeadLoss(V, d, scale=scale)
    loss, lse = op.loss(h, w, targets)
    H, W = h.double(), w.double()
    x, e = scale * H @ W.t(), abs(scale) * d * 2.0 ** -23 * (H.abs() @ W.abs().t())
    there = (targets >= 0) & (targets < V)
    at = torch.where(there, targets, 0).long()[:, None]
    want = torch.logsumexp(x, 1)
    size = x.abs().amax(1) + want.abs() + 1
    off = e.amax(1) + 192 * 2.0 ** -24 + 4 * 2.0 ** -22 * size
    assert ((lse.double() - want).abs() <= off).all()
    ref = torch.where(there, want - x.gather(1, at)[:, 0], 0.0)
    assert ((loss.double() - ref).abs() <= 2 * off + 4 * 2.0 ** -24 * size).all() and (loss[~there] == 0).all()
    # gradients
    dloss[~there] = float("nan")  # not read
    b = (torch.randn((V, d), device="cuda", generator=_gen(9)) * 0.1).to(BF16) if base else None
    dh, dw = op.grad(h, w, targets, lse, dloss, base=b)
    p = torch.softmax(x, 1)
    near = p * (2 * off[:, None])                           # of the exponential, by the logit's and lse's errors
    p.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float64))
    g = torch.where(there, dloss, 0.0).double()[:, None]
    p, near = p * g, (near + p.abs() * (2.0 ** -8 + 2.0 ** -22)) * g.abs()
    for got, ref, terms, noise, K, more in ((dh, scale * p @ W, abs(scale) * p.abs() @ W.abs(), abs(scale) * near @ W.abs(), V, 0.0),
                                            (dw, scale * p.t() @ H, abs(scale) * p.abs().t() @ H.abs(), abs(scale) * near.t() @ H.abs(), T, 0.0 if b is None else b.double())):
        ref = ref + more
        allow = noise + K * 2.0 ** -23 * terms + 2.0 ** -8 * ref.abs() * 1.01 + 1e-38
        bad = (got.double() - ref).abs() > allow
        assert got.dtype == BF16 and not bad.any(), (int(bad.sum()), torch.nonzero(bad)[:4].tolist())
        assert float((got.double() - ref).norm()) <= 2.0 ** -7 * float(ref.norm()) + 1e-30
    assert (dh[~there] == 0).all()
    again = op.grad(h, w, targets, lse, dloss, base=b)
    assert torch.equal(again[0], dh) and torch.equal(again[1], dw)                 # the same bits again
    if base:
        op.grad(h, w, targets, lse, dloss, base=b, out=b)                          # in place
        assert torch.equal(b, dw)
    op.sync_status()


SIZES = [(1, 1, 1), (1, 512, 64), (7, 3, 8), (128, 128, 64), (129, 257, 72), (300, 1000, 200), (64, 5003, 128), (1000, 511, 65), (33, 130, 1001), (2, 20000, 16)]


@pytest.mark.parametrize("T,V,d", SIZES)
def test_loss_and_gradients(T, V, d):
    _check(T, V, d)
    _check(T, V, d, scale=0.37, dtype=torch.int32, base=True)


@pytest.mark.parametrize("scale", [-1.5, 0.0, 8.0])
def test_scales(scale):
    _check(100, 700, 96, scale=scale, sigma=0.3)


def test_several_pieces():
    """Tokens enough that the logits' gradient takes the vocabulary in more than one piece."""
    T, V, d = 40000, 9000, 64
    assert T * V * 2 > 512 << 20
    _check(T, V, d, base=True)
    _check(T - 1, V + 3, d - 1, dtype=torch.int32)


def test_rows_that_lie_apart():
    def apart(t):
        big = torch.full((t.shape[0], t.shape[1] + 24), float("nan"), dtype=t.dtype, device="cuda")
        big[:, 8:8 + t.shape[1]] = t
        return big[:, 8:8 + t.shape[1]]

    def off(t):
        big = torch.full((t.shape[0], t.shape[1] + 3), float("nan"), dtype=t.dtype, device="cuda")
        big[:, 1:1 + t.shape[1]] = t
        return big[:, 1:1 + t.shape[1]]
    _check(70, 300, 128, lay=apart)
    _check(70, 300, 128, lay=off)


def test_a_table_off_16_bytes():
    T, V, d = 90, 200, 64
    h, w, t, g = _inputs(T, V, d, 0.1, torch.int64)
    def off(x):
        big = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")
        big[1:] = x.reshape(-1)
        return big[1:].view(x.shape)
    op = S.HeadLoss(V, d)
    loss, lse = op.loss(h, w, t)
    assert torch.equal(op.loss(h, off(w), t)[1], lse)
    dh, dw = op.grad(h, w, t, lse, g)
    dh2, dw2 = op.grad(h, off(w), t, lse, g, out=off(torch.zeros_like(w)))
    assert torch.equal(dh, dh2) and torch.equal(dw, dw2)


def test_large_and_infinite_logits():
    """Logits of hundreds: the largest is taken off. Rows of the table that are -Inf times a positive activation have no probability;
    a NaN stays with its token."""
    T, V, d = 50, 600, 32
    h, w, t, g = _inputs(T, V, d, 20.0, torch.int64)
    t = t.clamp(0, V - 1)
    op = S.HeadLoss(V, d)
    loss, lse = op.loss(h, w, t)
    want = torch.logsumexp(h.double() @ w.double().t(), 1)
    assert loss.isfinite().all() and ((lse.double() - want).abs() <= 1e-5 * want.abs() + 1e-3).all()
    h = h.abs() + 0.1
    w[:, 0] = 0.0
    w[300:, 0] = float("-inf")  # the last tiles whole
    t = t.clamp(max=299)
    loss, lse = op.loss(h, w, t)
    want = torch.logsumexp(h.double() @ w[:300].double().t(), 1)
    assert ((lse.double() - want).abs() <= 1e-5 * want.abs() + 1e-3).all()
    w[:, 0] = 0.0
    w[:300, 0] = float("-inf")  # the first
    loss, lse = op.loss(h, w, t + 300)
    want = torch.logsumexp(h.double() @ w[300:].double().t(), 1)
    assert ((lse.double() - want).abs() <= 1e-5 * want.abs() + 1e-3).all()
    w[:, 0] = 0.0
    h[7, 3] = float("nan")
    loss, lse = op.loss(h, w, t)
    assert lse[7].isnan() and loss[7].isnan() and int(lse.isnan().sum()) == 1
    t[7] = -1                                              # a padded token: its NaN enters no gradient
    loss, lse = op.loss(h, w, t)
    assert loss[7] == 0
    dh, dw = op.grad(h, w, t, lse, g)
    assert (dh[7] == 0).all() and dh.isfinite().all()
    assert dw[:300].isfinite().all()


def test_no_tokens_and_padding_alone():
    op = S.HeadLoss(300, 64)
    w = _inputs(1, 300, 64, 0.1, torch.int64)[1]
    none = torch.empty((0, 64), dtype=BF16, device="cuda")
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    loss, lse = op.loss(none, w, ids)
    assert loss.shape == lse.shape == (0,)
    dh, dw = op.grad(none, w, ids, lse, lse)
    assert dh.shape == (0, 64) and (dw == 0).all()
    dh, dw = op.grad(none, w, ids, lse, lse, base=w)
    assert torch.equal(dw, w)
    h = _inputs(20, 300, 64, 0.1, torch.int64)[0]
    ids = torch.full((20,), -1, device="cuda")
    loss, lse = op.loss(h, w, ids)
    dh, dw = op.grad(h, w, ids, lse, torch.ones(20, device="cuda"), base=w)
    assert (loss == 0).all() and (dh == 0).all() and torch.equal(dw, w)


def test_gradients_by_differences():
    """The loss's change along a direction, by central differences in 64 bits of the formula, is what the gradients say: within what their
    terms' rounding to bf16 (2^-8, twice) leaves of the magnitudes."""
    T, V, d = 60, 250, 48
    h, w, t, g = _inputs(T, V, d, 0.2, torch.int64)
    op = S.HeadLoss(V, d)
    _, lse = op.loss(h, w, t)
    dh, dw = op.grad(h, w, t, lse, g)
    there = (t >= 0) & (t < V)
    at = torch.where(there, t, 0)[:, None]

    def total(H, W):
        x = H @ W.t()
        return float((torch.where(there, torch.logsumexp(x, 1) - x.gather(1, at)[:, 0], 0.0) * torch.where(there, g, 0.0).double()).sum())
    u, v = (torch.randn(s, device="cuda", dtype=torch.float64, generator=_gen(3)) for s in (h.shape, w.shape))
    H, W, s = h.double(), w.double(), 1e-5
    for got, up, down, size in (((dh.double() * u).sum(), total(H + s * u, W), total(H - s * u, W), (dh.double() * u).abs().sum()),
                                ((dw.double() * v).sum(), total(H, W + s * v), total(H, W - s * v), (dw.double() * v).abs().sum())):
        assert abs(float(got) - (up - down) / (2 * s)) <= 2.0 ** -6 * float(size)
