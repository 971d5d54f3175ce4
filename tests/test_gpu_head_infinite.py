"""Infinite logits of the output head on the GPU: the definition's values, in 64 bits too."""
import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu

BF16, INF = torch.bfloat16, float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


def _inputs(T, V, d, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.randn((T, d), device="cuda", generator=g).abs().add(0.1).to(BF16)
    w = (torch.randn((V, d), device="cuda", generator=g) * 0.1).to(BF16)
    return h, w, torch.randint(0, V, (T,), device="cuda", generator=g)


@pytest.mark.parametrize("T,V,d", [(50, 600, 32), (7, 1000, 2048), (130, 37, 65), (3, 5000, 64)])
@pytest.mark.parametrize("scale", [1.0, -1.0])
def test_a_logit_of_plus_infinity(T, V, d, scale):
    """lse is +Inf, the loss too, unless the target's logit is itself infinite (Inf - Inf); a NaN logit stays NaN."""
    h, w, targets = _inputs(T, V, d)
    for v in (0, V // 2, V - 1):
        wi = w.clone()
        wi[v, 3] = INF * scale
        ti = targets.clone()
        ti[ti == v] = (v + 1) % V
        ti[0] = v
        op = S.HeadLoss(V, d, scale=scale)
        loss, lse = op.loss(h, wi, ti)
        assert (lse == INF).all()
        assert loss[0].isnan() and (loss[1:] == INF).all()
        # exp(l - lse) is 0 of every finite logit, so that their rows' gradients are the targets' alone; Inf - Inf stays NaN
        dw = op.grad(h, wi, ti, lse, torch.ones(T, device="cuda"))[1]
        there = torch.zeros((V, T), dtype=torch.float64, device="cuda")
        there[ti, torch.arange(T, device="cuda")] = 1
        want = -scale * there @ h.double()
        rest = torch.arange(V, device="cuda") != v
        # sums of up to T terms that are exact: fp32 additions, and one rounding to bf16
        assert ((dw[rest].double() - want[rest]).abs() <= (2.0 ** -8 + T * 2.0 ** -23) * want[rest].abs()).all() and dw[v].isnan().all()
        hn = h.clone()
        hn[T - 1, 5] = float("nan")
        lse = op.loss(hn, wi, ti)[1]
        assert lse[T - 1].isnan() and (lse[:T - 1] == INF).all()


def test_infinities_of_both_signs():
    T, V, d = 20, 700, 64
    h, w, targets = _inputs(T, V, d)
    w[::2, 0], w[1, 0] = -INF, INF
    loss, lse = S.HeadLoss(V, d).loss(h, w, torch.full_like(targets, 3))
    assert (lse == INF).all() and (loss == INF).all()
    loss, lse = S.HeadLoss(V, d).loss(h, w, torch.full_like(targets, 2))   # a target without probability
    assert (lse == INF).all() and (loss == INF).all()


@pytest.mark.parametrize("T,V,d", [(50, 600, 32), (70, 337, 65), (300, 700, 2048)])
def test_padding_enters_no_gradient_of_a_table_with_infinities(T, V, d):
    """Rows of the table that no token's target may be (-Inf times what is positive): none has a probability, and padded tokens add nothing to the table's gradient,
    whatever they hold."""
    h, w, targets = _inputs(T, V, d)
    w[V // 2:, 0] = -INF
    targets %= V // 2
    targets[::3] = -1
    h[::6] = float("nan")
    there = targets >= 0
    op = S.HeadLoss(V, d)
    _, lse = op.loss(h, w, targets)
    dloss = torch.rand(T, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)) + 0.5
    dloss[~there] = float("nan")
    dw = op.grad(h, w, targets, lse, dloss)[1]
    assert dw.isfinite().all() and (dw[V // 2:] == 0).all()
    kept = op.grad(h[there], w, targets[there], lse[there].contiguous(), dloss[there])[1]
    # the same terms, added up in another order: sums of up to T, each rounded to bf16
    size = (torch.softmax(h[there].double() @ w[: V // 2].double().t(), 1) + torch.nn.functional.one_hot(targets[there], V // 2)).t() @ (h[there].double() * 1.5)
    assert ((dw[: V // 2].double() - kept[: V // 2].double()).abs() <= 2.0 ** -7 * kept[: V // 2].double().abs() + T * 2.0 ** -22 * size).all()
