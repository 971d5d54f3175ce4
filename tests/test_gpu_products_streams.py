"""Rows by expert, products and the head's loss on streams other than the current one, and in graphs that share an object's workspace."""
import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_19058_gb300 import _build
    _build.build()


class Set:
    """Objects of each operator, and a pass over all of their calls."""

    def __init__(self, E=12, k=2, n=96, m=40, V=700):
        self.d, self.e, self.h = S.Dispatch(E, k), S.Experts(E, n, m), S.HeadLoss(V, n)
        self.E, self.k, self.n, self.m, self.V = E, k, n, m, V

    def inputs(self, T, seed=1):
        g = torch.Generator(device="cuda").manual_seed(seed)
        r = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
        return (torch.randint(-1, self.E, (T, self.k), device="cuda", generator=g).int(), r(T, self.n).to(BF16), r(self.E, self.n, self.m).to(BF16), torch.rand((T, self.k), device="cuda", generator=g),
                (r(self.V, self.n) * 0.1).to(BF16), torch.randint(-1, self.V, (T,), device="cuda", generator=g), r(T))

    def run(self, chosen, x, w, weights, table, targets, dloss, **s):
        order = self.d.order(chosen, **s)
        rows = self.d.spread(x, order, **s)
        y = self.e.product(rows, w, order[0], **s)
        out = self.d.combine(y, weights, order, **s)
        drows, dweights = self.d.combine_grad(out, y, weights, order, **s)
        dx = self.e.grad_rows(drows, w, order[0], **s)
        dw = self.e.grad(rows, drows, order[0], **s)
        loss, lse = self.h.loss(x, table, targets, **s)
        return [*order, rows, y, out, drows, dweights, dx, dw, loss, lse, *self.h.grad(x, table, targets, lse, dloss, **s)]


@pytest.mark.parametrize("raw", [False, True])
def test_a_stream_given(raw):
    a = Set()
    ins = a.inputs(3000)
    want = a.run(*ins)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(10):  # blocks of dropped results go to nobody else before the stream has passed them
        got = a.run(*ins, stream=side.cuda_stream if raw else side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    a.e.sync_status(side)


def test_graphs_that_share_workspaces():
    """Two graphs of one object's calls, of different sizes, with larger eager calls between: each as without."""
    a = Set()
    small, large = a.inputs(500), a.inputs(2500, 2)
    want = [a.run(*i) for i in (small, large)]
    graphs, got = [], []
    for i in (small, large):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(a.run(*i))
        graphs.append(g)
    a.run(*a.inputs(60000, 3))  # workspaces grow: the graphs keep theirs
    junk = [torch.full((1 << 20,), -1, dtype=torch.int32, device="cuda") for _ in range(8)]
    for _ in range(2):
        for k in (1, 0):
            graphs[k].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(got[k], want[k])) and len(junk) == 8


def test_captured_behind_other_things_than_kernels():
    """A product right behind a copy, a zero-fill, and what comes from another stream: in a graph as without."""
    a = Set()
    chosen, x, w, weights, table, targets, dloss = a.inputs(700)
    order = a.d.order(chosen)
    rows = a.d.spread(x, order)
    want = a.e.product(rows, w, order[0]), a.h.loss(x, table, targets)[1]
    into, side = torch.empty_like(rows), torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        into.copy_(rows)
        side.wait_stream(main)
        with torch.cuda.stream(side):
            h = x * 1
            lse = a.h.loss(h, table, targets)[1]
        y = a.e.product(into, w, order[0])
        z = torch.zeros((1000, 1000), device="cuda")
        main.wait_stream(side)
        y2 = a.e.product(into, w, order[0])
        z += 1
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(y2, want[0]) and torch.equal(lse, want[1]) and (z == 1).all()


def test_rows_behind_a_view_are_left_as_they_were():
    """Results go where they belong: out= tensors that lie inside a larger one."""
    a = Set()
    chosen, x, w, weights, table, targets, dloss = a.inputs(300)
    order = a.d.order(chosen)
    rows = a.d.spread(x, order)
    dy = torch.randn((600, a.m), device="cuda").to(BF16)
    want = a.e.grad(rows, dy, order[0])
    big = torch.full((a.E + 2, a.n, a.m), 7.0, dtype=BF16, device="cuda")
    a.e.grad(rows, dy, order[0], out=big[1:-1])
    assert torch.equal(big[1:-1], want) and (big[0] == 7).all() and (big[-1] == 7).all()
    _, lse = a.h.loss(x, table, targets)
    want = a.h.grad(x, table, targets, lse, dloss)[1]
    big = torch.full((a.V + 3, a.n), 7.0, dtype=BF16, device="cuda")
    a.h.grad(x, table, targets, lse, dloss, out=big[2:-1])
    assert torch.equal(big[2:-1], want) and (big[:2] == 7).all() and (big[-1] == 7).all()


def test_wrappers_refuse():
    a = Set()
    chosen, x, w, weights, table, targets, dloss = a.inputs(50)
    order = a.d.order(chosen)
    rows = a.d.spread(x, order)
    _, lse = a.h.loss(x, table, targets)
    bad = [lambda: a.d.order(chosen.long()), lambda: a.d.order(chosen[:, :1]), lambda: a.d.order(chosen.t()), lambda: a.d.spread(x.float(), order), lambda: a.d.spread(x[:-1], order),
           lambda: a.d.spread(x.t(), order), lambda: a.d.combine(rows[:-1], weights, order), lambda: a.d.combine(rows, weights.double(), order), lambda: a.d.combine(rows.float(), weights, order),
           lambda: a.d.combine(rows, weights, (order[0][:-1], order[1])) and a.d.spread(x, (order[0][:-1], order[1])), lambda: a.d.combine_grad(x[:, :-1], rows, weights, order),
           lambda: a.e.product(rows[:, :-1], w, order[0]), lambda: a.e.product(rows.float(), w, order[0]), lambda: a.e.product(rows, w[:-1], order[0]), lambda: a.e.product(rows, w, order[0].long()),
           lambda: a.e.product(rows, w.transpose(1, 2), order[0]), lambda: a.e.grad(rows, rows, order[0]), lambda: a.e.grad(rows, rows[:-1, :a.m].contiguous(), order[0]),
           lambda: a.e.grad(rows, rows[:, :a.m].contiguous(), order[0], base=w.float()), lambda: a.h.loss(x.float(), table, targets), lambda: a.h.loss(x, table[:-1], targets),
           lambda: a.h.loss(x, table, targets[:-1]), lambda: a.h.grad(x, table, targets, lse[:-1], dloss), lambda: a.h.grad(x, table, targets, lse, dloss.double()),
           lambda: a.h.grad(x, table, targets, lse, dloss, base=table.float()), lambda: a.h.grad(x, table, targets.cpu(), lse, dloss)]
    for k, call in enumerate(bad):
        with pytest.raises((ValueError, TypeError)):
            call()
            pytest.fail(f"call {k} was taken")
    with pytest.raises(TypeError):
        a.h.loss(x, table, targets.float())
