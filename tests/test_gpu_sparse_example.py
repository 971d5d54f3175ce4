"""The example that runs every operator in a row: its gradients against 64 bits, that it runs, and that it can be captured."""
import os
import sys

import pytest
import torch
import torch.nn.functional as F

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def toy():
    from paper_2607_19058_gb300 import _build
    _build.build()
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import sparse_moe
    return sparse_moe


def _want(toy, params, ids, targets, chosen):
    table, gate, up, down = [p.double().requires_grad_() for p in params]
    h = table[ids] * toy.WIDTH ** 0.5
    s = torch.sigmoid(h @ gate)
    w = s.gather(1, chosen.long())
    w = w / w.sum(1, keepdim=True)
    y = torch.einsum("tef,efd->ted", torch.relu(torch.einsum("td,edf->tef", h, up)), down)
    y = torch.gather(y, 1, chosen.long()[:, :, None].expand(-1, -1, toy.WIDTH))
    loss = F.cross_entropy((h + (y * w[:, :, None]).sum(1)) @ table.t(), targets, ignore_index=-1)
    loss.backward()
    return loss.detach(), [p.grad for p in (table, gate, up, down)]


def test_gradients(toy):
    """Activations go through up to six roundings to bf16 on their way (lookup, rows, hidden, down, combined, and a gradient's own), each by half a step of 2^-8
    at most; errors of different elements are independent, so that a gradient's 2-norm is off by less than six half steps together, 6 * 2^-8; the
    router's goes through the difference of two such, and is allowed twice that."""
    m = toy.Model()
    ids, targets = toy.batch(torch.Generator(device="cuda").manual_seed(1))
    loss, counts = m.gradients(ids, targets)
    h = m.embedding.lookup(m.table, ids)
    chosen, _, want_counts = m.router.route(h.float() @ m.gate)
    want, grads = _want(toy, m.params, ids, targets, chosen)
    assert torch.equal(counts, want_counts)
    assert abs(float(loss) - float(want)) <= 2.0 ** -8 * float(want)
    for got, ref, k in zip(m.grads, grads, (6, 12, 6, 6)):
        assert float((got.double() - ref).norm()) <= k * 2.0 ** -8 * float(ref.norm())


def test_it_runs(toy):
    losses = toy.train(5)
    assert len(losses) == 5 and all(v == v and abs(v) < 10 for v in losses)


def test_captured_and_replayed(toy):
    """A step's gradients in a graph, replayed on other tokens: the same bits as without."""
    m = toy.Model()
    gen = torch.Generator(device="cuda").manual_seed(2)
    first, second = toy.batch(gen), toy.batch(gen)
    ids, targets = first[0].clone(), first[1].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.gradients(ids, targets)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, counts = m.gradients(ids, targets)
    for b in (second, first):
        ids.copy_(b[0])
        targets.copy_(b[1])
        graph.replay()
        got = [loss.clone(), counts.clone()] + [g.clone() for g in m.grads]
        again = m.gradients(*b)
        assert all(torch.equal(x, y) for x, y in zip(got, [*again, *m.grads]))
