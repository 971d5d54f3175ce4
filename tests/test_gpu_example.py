"""The example that runs the operators together: its gradients against 64 bits, and that it learns."""
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
    import toy_moe
    return toy_moe


def test_gradients_and_factor(toy):
    """Every gradient that a step leaves for the optimizer. bf16 ones are rounded once (2^-8), the table's twice: the head's part, and
    the sum. The fp32 products between add far less than 1e-4 of a tensor's largest element."""
    m = toy.Model()
    ids, targets = toy.batch(torch.Generator(device="cuda").manual_seed(1))
    before = [p.clone() for p in m.params]
    loss, counts = m.step(1, ids, targets)
    table, gate, up, down = [p.double().requires_grad_() for p in before]
    rows = table.detach().clone().requires_grad_()                     # the lookup's share of the table's gradient
    h = F.embedding(ids, rows) * toy.WIDTH ** 0.5
    s = torch.sigmoid(h @ gate)
    chosen = torch.topk(h @ gate, toy.TOP_K, dim=1).indices
    w = s.gather(1, chosen)
    w = w / w.sum(1, keepdim=True)
    y = torch.einsum("tef,efd->ted", torch.relu(torch.einsum("td,edf->tef", h, up)), down)
    y = torch.gather(y, 1, chosen[:, :, None].expand(-1, -1, toy.WIDTH))
    want = F.cross_entropy((h + (y * w[:, :, None]).sum(1)) @ table.t(), targets)
    assert abs(float(loss) - float(want)) <= 1e-4 * float(want)
    assert torch.equal(counts.long(), torch.bincount(chosen.reshape(-1), minlength=toy.EXPERTS))
    want.backward()
    total = table.grad + rows.grad
    u = 2.0 ** -8
    for got, ref, off in ((m.grads[0], total, u * (table.grad.abs() + total.abs()) * 1.01), (m.grads[1], gate.grad, 0.0),
                          (m.grads[2], up.grad, u * up.grad.abs()), (m.grads[3], down.grad, u * down.grad.abs())):
        assert ((got.double() - ref).abs() <= off + 1e-4 * ref.abs().max()).all()
    norm, gamma = m.clip.result.tolist()
    ref = sum(float(g.double().square().sum()) for g in m.grads) ** 0.5
    assert abs(norm - ref) <= 1e-5 * ref and abs(gamma - min(1.0, toy.MAX_NORM / (ref + 1e-6))) <= 1e-5


def test_it_learns(toy):
    """A uniform guess costs ln 512 = 6.24; seven targets in eight are settled by their token, which costs about 1.0 in the end."""
    losses = toy.train(60)
    assert abs(losses[0] - 6.24) < 0.3
    assert sum(losses[-5:]) / 5 < 4.0
