"""How much workspace the wrappers pass, host side: it goes by the device (by its SMs), and what is kept of the answers is bounded."""
import pytest
import torch

from paper_2607_19058_gb300 import skewadam as S
from test_ops_host_experts import _fakes
from test_ops_host_streams import FakeTensor


def _by_device(monkeypatch, current, asked):
    for name in ("skew_dispatch_workspace_bytes", "skew_experts_workspace_bytes", "skew_head_loss_workspace_bytes", "skew_head_grad_workspace_bytes"):
        true = getattr(S, name)

        def fake(c, *tokens, true=true):
            asked.append(tokens)
            n = true(c, *tokens)
            return n and n + 4096 * (1 + current[0])
        monkeypatch.setattr(S, name, fake)


def test_workspaces_are_of_the_size_that_the_device_asks_for(monkeypatch):
    launched, current, calls = _fakes(monkeypatch)
    asked = []
    _by_device(monkeypatch, current, asked)
    sizes = {0: [], 1: []}
    for i in (0, 1, 0, 1):
        current[0] = i
        launched.clear()
        for k in (0, 6, 7, 8):
            calls(i)[k]()
        sizes[i].append([a[-2] for a in launched])
        if len(sizes[i]) == 1:
            asked.clear()
    assert sizes[0][0] == sizes[0][1] and sizes[1][0] == sizes[1][1]
    assert [b - a for a, b in zip(sizes[0][0], sizes[1][0])] == [4096] * 4
    assert not asked  # a second call of a size asks for nothing


def test_what_is_kept_of_the_sizes_is_bounded(monkeypatch):
    launched, current, _ = _fakes(monkeypatch)
    monkeypatch.setattr(S, "_raw_stream", lambda: lambda index: 100 + index)
    d, h = S.Dispatch(8, 2), S.HeadLoss(50, 16)
    d._new = h._new = lambda shape, strides, dtype, device: FakeTensor(shape, dtype, device.index)
    d._order = h._loss = lambda *a: 0
    table = FakeTensor((50, 16))
    for T in range(1, 5000):
        d.order(FakeTensor((T, 2), torch.int32))
        h.loss(FakeTensor((T, 16)), table, FakeTensor((T,), torch.int64))
    for o in (d, h):
        kept = [v for v in (*vars(o).values(), *(getattr(o._workspace, s) for s in o._workspace.__slots__)) if isinstance(v, dict)]
        assert kept and all(len(v) <= 1024 for v in kept)
    with pytest.raises(S.SkewError):  # more tokens than there may be: refused each time
        d.order(FakeTensor(((1 << 29) + 1, 2), torch.int32))
    with pytest.raises(S.SkewError):
        d.order(FakeTensor(((1 << 29) + 1, 2), torch.int32))
