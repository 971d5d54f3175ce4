"""Refusals of the operators between the router and the loss, host side (no GPU needed: nothing is launched)."""
import ctypes as C
import os
import subprocess
import tempfile

import pytest
import torch

from paper_2607_19058_gb300 import _build
from paper_2607_19058_gb300 import skewadam as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000  # never read: every call here is refused, or has nothing to do
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module", autouse=True)
def lib():
    _build.build()
    return S.load()


def _refused(what, f, *a, code=S.SKEW_EINVAL):
    with pytest.raises(S.SkewError) as e:
        f(*a)
    assert e.value.code == code and what in str(e.value), str(e.value)


def test_struct_layouts():
    expr = ["sizeof(skew_dispatch_config_t)", "offsetof(skew_dispatch_config_t, flags)", "sizeof(skew_experts_config_t)", "offsetof(skew_experts_config_t, flags)",
            "sizeof(skew_head_config_t)", "offsetof(skew_head_config_t, scale)", "offsetof(skew_head_config_t, flags)"]
    prog = '#include <stdio.h>\n#include <stddef.h>\n#include "skewadam.h"\nint main(void) { ' + \
        "".join(f'printf("%zu ", (size_t)({e}));' for e in expr) + " return 0; }\n"
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "l.c"), os.path.join(d, "l")
        open(src, "w").write(prog)
        subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), src, "-o", exe])
        got = [int(x) for x in subprocess.check_output([exe]).split()]
    assert got == [C.sizeof(S.DispatchConfig), S.DispatchConfig.flags.offset, C.sizeof(S.ExpertsConfig), S.ExpertsConfig.flags.offset,
                   C.sizeof(S.HeadConfig), S.HeadConfig.scale.offset, S.HeadConfig.flags.offset]


@pytest.mark.parametrize("config,tokens,what", [
    ((0, 2, 0, 0), 5, "experts"), ((1025, 2, 0, 0), 5, "experts"), ((8, 0, 0, 0), 5, "top_k"), ((8, 65, 0, 0), 5, "top_k"), ((8, 2, 4, 0), 5, "flags"),
    ((8, 2, 0, 1), 5, "flags"), ((8, 2, 0, 0), -1, "tokens"), ((8, 2, 0, 0), (1 << 29) + 1, "tokens"),
])
def test_dispatch_refuses_configs(config, tokens, what):
    c = S.DispatchConfig(*config)
    assert S.skew_dispatch_workspace_bytes(c, tokens) == 0
    _refused(what, S.skew_dispatch_order, c, P, tokens, P, P, P, 1 << 30, 0)
    _refused(what, S.skew_dispatch_spread, c, P, 64, P, P, tokens, 64, P, 0)
    _refused(what, S.skew_dispatch_combine, c, P, P, P, tokens, 64, P, 64, 0)
    _refused(what, S.skew_dispatch_combine_grad, c, P, 64, P, P, P, P, tokens, 64, P, P, 0)


def test_dispatch_refuses_arguments():
    c = S.DispatchConfig(8, 2, 0, 0)
    n = S.skew_dispatch_workspace_bytes(c, 100)
    assert n > 0
    _refused("chosen", S.skew_dispatch_order, c, 0, 100, P, P, P, n, 0)
    _refused("chosen", S.skew_dispatch_order, c, P + 2, 100, P, P, P, n, 0)
    _refused("offsets", S.skew_dispatch_order, c, P, 100, 0, P, P, n, 0)
    _refused("places", S.skew_dispatch_order, c, P, 100, P, 0, P, n, 0)
    for ws, size in ((0, n), (P + 16, n), (P, n - 1)):
        _refused("workspace", S.skew_dispatch_order, c, P, 100, P, P, ws, size, 0)
    for width, ld in ((0, 64), ((1 << 20) + 1, 1 << 21), (64, 63), (64, (1 << 31) + 1)):
        _refused("width", S.skew_dispatch_spread, c, P, ld, P, P, 100, width, P, 0)
        _refused("width", S.skew_dispatch_combine, c, P, P, P, 100, width, P, ld, 0)
        _refused("width", S.skew_dispatch_combine_grad, c, P, ld, P, P, P, P, 100, width, P, P, 0)
    wide = S.DispatchConfig(8, 2, S.DISPATCH_TOKENS_FP32 | S.DISPATCH_ROWS_FP32, 0)
    _refused("x must", S.skew_dispatch_spread, wide, P + 2, 64, P, P, 100, 64, P, 0)
    _refused("rows must", S.skew_dispatch_spread, wide, P, 64, P, P, 100, 64, P + 2, 0)
    _refused("offsets", S.skew_dispatch_spread, c, P, 64, 0, P, 100, 64, P, 0)
    _refused("weights", S.skew_dispatch_combine, c, P, P + 1, P, 100, 64, P, 64, 0)
    _refused("weights", S.skew_dispatch_combine_grad, c, P, 64, P, 0, P, P, 100, 64, P, P, 0)
    _refused("dweights", S.skew_dispatch_combine_grad, c, P, 64, P, P, P, P, 100, 64, P, 0, 0)
    _refused("drows", S.skew_dispatch_combine_grad, c, P, 64, P, P, P, P, 100, 64, P + 1, P, 0)
    S.skew_dispatch_spread(c, 0, 64, P, 0, 0, 64, 0, 0)  # no tokens: nothing to do


@pytest.mark.parametrize("config,rows,what", [
    ((0, 8, 8, 0), 5, "experts"), ((1025, 8, 8, 0), 5, "experts"), ((2, 0, 8, 0), 5, "n and m"), ((2, 8, (1 << 20) + 1, 0), 5, "n and m"), ((2, 8, 8, 4), 5, "flags"),
    ((2, 8, 8, 0), -1, "rows"), ((2, 8, 8, 0), (1 << 30) + 1, "rows"),
])
def test_experts_refuse_configs(config, rows, what):
    c = S.ExpertsConfig(*config)
    assert what == "rows" or S.skew_experts_workspace_bytes(c) == 0
    _refused(what, S.skew_experts_product, c, P, 8, P, P, rows, P, 0)
    _refused(what, S.skew_experts_grad_rows, c, P, 8, P, P, rows, P, 0)
    _refused(what, S.skew_experts_grad, c, P, 8, P, 8, P, rows, 0, P, P, 1 << 40, 0)


def test_experts_refuse_arguments():
    c = S.ExpertsConfig(2, 8, 16, S.EXPERTS_ROWS_FP32 | S.EXPERTS_GRAD_FP32)
    _refused("offsets", S.skew_experts_product, c, P, 8, P, 0, 5, P, 0)
    _refused("offsets", S.skew_experts_product, c, P, 8, P, P + 2, 5, P, 0)
    _refused("rows must", S.skew_experts_product, c, 0, 8, P, P, 5, P, 0)
    _refused("rows must", S.skew_experts_product, c, P + 1, 8, P, P, 5, P, 0)
    _refused("stride", S.skew_experts_product, c, P, 7, P, P, 5, P, 0)
    _refused("stride", S.skew_experts_grad_rows, c, P, 15, P, P, 5, P, 0)
    n = S.skew_experts_workspace_bytes(c)
    _refused("stride", S.skew_experts_grad, c, P, 8, P, (1 << 31) + 1, P, 5, 0, P, P, n, 0)
    _refused("w must", S.skew_experts_product, c, P, 8, 0, P, 5, P, 0)
    _refused("result", S.skew_experts_product, c, P, 8, P, P, 5, P + 2, 0)
    _refused("base", S.skew_experts_grad, c, P, 8, P, 16, P, 5, P + 2, P, P, n, 0)
    _refused("dw", S.skew_experts_grad, c, P, 8, P, 16, P, 5, P, 0, P, n, 0)
    for ws, size in ((0, n), (P + 16, n), (P, n - 1)):
        _refused("workspace", S.skew_experts_grad, c, P, 8, P, 16, P, 5, 0, P, ws, size, 0)
    S.skew_experts_product(c, 0, 8, P, P, 0, 0, 0)  # no rows: nothing to do


@pytest.mark.parametrize("config,tokens,what", [
    ((0, 8, 1.0, 0), 5, "rows"), (((1 << 24) + 1, 8, 1.0, 0), 5, "rows"), ((9, 0, 1.0, 0), 5, "width"), ((9, (1 << 20) + 1, 1.0, 0), 5, "width"),
    ((9, 8, float("inf"), 0), 5, "scale"), ((9, 8, float("nan"), 0), 5, "scale"), ((9, 8, 1.0, 2), 5, "flags"), ((9, 8, 1.0, 0), -1, "tokens"),
    ((9, 8, 1.0, 0), (1 << 24) + 1, "tokens"),
])
def test_head_refuses_configs(config, tokens, what):
    c = S.HeadConfig(*config)
    assert S.skew_head_loss_workspace_bytes(c, tokens) == S.skew_head_grad_workspace_bytes(c, tokens) == 0
    _refused(what, S.skew_head_loss, c, P, 8, P, P, tokens, P, P, P, 1 << 40, 0)
    _refused(what, S.skew_head_grad, c, P, 8, P, P, tokens, P, P, P, 0, P, P, 1 << 40, 0)


def test_head_refuses_arguments():
    c = S.HeadConfig(100, 8, 1.0, S.HEAD_IDS_64)
    n, m = S.skew_head_loss_workspace_bytes(c, 5), S.skew_head_grad_workspace_bytes(c, 5)
    good = [P, 8, P, P, 5, P, P, P, n, 0]
    for k, v, what in ((0, 0, "h must"), (0, P + 1, "h must"), (1, 7, "stride"), (2, 0, "table"), (3, P + 4, "targets"), (5, 0, "loss"), (6, P + 2, "lse"),
                       (7, 0, "workspace"), (7, P + 128, "workspace"), (8, n - 1, "workspace")):
        _refused(what, S.skew_head_loss, c, *[v if i == k else a for i, a in enumerate(good)])
    good = [P, 8, P, P, 5, P, P, P, 0, P, P, m, 0]
    for k, v, what in ((0, 0, "h must"), (1, (1 << 31) + 1, "stride"), (2, P + 1, "table"), (3, 0, "targets"), (5, 0, "lse"), (6, 0, "dloss"), (7, P + 1, "dh"),
                       (8, P + 1, "base"), (9, 0, "dtable"), (10, P + 8, "workspace"), (11, m - 1, "workspace")):
        _refused(what, S.skew_head_grad, c, *[v if i == k else a for i, a in enumerate(good)])


def test_head_does_not_keep_the_logits():
    """The gradients' workspace stays below the logits' size where these are large, whatever the number of tokens."""
    for T, V, d in ((8192, 50304, 4096), (65536, 131072, 1024), (1 << 20, 50257, 768)):
        c = S.HeadConfig(V, d, 1.0, 0)
        assert S.skew_head_grad_workspace_bytes(c, T) <= max(512 << 20, T * 256 * 2) + T * d * 6 + (100 << 20)
        assert S.skew_head_loss_workspace_bytes(c, T) < T * V // 8 + 2 * T * d + 1024


def test_wrappers_refuse():
    with pytest.raises(TypeError):
        S.Dispatch(8, 2, token_dtype=torch.float16)
    with pytest.raises(TypeError):
        S.Experts(8, 2, 2, grad_dtype=torch.float64)
    for make in (lambda: S.Dispatch(0, 2), lambda: S.Dispatch(8, 65), lambda: S.Experts(0, 4, 4), lambda: S.Experts(4, 4, 1 << 21), lambda: S.Experts(4, -4, 4),
                 lambda: S.HeadLoss(0, 4), lambda: S.HeadLoss(10, 4, scale=float("nan"))):
        with pytest.raises(S.SkewError) as e:
            make()
        assert e.value.code == S.SKEW_EINVAL
    for make in (lambda: S.Dispatch((1 << 32) + 8, 2), lambda: S.Experts(4, (1 << 32) + 4, 4), lambda: S.HeadLoss(1 << 70, 4)):
        with pytest.raises(ValueError):
            make()
    host = torch.zeros((4, 2), dtype=torch.int32)
    d = S.Dispatch(8, 2)
    with pytest.raises(ValueError):
        d.order(host)
    with pytest.raises(ValueError):
        d.spread(torch.zeros((4, 16), dtype=BF16), (torch.zeros(9, dtype=torch.int32), host))
    ex = S.Experts(2, 8, 8)
    x, w, o = torch.zeros((4, 8), dtype=BF16), torch.zeros((2, 8, 8), dtype=BF16), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: ex.product(x, w, o), lambda: ex.grad_rows(x, w, o), lambda: ex.grad(x, x, o)):
        with pytest.raises(ValueError):
            call()
    head = S.HeadLoss(10, 8)
    with pytest.raises(ValueError):
        head.loss(x, torch.zeros((10, 8), dtype=BF16), torch.zeros(4, dtype=torch.int64))


def test_workspaces_are_what_the_tiles_need():
    """Matrices of many tiles are not cut along the rows, and keep nothing for it."""
    assert S.skew_experts_workspace_bytes(S.ExpertsConfig(128, 4096, 4096, 0)) == 256
    small = S.skew_experts_workspace_bytes(S.ExpertsConfig(1, 64, 64, 0))
    assert 256 * 256 * 4 < small <= 100 << 20
    assert S.skew_head_grad_workspace_bytes(S.HeadConfig(50304, 4096, 1.0, 0), 8192) < (512 << 20) + 8192 * 4096 * 6 + 8192


def _fakes(monkeypatch):
    from test_ops_host_streams import FakeTensor as F
    launched, current = [], [0]
    launch = lambda *a: launched.append(a) or 0  # noqa: E731
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 2)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(S, "_raw_stream", lambda: lambda index: 100 + index)
    monkeypatch.setattr(torch, "empty", lambda n, dtype=None, device=None: F((n,), dtype, torch.device(device).index))
    d, e, h = S.Dispatch(8, 2), S.Experts(8, 16, 24), S.HeadLoss(50, 16)
    for o in (d, e, h):
        o._new = lambda shape, strides, dtype, device: F(shape, dtype, device.index)
    d._order = d._spread = d._combine = d._combine_grad = e._product = e._grad_rows = e._grad = h._loss = h._grad = launch

    def calls(i):
        f = lambda shape, dtype=BF16: F(shape, dtype, i)  # noqa: E731
        I, W = torch.int32, torch.float32
        order, x, rows, w = (f((9,), I), f((5, 2), I)), f((5, 16)), f((10, 16)), f((5, 2), W)
        dy, m, t, l = f((10, 24)), f((8, 16, 24)), f((5,), torch.int64), f((5,), W)
        return [lambda: d.order(f((5, 2), I)), lambda: d.spread(x, order), lambda: d.combine(rows, w, order), lambda: d.combine_grad(x, rows, w, order),
                lambda: e.product(rows, m, order[0]), lambda: e.grad_rows(dy, m, order[0]), lambda: e.grad(rows, dy, order[0]),
                lambda: h.loss(x, f((50, 16)), t), lambda: h.grad(x, f((50, 16)), t, l, l)]
    return launched, current, calls


def test_tensors_of_another_device_are_refused(monkeypatch):
    launched, current, calls = _fakes(monkeypatch)
    for k, call in enumerate(calls(0)):
        call()
        assert len(launched) == k + 1
    launched.clear()
    for call in calls(1):
        with pytest.raises(ValueError, match="current device"):
            call()
    assert not launched
    current[0] = 1
    for call in calls(1):
        call()
    assert len(launched) == 9 and all(a[-1] == 101 for a in launched)


def test_a_workspace_for_each_device(monkeypatch):
    launched, current, calls = _fakes(monkeypatch)
    at = {0: set(), 1: set()}
    for k in range(6):
        current[0] = i = k % 2
        for call in (calls(i)[0], calls(i)[6], calls(i)[8]):
            call()
            at[i].add(launched[-1][-3])
    assert len(at[0]) == len(at[1]) == 3 and not at[0] & at[1]
