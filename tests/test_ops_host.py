"""Refusals of the operators around the step, host side (no GPU needed: nothing is launched)."""
import ctypes as C
import os
import subprocess
import tempfile

import pytest

from paper_2607_19058_gb300 import _build
from paper_2607_19058_gb300 import skewadam as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def lib():
    _build.build()
    return S.load()


def _sizes(expr):
    prog = '#include <stdio.h>\n#include <stddef.h>\n#include "skewadam.h"\nint main(void) { ' + \
        "".join(f'printf("%zu ", (size_t)({e}));' for e in expr) + " return 0; }\n"
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "l.c"), os.path.join(d, "l")
        open(src, "w").write(prog)
        subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), src, "-o", exe])
        return [int(x) for x in subprocess.check_output([exe]).split()]


def test_clip_struct_layout():
    assert _sizes(["sizeof(skew_clip_desc_t)", "offsetof(skew_clip_desc_t, numel)", "offsetof(skew_clip_desc_t, flags)"]) == \
        [C.sizeof(S.ClipDesc), S.ClipDesc.numel.offset, S.ClipDesc.flags.offset]


def _refused(code, what, f, *a):
    with pytest.raises(S.SkewError) as e:
        f(*a)
    assert e.value.code == code and what in str(e.value), str(e.value)


@pytest.mark.parametrize("desc,what", [
    ((0, 0, 5, 0, 0), "null grad"),
    ((0x1000, 0x1000, -1, 0, 0), "numel"),
    ((0x1000, 0x1000, (1 << 40) + 1, 0, 0), "numel"),
    ((0x1001, 0x1000, 5, 0, 0), "aligned"),
    ((0x1002, 0x1000, 5, S.CLIP_GRAD_FP32, 0), "aligned"),
    ((0x1000, 0x1002, 5, S.CLIP_GRAD_FP32 | S.CLIP_OUT_FP32, 0), "aligned"),
    ((0x1000, 0x2000, 5, S.CLIP_OUT_FP32, 0), "bf16"),
    ((0x1000, 0x1000, 5, S.CLIP_GRAD_FP32, 0), "in place"),
    ((0x1000, 0x1000, 5, 4, 0), "flags"),
    ((0x1000, 0x1000, 5, 0, 1), "flags"),
])
def test_clip_refuses(desc, what):
    _refused(S.SKEW_EINVAL, what, S.skew_clip_create, [S.ClipDesc(*desc)])


def test_clip_refuses_calls_out_of_order():
    _refused(S.SKEW_EINVAL, "some tensors", S.skew_clip_create, [S.ClipDesc(0x1000, 0x1000, 5, 0, 0), S.ClipDesc(0x2000, 0, 5, 0, 0)])
    h = S.skew_clip_create([S.ClipDesc(0x1000, 0, 100, 0, 0)])
    n = S.skew_clip_workspace_bytes(h)
    assert n > 0
    _refused(S.SKEW_ESTATE, "before", S.skew_clip_norm, h, 1.0, 0x1000, 0)
    _refused(S.SKEW_EINVAL, "workspace", S.skew_clip_bind, h, 0, n, 0)
    _refused(S.SKEW_EINVAL, "workspace", S.skew_clip_bind, h, 0x1010, n, 0)
    _refused(S.SKEW_EINVAL, "workspace", S.skew_clip_bind, h, 0x1000, n - 1, 0)
    S.skew_clip_destroy(h)
    _refused(S.SKEW_EINVAL, "NULL", S.skew_clip_norm, None, 1.0, 0x1000, 0)
    assert S.skew_clip_workspace_bytes(None) == 0
    assert S.load().skew_clip_destroy(None) == S.SKEW_OK


def test_clip_wrapper_refuses_host_tensors_and_types():
    import torch
    with pytest.raises(ValueError):
        S.GradClip([torch.zeros(4)])
    with pytest.raises(TypeError):
        S.GradClip([torch.zeros(4, dtype=torch.float16)])
    with pytest.raises(ValueError):
        S.GradClip([torch.zeros(4)], out=[])
    with pytest.raises(TypeError):
        S.GradClip([torch.zeros(4, dtype=torch.bfloat16)], out=[torch.zeros(4)])


def _gate(experts=8, top_k=2, groups=1, top_groups=1, group_top=1, score=0, scale=1.0, flags=S.GATE_FP32):
    return S.GateConfig(experts, top_k, groups, top_groups, group_top, score, scale, flags)


def test_gate_struct_layout():
    assert _sizes(["sizeof(skew_gate_config_t)", "offsetof(skew_gate_config_t, scale)", "offsetof(skew_gate_config_t, flags)"]) == \
        [C.sizeof(S.GateConfig), S.GateConfig.scale.offset, S.GateConfig.flags.offset]


@pytest.mark.parametrize("kw,what", [
    (dict(experts=0), "experts"), (dict(experts=513), "experts"), (dict(experts=8, groups=3), "groups"), (dict(experts=66, groups=33), "groups"),
    (dict(groups=0), "groups"), (dict(groups=2, top_groups=3), "top_groups"), (dict(top_groups=0), "top_groups"),
    (dict(group_top=3), "group_top"), (dict(group_top=0), "group_top"), (dict(top_k=0), "top_k"), (dict(top_k=9), "top_k"),
    (dict(experts=64, top_k=33), "top_k"), (dict(groups=4, top_groups=1, top_k=3), "top_k"), (dict(score=2), "score"),
    (dict(flags=4), "flags"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale")])
def test_gate_refuses_configs(kw, what):
    c = _gate(**kw)
    assert S.skew_gate_workspace_bytes(c) == 0 and what in S.skew_ops_last_error()
    _refused(S.SKEW_EINVAL, what, S.skew_gate_forward, c, 0x1000, 8, 0, 4, 0x1000, 0x1000, 0x1000, 0x1000, 4096, 0)
    _refused(S.SKEW_EINVAL, what, S.skew_gate_grad, c, 0x1000, 8, 0x1000, 0x1000, 4, 0x1000, 8, 0)


@pytest.mark.parametrize("at,value,what", [
    (0, 0, "logits"), (0, 0x1002, "logits"), (1, 7, "stride"), (1, (1 << 31) + 1, "stride"), (2, 0x1002, "bias"), (3, -1, "tokens"), (3, 1 << 31, "tokens"),
    (4, 0, "chosen"), (5, 0x1001, "chosen"), (6, 0x1002, "workspace"), (7, 0, "workspace"), (8, 35, "workspace")])
def test_gate_forward_refuses(at, value, what):
    a = [0x1000, 8, 0, 4, 0x1000, 0x1000, 0x1000, 0x1000, 36]
    a[at] = value
    _refused(S.SKEW_EINVAL, what, S.skew_gate_forward, _gate(), *a, 0)


@pytest.mark.parametrize("at,value,what", [
    (0, 0, "logits"), (1, 7, "logits"), (2, 0, "chosen"), (3, 0x1002, "chosen"), (4, -1, "tokens"), (5, 0, "dlogits"), (5, 0x1002, "dlogits"), (6, 7, "dlogits")])
def test_gate_grad_refuses(at, value, what):
    a = [0x1000, 8, 0x1000, 0x1000, 4, 0x1000, 8]
    a[at] = value
    _refused(S.SKEW_EINVAL, what, S.skew_gate_grad, _gate(), *a, 0)


def test_router_refuses():
    import torch
    with pytest.raises(ValueError):
        S.Router(8, 2, score="relu")
    with pytest.raises(S.SkewError):
        S.Router(8, 9)
    with pytest.raises(ValueError):
        S.Router(8, 2).route(torch.zeros((4, 8)))
    assert S.skew_gate_forward(_gate(), 0, 8, 0, 0, 0, 0, 0, 0, 0, 0) is None  # no tokens, no counts: nothing to do


def _embed(rows=100, width=16, scale=1.0, flags=0):
    return S.EmbedConfig(rows, width, scale, flags)


def test_embed_struct_layout():
    assert _sizes(["sizeof(skew_embed_config_t)", "offsetof(skew_embed_config_t, scale)", "offsetof(skew_embed_config_t, flags)"]) == \
        [C.sizeof(S.EmbedConfig), S.EmbedConfig.scale.offset, S.EmbedConfig.flags.offset]


@pytest.mark.parametrize("kw,what", [(dict(rows=0), "rows"), (dict(rows=1 << 31), "rows"), (dict(width=0), "width"), (dict(width=(1 << 20) + 1), "width"),
                                     (dict(scale=float("nan")), "scale"), (dict(flags=8), "flags")])
def test_embed_refuses_configs(kw, what):
    c = _embed(**kw)
    assert S.skew_embed_workspace_bytes(c, 4) == 0 and what in S.skew_ops_last_error()
    _refused(S.SKEW_EINVAL, what, S.skew_embed_lookup, c, 0x1000, 0x1000, 4, 0x1000, 16, 0)
    _refused(S.SKEW_EINVAL, what, S.skew_embed_grad, c, 0x1000, 4, 0x1000, 16, 0, 0x1000, 0x1000, 1 << 30, 0)


@pytest.mark.parametrize("at,value,what", [(0, 0, "table"), (0, 0x1001, "table"), (1, 0, "ids"), (1, 0x1002, "ids"), (2, -1, "tokens"), (2, 1 << 31, "tokens"),
                                           (3, 0, "out"), (3, 0x1001, "out"), (4, 15, "stride"), (4, (1 << 31) + 1, "stride")])
def test_embed_lookup_refuses(at, value, what):
    a = [0x1000, 0x1000, 4, 0x1000, 16]
    a[at] = value
    _refused(S.SKEW_EINVAL, what, S.skew_embed_lookup, _embed(), *a, 0)


@pytest.mark.parametrize("at,value,what", [(0, 0, "ids"), (0, 0x1002, "ids"), (1, -1, "tokens"), (2, 0, "dout"), (2, 0x1001, "dout"), (3, 15, "stride"),
                                           (4, 0x1001, "base"), (5, 0, "dtable"), (5, 0x1001, "dtable"), (6, 0, "workspace"), (6, 0x1010, "workspace"), (7, 1024, "workspace")])
def test_embed_grad_refuses(at, value, what):
    a = [0x1000, 4, 0x1000, 16, 0, 0x1000, 0x1000, 1 << 20]
    a[at] = value
    _refused(S.SKEW_EINVAL, what, S.skew_embed_grad, _embed(), *a, 0)


def test_embedding_refuses():
    import torch
    with pytest.raises(TypeError):
        S.Embedding(10, 8, torch.float16)
    with pytest.raises(S.SkewError):
        S.Embedding(0, 8)
    e = S.Embedding(10, 8)
    with pytest.raises(TypeError):
        e.lookup(torch.zeros((10, 8), dtype=torch.bfloat16), torch.zeros(3))
    with pytest.raises(ValueError):
        e.lookup(torch.zeros((10, 8), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64))


def test_clip_refuses_more_than_it_can_count():
    many = [S.ClipDesc(0x1000, 0, 1 << 40, S.CLIP_GRAD_FP32, 0)] * 17
    _refused(S.SKEW_EINVAL, "too many", S.skew_clip_create, many)


def test_embed_refuses_too_many_tokens():
    _refused(S.SKEW_EINVAL, "tokens", S.skew_embed_lookup, _embed(), 0x1000, 0x1000, (1 << 30) + 1, 0x1000, 16, 0)
    assert S.skew_embed_workspace_bytes(_embed(), 1 << 30) > 0
