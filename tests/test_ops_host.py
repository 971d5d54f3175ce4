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
