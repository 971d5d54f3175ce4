"""ctypes binding of libskewadam (include/skewadam.h).

Argument marshalling only: every step of the optimizer runs in the library's
CUDA kernels. PyTorch provides device memory (state and workspace buffers are
``torch.empty`` allocations) and the current CUDA stream. The functions keep the
C names; ``SkewAdam`` bundles create / bind / step for torch tensors.

If the library has not been built this module raises on first use; there is no
CPU fallback.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
import threading
from typing import Iterable, List, Optional, Sequence

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libskewadam.so")

SKEW_OK, SKEW_EINVAL, SKEW_ENOMEM, SKEW_ECUDA, SKEW_ETIMEOUT, SKEW_ESTATE, SKEW_ETOOBIG = 0, -1, -2, -3, -4, -5, -6
NOALLOC_SCRATCH_BYTES = 16 * 1024 * 1024
TIER_BACKBONE, TIER_EXPERT, TIER_ROUTER = 0, 1, 2
POLICY_TIERED, POLICY_EXPERT_MOMENTUM, POLICY_FACTORED_ROUTER, POLICY_UNIFORM, POLICY_ADAFACTOR = 0, 1, 2, 3, 4
F_NO_DECAY = 1
F_FP32 = 2
KIND_FULL, KIND_FACTORED = 0, 1
ROUTE_OWN, ROUTE_RIDING, ROUTE_ROWS, ROUTE_SMALL = 0, 1, 2, 3
CLIP_GRAD_FP32, CLIP_OUT_FP32 = 1, 2
GATE_SOFTMAX, GATE_SIGMOID = 0, 1
GATE_RENORM, GATE_FP32 = 1, 2
EMBED_TABLE_FP32, EMBED_ACT_FP32, EMBED_IDS_64 = 1, 2, 4

EXPORTS = ["skew_create", "skew_destroy", "skew_state_bytes", "skew_workspace_bytes", "skew_bind", "skew_step",
           "skew_sync_status", "skew_tensor_scalars", "skew_matrix_scalars", "skew_tensor_info", "skew_num_tensors", "skew_last_error",
           "skew_profile_begin", "skew_profile_end", "skew_kernel_name", "skew_step_tensor_noalloc",
           "skew_launches_per_step", "skew_selftest_wait_timeout", "skew_noalloc_sync_status", "skew_step_scaled",
           "skew_noalloc_selftest_wait_timeout", "skew_tensor_route", "skew_ops_last_error",
           "skew_clip_create", "skew_clip_destroy", "skew_clip_workspace_bytes", "skew_clip_bind", "skew_clip_norm",
           "skew_clip_apply", "skew_gate_workspace_bytes", "skew_gate_forward", "skew_gate_grad",
           "skew_embed_lookup", "skew_embed_workspace_bytes", "skew_embed_grad"]


class SkewError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libskewadam error {code}: {msg}")
        self.code = code


class ParamDesc(C.Structure):
    _fields_ = [("weight", C.c_void_p), ("grad", C.c_void_p), ("shape", C.c_int64 * 2), ("ndim", C.c_int32),
                ("tier", C.c_int32), ("flags", C.c_uint32), ("stack", C.c_uint32)]


class HParams(C.Structure):
    _fields_ = [("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float), ("clip_d", C.c_float),
                ("weight_decay", C.c_float), ("policy", C.c_int32)]


class TensorInfo(C.Structure):
    _fields_ = [("kind", C.c_int32), ("momentum", C.c_int32), ("decay", C.c_int32), ("vectorized", C.c_int32),
                ("rows", C.c_int64), ("cols", C.c_int64), ("numel", C.c_int64), ("m_offset", C.c_int64),
                ("v_offset", C.c_int64), ("r_offset", C.c_int64), ("c_offset", C.c_int64), ("rowpath", C.c_int32),
                ("stack", C.c_int32)]


class ClipDesc(C.Structure):
    _fields_ = [("grad", C.c_void_p), ("out", C.c_void_p), ("numel", C.c_int64), ("flags", C.c_uint32),
                ("zero", C.c_uint32)]


class GateConfig(C.Structure):
    _fields_ = [("experts", C.c_int32), ("top_k", C.c_int32), ("groups", C.c_int32), ("top_groups", C.c_int32),
                ("group_top", C.c_int32), ("score", C.c_int32), ("scale", C.c_float), ("flags", C.c_uint32)]


class EmbedConfig(C.Structure):
    _fields_ = [("rows", C.c_int64), ("width", C.c_int64), ("scale", C.c_float), ("flags", C.c_uint32)]


_lock = threading.Lock()
_lib = None


def load(path: Optional[str] = None) -> C.CDLL:
    """Loads libskewadam.so (built by ``__graft_entry__.build()``); raises if absent."""
    global _lib
    with _lock:
        if _lib is not None and path is None:
            return _lib
        p = path or LIB_PATH
        if not os.path.exists(p):
            raise RuntimeError(f"{p} is missing: build it with __graft_entry__.build() "
                               "(no CPU fallback exists)")
        L = C.CDLL(p)
        vp, i32, i64, u64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_size_t
        L.skew_create.argtypes = [C.POINTER(ParamDesc), i32, C.POINTER(HParams), C.POINTER(vp)]
        L.skew_create.restype = C.c_int
        L.skew_destroy.argtypes = [vp]
        L.skew_destroy.restype = C.c_int
        L.skew_state_bytes.argtypes = [vp]
        L.skew_state_bytes.restype = sz
        L.skew_workspace_bytes.argtypes = [vp]
        L.skew_workspace_bytes.restype = sz
        L.skew_bind.argtypes = [vp, vp, sz, vp, sz, vp]
        L.skew_bind.restype = C.c_int
        L.skew_step.argtypes = [vp, i64, C.c_float, u64, vp]
        L.skew_step.restype = C.c_int
        L.skew_step_scaled.argtypes = [vp, i64, C.c_float, u64, vp, vp]
        L.skew_step_scaled.restype = C.c_int
        L.skew_sync_status.argtypes = [vp, vp]
        L.skew_sync_status.restype = C.c_int
        L.skew_selftest_wait_timeout.argtypes = [vp, vp]
        L.skew_selftest_wait_timeout.restype = C.c_int
        L.skew_tensor_scalars.argtypes = [vp, i32, C.POINTER(C.c_double), vp]
        L.skew_tensor_scalars.restype = C.c_int
        L.skew_matrix_scalars.argtypes = [vp, i32, i32, C.POINTER(C.c_double), vp]
        L.skew_matrix_scalars.restype = C.c_int
        L.skew_tensor_info.argtypes = [vp, i32, C.POINTER(TensorInfo)]
        L.skew_tensor_info.restype = C.c_int
        L.skew_tensor_route.argtypes = [vp, i32]
        L.skew_tensor_route.restype = C.c_int
        L.skew_launches_per_step.argtypes = [vp]
        L.skew_launches_per_step.restype = i64
        L.skew_num_tensors.argtypes = [vp]
        L.skew_num_tensors.restype = i32
        L.skew_last_error.argtypes = [vp]
        L.skew_last_error.restype = C.c_char_p
        L.skew_profile_begin.argtypes = [vp, i32]
        L.skew_profile_begin.restype = C.c_int
        L.skew_profile_end.argtypes = [vp, C.POINTER(C.c_double), i64, C.POINTER(i32), C.POINTER(i32)]
        L.skew_profile_end.restype = C.c_int
        L.skew_kernel_name.argtypes = [i32]
        L.skew_kernel_name.restype = C.c_char_p
        L.skew_step_tensor_noalloc.argtypes = [vp, vp, i32, i64, i64, i32, C.c_uint32, C.POINTER(HParams), vp, sz,
                                               C.c_uint32, i64, C.c_float, u64, vp]
        L.skew_step_tensor_noalloc.restype = C.c_int
        L.skew_noalloc_sync_status.argtypes = [vp]
        L.skew_noalloc_sync_status.restype = C.c_int
        L.skew_noalloc_selftest_wait_timeout.argtypes = [vp]
        L.skew_noalloc_selftest_wait_timeout.restype = C.c_int
        L.skew_ops_last_error.argtypes = []
        L.skew_ops_last_error.restype = C.c_char_p
        L.skew_clip_create.argtypes = [C.POINTER(ClipDesc), i32, C.POINTER(vp)]
        L.skew_clip_create.restype = C.c_int
        L.skew_clip_destroy.argtypes = [vp]
        L.skew_clip_destroy.restype = C.c_int
        L.skew_clip_workspace_bytes.argtypes = [vp]
        L.skew_clip_workspace_bytes.restype = sz
        L.skew_clip_bind.argtypes = [vp, vp, sz, vp]
        L.skew_clip_bind.restype = C.c_int
        for f in (L.skew_clip_norm, L.skew_clip_apply):
            f.argtypes = [vp, C.c_float, vp, vp]
            f.restype = C.c_int
        L.skew_gate_workspace_bytes.argtypes = [C.POINTER(GateConfig)]
        L.skew_gate_workspace_bytes.restype = sz
        L.skew_gate_forward.argtypes = [C.POINTER(GateConfig), vp, i64, vp, i64, vp, vp, vp, vp, sz, vp]
        L.skew_gate_forward.restype = C.c_int
        L.skew_gate_grad.argtypes = [C.POINTER(GateConfig), vp, i64, vp, vp, i64, vp, i64, vp]
        L.skew_gate_grad.restype = C.c_int
        L.skew_embed_lookup.argtypes = [C.POINTER(EmbedConfig), vp, vp, i64, vp, i64, vp]
        L.skew_embed_lookup.restype = C.c_int
        L.skew_embed_workspace_bytes.argtypes = [C.POINTER(EmbedConfig), i64]
        L.skew_embed_workspace_bytes.restype = sz
        L.skew_embed_grad.argtypes = [C.POINTER(EmbedConfig), vp, i64, vp, i64, vp, vp, vp, sz, vp]
        L.skew_embed_grad.restype = C.c_int
        if path is None:
            _lib = L
        return L


def _check(rc: int, h=None):
    if rc != SKEW_OK:
        msg = load().skew_last_error(h)
        raise SkewError(rc, msg.decode() if msg else "")


def _check_op(rc: int):
    if rc != SKEW_OK:
        raise SkewError(rc, skew_ops_last_error())


# --------------------------------------------------------------------------
# C entry points, same names
# --------------------------------------------------------------------------
def skew_create(params: Sequence[ParamDesc], hp: HParams) -> C.c_void_p:
    arr = (ParamDesc * max(1, len(params)))(*params)
    h = C.c_void_p()
    _check(load().skew_create(arr, len(params), C.byref(hp), C.byref(h)))
    return h


def skew_destroy(h) -> None:
    load().skew_destroy(h)


def skew_state_bytes(h) -> int:
    return int(load().skew_state_bytes(h))


def skew_workspace_bytes(h) -> int:
    return int(load().skew_workspace_bytes(h))


def skew_bind(h, state_ptr: int, state_bytes: int, ws_ptr: int, ws_bytes: int, stream: int) -> None:
    _check(load().skew_bind(h, state_ptr, state_bytes, ws_ptr, ws_bytes, stream), h)


def skew_step(h, step: int, lr: float, seed: int, stream: int) -> None:
    _check(load().skew_step(h, step, lr, seed & (2**64 - 1), stream), h)


def skew_step_scaled(h, step: int, lr: float, seed: int, grad_scale_ptr: int, stream: int) -> None:
    """skew_step on gamma * G, gamma read by the kernels from the device pointer (0: gamma = 1)."""
    _check(load().skew_step_scaled(h, step, lr, seed & (2**64 - 1), grad_scale_ptr or None, stream), h)


def skew_sync_status(h, stream: int) -> None:
    _check(load().skew_sync_status(h, stream), h)


def skew_selftest_wait_timeout(h, stream: int) -> None:
    _check(load().skew_selftest_wait_timeout(h, stream), h)


def skew_tensor_scalars(h, tid: int, stream: int):
    out = (C.c_double * 4)()
    _check(load().skew_tensor_scalars(h, tid, out, stream), h)
    return {"rbar": out[0], "sumu2": out[1], "rms": out[2], "kappa": out[3]}


def skew_matrix_scalars(h, tid: int, e: int, stream: int):
    out = (C.c_double * 4)()
    _check(load().skew_matrix_scalars(h, tid, e, out, stream), h)
    return {"rbar": out[0], "sumu2": out[1], "rms": out[2], "kappa": out[3]}


def skew_tensor_info(h, tid: int) -> TensorInfo:
    info = TensorInfo()
    _check(load().skew_tensor_info(h, tid, C.byref(info)), h)
    return info


def skew_tensor_route(h, tid: int) -> int:
    """ROUTE_*: which launches step the tensor."""
    r = load().skew_tensor_route(h, tid)
    if r < 0:
        raise SkewError(r, f"tensor {tid} out of range")
    return r


def skew_launches_per_step(h) -> int:
    return int(load().skew_launches_per_step(h))


def skew_num_tensors(h) -> int:
    return int(load().skew_num_tensors(h))


def skew_last_error(h=None) -> str:
    m = load().skew_last_error(h)
    return m.decode() if m else ""


def skew_profile_begin(h, max_steps: int) -> None:
    _check(load().skew_profile_begin(h, max_steps), h)


def skew_profile_end(h, cap: int = 1 << 16):
    """-> (kernel names, list of per-step lists of per-kernel milliseconds)."""
    buf = (C.c_double * cap)()
    ns, nk = C.c_int32(), C.c_int32()
    _check(load().skew_profile_end(h, buf, cap, C.byref(ns), C.byref(nk)), h)
    names = [skew_kernel_name(k) for k in range(nk.value)]
    rows = [[buf[s * nk.value + k] for k in range(nk.value)] for s in range(ns.value) if (s + 1) * nk.value <= cap]
    return names, rows


def skew_kernel_name(k: int) -> str:
    m = load().skew_kernel_name(k)
    return m.decode() if m else ""


def skew_step_tensor_noalloc(weight_ptr: int, grad_ptr: int, ndim: int, rows: int, cols: int, tier: int, flags: int,
                             hp: HParams, state_ptr: int, state_bytes: int, tensor_id: int, step: int, lr: float,
                             seed: int, stream: int) -> None:
    """One tensor's step with the library's fixed scratch array (no allocation of any kind)."""
    rc = load().skew_step_tensor_noalloc(weight_ptr, grad_ptr, ndim, rows, cols, tier, flags, C.byref(hp), state_ptr,
                                         state_bytes, tensor_id, step, lr, seed & (2**64 - 1), stream)
    if rc != SKEW_OK:
        why = {SKEW_EINVAL: "invalid argument or state size", SKEW_ECUDA: "CUDA error",
               SKEW_ETOOBIG: f"tensor needs more than the {NOALLOC_SCRATCH_BYTES} bytes of fixed scratch"}
        raise SkewError(rc, why.get(rc, "error"))


def skew_noalloc_sync_status(stream: int) -> None:
    """Synchronises `stream`; raises SkewError(SKEW_ETIMEOUT) once if a bounded device wait of a
    no-alloc call gave up since the last read (the status word is then cleared)."""
    rc = load().skew_noalloc_sync_status(stream)
    if rc != SKEW_OK:
        why = {SKEW_ETIMEOUT: "a bounded device wait of a no-alloc step gave up", SKEW_ECUDA: "CUDA error"}
        raise SkewError(rc, why.get(rc, "error"))


def skew_noalloc_selftest_wait_timeout(stream: int) -> None:
    """Makes one bounded device wait run out against the no-alloc status word."""
    rc = load().skew_noalloc_selftest_wait_timeout(stream)
    if rc != SKEW_OK:
        raise SkewError(rc, "CUDA error")


def skew_ops_last_error() -> str:
    m = load().skew_ops_last_error()
    return m.decode() if m else ""


def skew_clip_create(tensors: Sequence[ClipDesc]) -> C.c_void_p:
    arr = (ClipDesc * max(1, len(tensors)))(*tensors)
    h = C.c_void_p()
    _check_op(load().skew_clip_create(arr, len(tensors), C.byref(h)))
    return h


def skew_clip_destroy(h) -> None:
    load().skew_clip_destroy(h)


def skew_clip_workspace_bytes(h) -> int:
    return int(load().skew_clip_workspace_bytes(h))


def skew_clip_bind(h, ws_ptr: int, ws_bytes: int, stream: int) -> None:
    _check_op(load().skew_clip_bind(h, ws_ptr, ws_bytes, stream))


def skew_clip_norm(h, max_norm: float, result_ptr: int, stream: int) -> None:
    _check_op(load().skew_clip_norm(h, max_norm, result_ptr, stream))


def skew_clip_apply(h, max_norm: float, result_ptr: int, stream: int) -> None:
    _check_op(load().skew_clip_apply(h, max_norm, result_ptr, stream))


def skew_gate_workspace_bytes(c: GateConfig) -> int:
    return int(load().skew_gate_workspace_bytes(C.byref(c)))


def skew_gate_forward(c: GateConfig, logits_ptr: int, ld: int, bias_ptr: int, tokens: int, chosen_ptr: int,
                      weights_ptr: int, counts_ptr: int, ws_ptr: int, ws_bytes: int, stream: int) -> None:
    """`bias_ptr`, `counts_ptr`: 0 for none."""
    _check_op(load().skew_gate_forward(C.byref(c), logits_ptr, ld, bias_ptr or None, tokens, chosen_ptr, weights_ptr,
                                       counts_ptr or None, ws_ptr, ws_bytes, stream))


def skew_gate_grad(c: GateConfig, logits_ptr: int, ld: int, chosen_ptr: int, dweights_ptr: int, tokens: int,
                   dlogits_ptr: int, ld_out: int, stream: int) -> None:
    _check_op(load().skew_gate_grad(C.byref(c), logits_ptr, ld, chosen_ptr, dweights_ptr, tokens, dlogits_ptr, ld_out,
                                    stream))


def skew_embed_lookup(c: EmbedConfig, table_ptr: int, ids_ptr: int, tokens: int, out_ptr: int, ld_out: int,
                      stream: int) -> None:
    _check_op(load().skew_embed_lookup(C.byref(c), table_ptr, ids_ptr, tokens, out_ptr, ld_out, stream))


def skew_embed_workspace_bytes(c: EmbedConfig, tokens: int) -> int:
    return int(load().skew_embed_workspace_bytes(C.byref(c), tokens))


def skew_embed_grad(c: EmbedConfig, ids_ptr: int, tokens: int, dout_ptr: int, ld_dout: int, base_ptr: int,
                    dtable_ptr: int, ws_ptr: int, ws_bytes: int, stream: int) -> None:
    """`base_ptr`: 0 for none."""
    _check_op(load().skew_embed_grad(C.byref(c), ids_ptr, tokens, dout_ptr, ld_dout, base_ptr or None, dtable_ptr,
                                     ws_ptr, ws_bytes, stream))


def hparams(beta1=0.9, beta2=0.999, eps=1e-8, clip_d=1.0, weight_decay=0.05, policy=POLICY_TIERED) -> HParams:
    return HParams(beta1, beta2, eps, clip_d, weight_decay, policy)


# --------------------------------------------------------------------------
# torch convenience wrappers
# --------------------------------------------------------------------------
def _stream_of(stream, device) -> int:
    """The raw handle of a stream; None: of the current one of a tensor's device."""
    if stream is None:
        return _raw_stream()(device.index)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _on(stream):
    """A context in which a stream (or its raw handle) is torch's current one."""
    import torch
    return torch.cuda.stream(stream if hasattr(stream, "cuda_stream") else torch.cuda.ExternalStream(int(stream)))


_current = None


def _raw_stream():
    """A function from a device's index to the raw handle of its current stream."""
    global _current
    if _current is None:
        import torch
        _current = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # 0.1 us; the public call takes 2 to 3
        if _current is None:
            _current = lambda index: torch.cuda.current_stream(index).cuda_stream  # noqa: E731
    return _current


_fresh = None


def _allocator():
    """A function (shape, strides, dtype, device) -> a new tensor. Beside a kernel launch torch.empty costs 2.6 us a
    tensor, most of these operators' time on small inputs; the call behind compiled torch programs costs 1.2, for the current device."""
    global _fresh
    if _fresh is None:
        import torch
        quick = getattr(getattr(getattr(torch._C, "_dynamo", None), "guards", None), "_empty_strided_cuda", None)
        if quick is not None and torch.cuda.device_count() == 1:
            _fresh = lambda shape, strides, dtype, device: quick(shape, strides, dtype)  # noqa: E731
        else:
            _fresh = lambda shape, strides, dtype, device: torch.empty_strided(shape, strides, dtype=dtype, device=device)  # noqa: E731
    return _fresh


def _device_check():
    """A function that refuses tensors on a device other than the current one, where the library launches;
    None where there is no other."""
    import torch
    if torch.cuda.device_count() < 2:
        return None
    current = torch.cuda.current_device

    def check(dev):
        if dev.index != current():
            raise ValueError(f"the tensors are on {dev}, the current device is cuda:{current()}")
    return check


class _Block:
    """Device memory that an object keeps between calls, and the raw handles of the streams that may use it: the one it was
    allocated on and those of ``also_on``."""

    __slots__ = ("tensor", "ptr", "bytes", "streams")

    def __init__(self, tensor, handle: int):
        self.tensor, self.ptr, self.bytes, self.streams = tensor, tensor.data_ptr(), tensor.numel(), {handle}

    def also_on(self, handle: int):
        """Work on the current stream, of this handle, uses it: once it is dropped, its memory goes to nobody else before that
        is done. The allocator asks the stream at that time, so one that torch did not make, and that may be gone, is left out."""
        import torch
        stream = torch.cuda.current_stream(self.tensor.device)
        if not handle or stream.stream_id != handle:  # (the id of a stream from elsewhere is its handle)
            self.tensor.record_stream(stream)
        self.streams.add(handle)


class GradClip:
    """The global norm of many gradients, its clip factor, and clipping.

    ``grads``: contiguous bf16 or fp32 CUDA tensors of any shapes, on the current device. ``out``: where ``clip`` writes
    the clipped gradients, one tensor for each: of the gradient's type, or bf16 for an fp32 one
    (microbatches accumulated in fp32, handed to the step in bf16). ``None``: in place.

    ``norm`` and ``clip`` return ``result``, a device tensor [norm, gamma] that the next call
    overwrites; ``gamma`` is the view of its second element that ``SkewAdam.step`` takes as
    ``grad_scale``. The tensors are borrowed: they must live, and stay where they are, as long as this object: across steps,
    as with ``zero_grad(set_to_none=False)`` (a new object costs some 0.2 ms and waits for its stream); and it
    as long as a graph that captured its calls, or work that it was given on a stream torch did not make (a raw handle).
    """

    def __init__(self, grads: Iterable, out: Optional[Iterable] = None, stream=None):
        import torch
        grads = list(grads)
        outs = grads if out is None else list(out)
        if len(outs) != len(grads):
            raise ValueError("out must have one tensor for each gradient")
        f32, kinds = torch.float32, {torch.bfloat16: 0, torch.float32: CLIP_GRAD_FP32}
        first = grads[0].device if grads else None
        descs = (ClipDesc * max(1, len(grads)))()
        for d, g, o in zip(descs, grads, outs):
            flags = kinds.get(g.dtype)
            if flags is None or o.dtype not in kinds:
                raise TypeError("gradients must be bf16 or fp32")
            if o.dtype == f32:
                if not flags:
                    raise TypeError("a bf16 gradient is clipped to bf16")
                flags |= CLIP_OUT_FP32
            if not (g.is_cuda and g.is_contiguous()):
                raise ValueError("gradients must be contiguous CUDA tensors")
            if g.device != first:
                raise ValueError("all tensors must be on one device")
            d.grad = p = g.data_ptr()
            if o is not g:
                if not (o.is_contiguous() and g.shape == o.shape and o.device == first):
                    raise ValueError("out must be contiguous CUDA tensors of the gradients' shapes, on their device")
                p = o.data_ptr()
            d.out, d.numel, d.flags = p, g.numel(), flags
        self._elsewhere = _device_check()
        if grads and self._elsewhere:
            self._elsewhere(first)
        self.grads, self.out = grads, outs
        self.h = C.c_void_p()
        _check_op(load().skew_clip_create(descs, len(grads), C.byref(self.h)))
        dev = grads[0].device if grads else torch.device("cuda")
        n = skew_clip_workspace_bytes(self.h)
        with contextlib.nullcontext() if stream is None else _on(stream):  # the stream that fills them: no other's work comes between
            self.workspace = torch.empty(n, dtype=torch.uint8, device=dev)
            self.result = torch.zeros(2, dtype=torch.float32, device=dev)
        self.gamma = self.result[1:]
        self._device = self.result.device
        self._norm, self._apply, self._stream = load().skew_clip_norm, load().skew_clip_apply, _raw_stream()
        self._index = self._device.index
        handle = _stream_of(stream, self._device)
        self._blocks = _Block(self.workspace, handle), _Block(self.result, handle)
        self._result, self._streams = self._blocks[1].ptr, self._blocks[1].streams
        skew_clip_bind(self.h, self._blocks[0].ptr, n, handle)

    def _handle(self, stream) -> int:
        handle = self._stream(self._index) if stream is None else _stream_of(stream, None)
        if handle not in self._streams:
            with contextlib.nullcontext() if stream is None else _on(stream):
                for b in self._blocks:
                    b.also_on(handle)
        return handle

    def norm(self, max_norm: float, stream=None):
        """[norm, gamma] with gamma = min(1, max_norm / (norm + 1e-6)); the gradients are only read."""
        if self._elsewhere:
            self._elsewhere(self._device)
        rc = self._norm(self.h, max_norm, self._result, self._handle(stream))
        if rc:
            _check_op(rc)
        return self.result

    def clip(self, max_norm: float, stream=None):
        """``norm``, then out = gamma * g for every tensor."""
        if self._elsewhere:
            self._elsewhere(self._device)
        rc = self._apply(self.h, max_norm, self._result, self._handle(stream))
        if rc:
            _check_op(rc)
        return self.result

    def close(self):
        if getattr(self, "h", None):
            skew_clip_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Embedding:
    """Lookup of a (rows, width) table by token ids, scaled, and the table's gradient, which is a call of its
    own: for autograd a looked-up tensor is a leaf, whether the table requires a gradient or not.

    ``table_dtype`` (of the table and its gradient) and ``act_dtype`` (of the looked-up rows and their
    gradient) are bf16 or fp32. Ids are int32 or int64, of any shape; one outside [0, rows) is padding: its
    row is zero and it has no gradient. Tensors are to be on the current device. The object must live as long as a graph that
    captured its calls, or work that it was given on a stream torch did not make (a raw handle).
    """

    def __init__(self, rows: int, width: int, table_dtype=None, act_dtype=None, scale: float = 1.0):
        import torch
        self.table_dtype, self.act_dtype = table_dtype or torch.bfloat16, act_dtype or torch.bfloat16
        if not {self.table_dtype, self.act_dtype} <= {torch.bfloat16, torch.float32}:
            raise TypeError("table and activations must be bf16 or fp32")
        self.rows, self.width = rows, width
        flags = (EMBED_TABLE_FP32 if self.table_dtype == torch.float32 else 0) | \
                (EMBED_ACT_FP32 if self.act_dtype == torch.float32 else 0)
        self.config = {torch.int32: EmbedConfig(rows, width, scale, flags),
                       torch.int64: EmbedConfig(rows, width, scale, flags | EMBED_IDS_64)}
        if not skew_embed_workspace_bytes(self.config[torch.int32], 0):
            raise SkewError(SKEW_EINVAL, skew_ops_last_error())
        self._ref = {dt: C.byref(c) for dt, c in self.config.items()}
        self._shape = (rows, width)
        self._new, self._lookup, self._grad = _allocator(), load().skew_embed_lookup, load().skew_embed_grad
        self._stream, self._elsewhere = _raw_stream(), _device_check()
        self._workspaces, self._sizes, self._kept = {}, {}, []  # the first: by device

    def _ids(self, ids):
        c = self._ref.get(ids.dtype)
        if c is None:
            raise TypeError("ids must be int32 or int64")
        if not (ids.is_cuda and ids.is_contiguous()):
            raise ValueError("ids must be a contiguous CUDA tensor")
        if self._elsewhere:
            self._elsewhere(ids.device)
        return c

    def _table(self, t, dev, what: str):
        if not (t.dtype == self.table_dtype and t.shape == self._shape and t.is_contiguous() and t.device == dev):
            raise ValueError(f"{what} must be a contiguous {self._shape} {self.table_dtype} tensor on the ids' device")
        return t.data_ptr()

    def lookup(self, table, ids, stream=None):
        """scale * table[ids], of shape ids.shape + (width,). With ``stream`` the result belongs to that stream."""
        if stream is not None:
            with _on(stream):
                return self.lookup(table, ids)
        c, dev = self._ids(ids), ids.device
        p = self._table(table, dev, "table")
        n, d = ids.numel(), self.width
        out = self._new((n, d), (d, 1), self.act_dtype, dev)
        rc = self._lookup(c, p, ids.data_ptr(), n, out.data_ptr(), d, self._stream(dev.index))
        if rc:
            _check_op(rc)
        return out if ids.dim() == 1 else out.view(*ids.shape, d)

    def grad(self, ids, dy, base=None, out=None, stream=None):
        """The table's gradient, every row of it, from the looked-up rows' (``ids.shape + (width,)``; a 2-D one may
        have rows apart). ``base``: what it adds to; ``out``: where it goes (``base`` itself: in place, and rows
        without tokens are not touched; None: a new tensor). Calls on one object share a
        workspace: they must not overlap on the GPU."""
        if stream is not None:
            with _on(stream):
                return self.grad(ids, dy, base, out)
        c, dev, n = self._ids(ids), ids.device, ids.numel()
        if dy.dtype != self.act_dtype or dy.shape != (*ids.shape, self.width) or dy.device != dev:
            raise ValueError(f"dy must be a {(*ids.shape, self.width)} {self.act_dtype} tensor on the ids' device")
        ld = self.width if dy.is_contiguous() else _rows(dy, self.width, "dy that is not contiguous")
        b = None if base is None else self._table(base, dev, "base")
        if out is None:
            out = self._new(self._shape, (self.width, 1), self.table_dtype, dev)
            p = out.data_ptr()
        else:
            p = self._table(out, dev, "out")
        ws, handle = self._workspaces.get(dev.index), self._stream(dev.index)
        need = self._sizes.get(n)
        if need is None:
            need = self._sizes[n] = skew_embed_workspace_bytes(self.config[ids.dtype], n)
        if ws is None or ws.bytes < need:
            import torch
            if ws is not None:
                self._kept.append(ws)  # a graph, or work on another stream, may still use it
                need = max(need, 3 * ws.bytes // 2)
            ws = self._workspaces[dev.index] = _Block(torch.empty(need, dtype=torch.uint8, device=dev), handle)
        elif handle not in ws.streams:
            ws.also_on(handle)
        rc = self._grad(c, ids.data_ptr(), n, dy.data_ptr(), ld, b, p, ws.ptr, need, handle)
        if rc:
            _check_op(rc)
        return out


def _rows(t, width: int, what: str) -> int:
    """The row stride of a 2-D CUDA tensor whose rows are contiguous."""
    if not t.is_cuda or t.dim() != 2 or t.shape[1] != width or (width > 1 and t.stride(1) != 1):
        raise ValueError(f"{what} must be a 2-D CUDA tensor of {width} columns, contiguous within a row")
    return t.stride(0) if t.shape[0] > 1 else max(width, t.stride(0))


class Router:
    """Routing of tokens to experts (the gate of an MoE layer) and its gradient, which is a call of its own (no
    autograd function: the weights are a leaf).

    ``score``: "softmax" or "sigmoid"; ``renorm``: weights divided by their sum over the chosen;
    ``groups``, ``top_groups``, ``group_top``: experts are first narrowed to the best groups, each by its
    best one or the sum of its best two choices; ``scale``: a factor on the weights. See
    ``skew_gate_forward`` in the header for the definition, masked experts and ties. Tensors are to be on the current device. The
    object must live as long as a graph that captured its calls, or work that it was given on a stream torch did not make (a raw handle).
    """

    def __init__(self, experts: int, top_k: int, score: str = "softmax", renorm: bool = True, groups: int = 1,
                 top_groups: int = 1, group_top: int = 1, scale: float = 1.0):
        import torch
        kinds = {"softmax": GATE_SOFTMAX, "sigmoid": GATE_SIGMOID}
        if score not in kinds:
            raise ValueError("score must be 'softmax' or 'sigmoid'")
        if not all(-2**31 <= v < 2**31 for v in (experts, top_k, groups, top_groups, group_top)):  # (a C field would keep the low bits)
            raise ValueError("experts, top_k, groups, top_groups and group_top must fit 32 bits")
        self.experts, self.top_k = experts, top_k
        flags = GATE_RENORM if renorm else 0
        make = lambda f: GateConfig(experts, top_k, groups, top_groups, group_top, kinds[score], scale, f)  # noqa: E731
        self.config = {torch.bfloat16: make(flags), torch.float32: make(flags | GATE_FP32)}
        self._ws_bytes = skew_gate_workspace_bytes(self.config[torch.float32])
        if not self._ws_bytes:
            raise SkewError(SKEW_EINVAL, skew_ops_last_error())
        self._ref = {dt: C.byref(c) for dt, c in self.config.items()}
        self._new, self._i32, self._f32 = _allocator(), torch.int32, torch.float32
        self._forward, self._grad, self._stream = load().skew_gate_forward, load().skew_gate_grad, _raw_stream()
        self._elsewhere = _device_check()
        self._workspaces = {}  # by device

    def _logits(self, logits):
        c = self._ref.get(logits.dtype)
        if c is None:
            raise TypeError("logits must be bf16 or fp32")
        T, E = logits.shape if logits.dim() == 2 else (0, 0)
        if not (E == self.experts and logits.is_cuda and logits.is_contiguous()):
            E = _rows(logits, self.experts, "logits")
        if self._elsewhere:
            self._elsewhere(logits.device)
        return c, E, T, logits.device

    def route(self, logits, bias=None, stream=None):
        """(chosen int32 (T, k), weights fp32 (T, k), counts int32 (experts,)) of (T, experts) logits, whose rows
        may lie apart. ``bias``: fp32 (experts,), added to the scores for the choice alone. Calls on one
        object share a workspace: they must not overlap on the GPU. With ``stream`` the results belong to that stream."""
        if stream is not None:
            with _on(stream):
                return self.route(logits, bias)
        c, ld, T, dev = self._logits(logits)
        k, new, ws, handle = self.top_k, self._new, self._workspaces.get(dev.index), self._stream(dev.index)
        if bias is not None:
            if not (bias.dtype == self._f32 and bias.shape == (self.experts,) and bias.is_contiguous() and bias.device == dev):
                raise ValueError("bias must be a contiguous fp32 tensor of one value for each expert, on the logits' device")
            bias = bias.data_ptr()
        if ws is None:
            import torch
            if torch.cuda.is_current_stream_capturing():  # the zeros would be the graph's, and not there before it runs
                raise SkewError(SKEW_ESTATE, "a Router's first call cannot be captured")
            ws = self._workspaces[dev.index] = _Block(torch.zeros(self._ws_bytes, dtype=torch.uint8, device=dev), handle)
        elif handle not in ws.streams:
            ws.also_on(handle)
        chosen = new((T, k), (k, 1), self._i32, dev)
        weights = new((T, k), (k, 1), self._f32, dev)
        counts = new((self.experts,), (1,), self._i32, dev)
        rc = self._forward(c, logits.data_ptr(), ld, bias, T, chosen.data_ptr(), weights.data_ptr(), counts.data_ptr(),
                           ws.ptr, self._ws_bytes, handle)
        if rc:
            _check_op(rc)
        return chosen, weights, counts

    def grad(self, logits, chosen, dweights, stream=None):
        """The logits' gradient, (T, experts) of their type, from the weights' gradient (T, k) fp32."""
        if stream is not None:
            with _on(stream):
                return self.grad(logits, chosen, dweights)
        c, ld, T, dev = self._logits(logits)
        for t, dt in ((chosen, self._i32), (dweights, self._f32)):
            if not (t.dtype == dt and t.shape == (T, self.top_k) and t.is_contiguous() and t.device == dev):
                raise ValueError(f"chosen and dweights must be contiguous ({T}, {self.top_k}) int32 and fp32 tensors on the logits' device")
        dlogits = self._new((T, self.experts), (self.experts, 1), logits.dtype, dev)
        rc = self._grad(c, logits.data_ptr(), ld, chosen.data_ptr(), dweights.data_ptr(), T, dlogits.data_ptr(),
                        self.experts, self._stream(dev.index))
        if rc:
            _check_op(rc)
        return dlogits


class SkewAdam:
    """SkewAdam over a list of (weight, grad, tier[, flags]) CUDA tensors, bf16 or fp32
    (an fp32 pair, as the paper keeps the norms and the router, is stepped in fp32
    with no dithered cast; F_FP32 is set for it).

    A 3-D tensor (E, n, m) is a stack of E matrices (e.g. an MoE layer's experts
    kept in one array), each stepped with its own second-moment factors and clip
    factor. The optimizer state is one device buffer of exactly ``state_bytes``
    bytes (the paper's closed form); the workspace holds scratch and tables. Tensors are to be
    on the current device, and to stay where they are as long as this object.
    """

    def __init__(self, params: Iterable, hp: HParams, stream=None):
        import torch
        self.torch = torch
        self.params = []
        descs: List[ParamDesc] = []
        for p in params:
            w, g, tier = p[0], p[1], p[2]
            flags = p[3] if len(p) > 3 else 0
            if w.dtype != g.dtype or w.dtype not in (torch.bfloat16, torch.float32):
                raise TypeError("weights and gradients must both be bf16 or both fp32")
            if w.dtype == torch.float32:
                flags |= F_FP32
            if not (w.is_cuda and g.is_cuda and w.is_contiguous() and g.is_contiguous()):
                raise ValueError("weights and gradients must be contiguous CUDA tensors")
            if w.shape != g.shape or w.dim() not in (1, 2, 3):
                raise ValueError("weight / grad shapes must match and be 1-D, 2-D or 3-D")
            if w.dim() == 3:
                shape, stack = (int(w.shape[1]), int(w.shape[2])), int(w.shape[0])
            else:
                shape, stack = (int(w.shape[0]), int(w.shape[1]) if w.dim() == 2 else 0), 0
            descs.append(ParamDesc(w.data_ptr(), g.data_ptr(), (C.c_int64 * 2)(*shape), w.dim(), tier, flags, stack))
            self.params.append((w, g))
        dev = self.params[0][0].device if self.params else torch.device("cuda")
        self._elsewhere = _device_check()
        if self.params and self._elsewhere:
            self._elsewhere(dev)
        self.hp = hp
        self.h = skew_create(descs, hp)
        with contextlib.nullcontext() if stream is None else _on(stream):  # the stream that fills them: no other's work comes between
            self.state = torch.empty(max(1, skew_state_bytes(self.h)), dtype=torch.uint8, device=dev)
            self.workspace = torch.empty(max(1, skew_workspace_bytes(self.h)), dtype=torch.uint8, device=dev)
        skew_bind(self.h, self.state.data_ptr(), skew_state_bytes(self.h), self.workspace.data_ptr(),
                  skew_workspace_bytes(self.h), self._stream(stream))

    def _stream(self, stream) -> int:
        if stream is None:
            return self.torch.cuda.current_stream().cuda_stream
        return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)

    @property
    def state_bytes(self) -> int:
        return skew_state_bytes(self.h)

    @property
    def workspace_bytes(self) -> int:
        return skew_workspace_bytes(self.h)

    def step(self, step: int, lr: float, seed: int, stream=None, grad_scale=None) -> None:
        """One step. `grad_scale`: optional one-element fp32 device tensor gamma (the trainer's
        global gradient-norm clip factor); the step then sees gamma * G."""
        if self._elsewhere:
            self._elsewhere(self.state.device)
        if grad_scale is None:
            skew_step(self.h, step, lr, seed, self._stream(stream))
            return
        if not (grad_scale.is_cuda and grad_scale.dtype == self.torch.float32 and grad_scale.numel() == 1):
            raise ValueError("grad_scale must be a one-element float32 CUDA tensor")
        skew_step_scaled(self.h, step, lr, seed, grad_scale.data_ptr(), self._stream(stream))

    def sync_status(self, stream=None) -> None:
        skew_sync_status(self.h, self._stream(stream))

    def scalars(self, tid: int, stream=None, matrix: int = 0):
        """mean(R), sum of U^2, RMS and clip factor of tensor `tid` (of its matrix
        `matrix` when it is a stack)."""
        return skew_matrix_scalars(self.h, tid, matrix, self._stream(stream))

    def info(self, tid: int) -> TensorInfo:
        return skew_tensor_info(self.h, tid)

    def route(self, tid: int) -> int:
        return skew_tensor_route(self.h, tid)

    def state_views(self, tid: int):
        """fp32 views (M, v, R, C; None when absent) into the state buffer."""
        f = self.state[: self.state_bytes].view(self.torch.float32)
        i = self.info(tid)
        out = {}
        E = max(1, i.stack)  # a stack's arrays hold its matrices' in order
        for key, off, cnt in (("M", i.m_offset, i.numel), ("v", i.v_offset, i.numel), ("R", i.r_offset, E * i.rows),
                              ("C", i.c_offset, E * i.cols)):
            out[key] = None if off < 0 else f[off: off + cnt]
        return out

    def close(self):
        if getattr(self, "h", None):
            skew_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
