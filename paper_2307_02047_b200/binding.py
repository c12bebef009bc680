"""ctypes binding of the C-ABI library declared in ``include/came_b200.h``.

Argument marshalling only: every step of the optimizer runs in the CUDA
kernels of ``libcame_b200.so``.  The functions carry the C names
(``came_create``, ``came_step``, ...).  ``CameOptimizer`` is a small convenience
wrapper that owns the state tensors (allocated with torch) and a context.

There is no fallback: if the library is missing it is built with nvcc, and if
that fails, or a call returns an error status, a ``CameError`` is raised.
"""
from __future__ import annotations

import ctypes
import struct
from typing import List, Optional, Sequence

from . import build as _build

CAME_OK = 0
(CAME_ERR_NULL, CAME_ERR_SHAPE, CAME_ERR_DTYPE, CAME_ERR_ALIGN, CAME_ERR_HPARAM, CAME_ERR_STEP_ORDER,
 CAME_ERR_DEVICE, CAME_ERR_OOM, CAME_ERR_CUDA, CAME_ERR_INTERNAL, CAME_ERR_UNSUPPORTED,
 CAME_ERR_OVERLAP) = range(1, 13)
CAME_F32, CAME_BF16 = 0, 1
CAME_I32, CAME_I64 = 0, 1
CAME_EMBED_ACCUMULATE, CAME_EMBED_PADDING_ROW = 1, 2
CAME_T_NO_WEIGHT_DECAY = 1
CAME_T_VEC_NO_CONFIDENCE = 2
CAME_CREATE_KEEP_STATE = 1
CAME_CREATE_ADAFACTOR = 2
(CAME_Q_NUMEL, CAME_Q_STATE_BYTES, CAME_Q_STREAM_BYTES, CAME_Q_COMPULSORY_BYTES,
 CAME_Q_WORKSPACE_BYTES, CAME_Q_NUM_TILES, CAME_Q_LAUNCHES_PER_STEP, CAME_Q_LAST_STEP,
 CAME_Q_NUM_PHASES, CAME_Q_MATRIX_NUMEL, CAME_Q_SCHEDULE, CAME_Q_PIPE_GROUPS, CAME_Q_PIPE_GRID,
 CAME_Q_DEVICE_ERROR) = range(14)
CAME_Q_P1_STREAM_GRID = 14
CAME_TUNE_TILE_ELEMS = 0
CAME_TUNE_SCHED_GROUP_BYTES = 1
CAME_TUNE_HOST_GROUP_BYTES = 2
CAME_TUNE_PDL = 3
CAME_TUNE_F32_VEC8 = 4
CAME_TUNE_SCHEDULE = 5
CAME_TUNE_PIPE_TILE_ELEMS = 6
CAME_TUNE_PIPE_GROUP_BYTES = 7
CAME_TUNE_PIPE_WAIT_NS = 8
CAME_TUNE_PIPE_ORDER = 9
CAME_TUNE_P1_STREAM = 10
CAME_TUNE_P1_STREAM_RING = 11
CAME_SCHEDULE_AUTO, CAME_SCHEDULE_PHASE_GRIDS, CAME_SCHEDULE_PIPELINED = 0, 1, 2

EXPORTED = ["came_create", "came_step", "came_step_host", "came_destroy", "came_last_error",
            "came_status_string", "came_query", "came_set_profiling", "came_get_phase_ms",
            "came_phase_name", "came_plan_tensor", "came_tune", "came_factor_update_static",
            "came_factor_update_static_plan", "came_required_grad_alignment",
            "came_device_status", "came_lr_warmup", "came_clear_device_error",
            "came_selftest_wait_timeout", "came_debug_bounds", "came_step_scaled",
            "came_clip_create", "came_clip_norm", "came_clip_grads", "came_clip_destroy",
            "came_embed_forward", "came_embed_workspace", "came_embed_backward"]


class CameError(RuntimeError):
    def __init__(self, status: int, text: str):
        super().__init__(f"{text} (status {status})")
        self.status = status


class came_tensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("r", ctypes.c_void_p), ("c", ctypes.c_void_p), ("R", ctypes.c_void_p),
                ("C", ctypes.c_void_p), ("rows", ctypes.c_int64), ("cols", ctypes.c_int64),
                ("ndim", ctypes.c_int32), ("grad_dtype", ctypes.c_int32),
                ("flags", ctypes.c_uint32), ("reserved", ctypes.c_uint32),
                ("param_bf16", ctypes.c_void_p)]


class came_hparams(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("beta3", ctypes.c_double), ("eps1", ctypes.c_double), ("eps2", ctypes.c_double),
                ("clip_d", ctypes.c_double), ("weight_decay", ctypes.c_double),
                ("step", ctypes.c_int64), ("grad_scale", ctypes.c_double)]


class came_clip_tensor(ctypes.Structure):
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("numel", ctypes.c_int64),
                ("grad_dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32)]


class came_clip_params(ctypes.Structure):
    _fields_ = [("max_norm", ctypes.c_double), ("eps", ctypes.c_double),
                ("grad_scale", ctypes.c_double)]


class came_embed(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("data", ctypes.c_void_p), ("ids", ctypes.c_void_p),
                ("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("tokens", ctypes.c_int64),
                ("table_ld", ctypes.c_int64), ("data_ld", ctypes.c_int64),
                ("padding_row", ctypes.c_int64), ("scale", ctypes.c_double),
                ("table_dtype", ctypes.c_int32), ("data_dtype", ctypes.c_int32),
                ("id_dtype", ctypes.c_int32), ("flags", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]


_lib = None


def load():
    """Load (building first if needed) the shared library; raises if it cannot be had."""
    global _lib
    if _lib is not None:
        return _lib
    _lib = _bind(ctypes.CDLL(_build.build()))
    return _lib


_lib_debug = None


def load_debug():
    """The bounds-checking build of the same library (``-DCAME_DEBUG_BOUNDS``), built on demand."""
    global _lib_debug
    if _lib_debug is None:
        _lib_debug = _bind(ctypes.CDLL(_build.build(debug=True)))
    return _lib_debug


class using_debug_build:
    """``with using_debug_build():`` routes every call of this module through the
    bounds-checking build for the duration of the block."""

    def __enter__(self):
        global _lib
        load()
        self.saved = _lib
        _lib = load_debug()
        return self

    def __exit__(self, *exc):
        global _lib
        _lib = self.saved


def _bind(L):
    """Declare the prototypes of every entry point on a freshly loaded library."""
    vp, i32, i64, u32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32
    L.came_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(came_tensor), i32, i32, u32]
    L.came_create.restype = i32
    L.came_step.argtypes = [vp, ctypes.POINTER(came_hparams), ctypes.POINTER(vp), vp]
    L.came_step.restype = i32
    L.came_step_host.argtypes = [vp, ctypes.POINTER(came_hparams), ctypes.POINTER(vp),
                                 ctypes.POINTER(vp), vp]
    L.came_step_host.restype = i32
    L.came_destroy.argtypes = [vp]
    L.came_destroy.restype = i32
    L.came_last_error.argtypes = [vp]
    L.came_last_error.restype = ctypes.c_char_p
    L.came_status_string.argtypes = [i32]
    L.came_status_string.restype = ctypes.c_char_p
    L.came_query.argtypes = [vp, i32, ctypes.POINTER(i64)]
    L.came_query.restype = i32
    L.came_set_profiling.argtypes = [vp, i32]
    L.came_set_profiling.restype = i32
    L.came_get_phase_ms.argtypes = [vp, ctypes.POINTER(ctypes.c_float), i32, ctypes.POINTER(i32)]
    L.came_get_phase_ms.restype = i32
    L.came_phase_name.argtypes = [vp, i32]
    L.came_phase_name.restype = ctypes.c_char_p
    L.came_plan_tensor.argtypes = [i64, i64, i32, i32, i32, i64] + [ctypes.POINTER(i32)] * 5
    L.came_plan_tensor.restype = i32
    L.came_tune.argtypes = [i32, i64]
    L.came_tune.restype = i32
    L.came_factor_update_static.argtypes = [vp, i32, i64, i64, vp, vp, ctypes.c_double,
                                            ctypes.c_double, vp, i32, vp]
    L.came_factor_update_static.restype = i32
    L.came_factor_update_static_plan.argtypes = [vp, i32, i64, i64, vp, vp, ctypes.c_double,
                                                 ctypes.c_double, i32, ctypes.POINTER(i32),
                                                 ctypes.POINTER(i64)]
    L.came_factor_update_static_plan.restype = i32
    L.came_required_grad_alignment.argtypes = [i32, i32]
    L.came_required_grad_alignment.restype = i32
    L.came_device_status.argtypes = [i32, i32]
    L.came_device_status.restype = i32
    L.came_lr_warmup.argtypes = [ctypes.c_double, ctypes.c_double, i64, i64]
    L.came_lr_warmup.restype = ctypes.c_double
    L.came_clear_device_error.argtypes = [vp, vp]
    L.came_clear_device_error.restype = i32
    L.came_selftest_wait_timeout.argtypes = [i32, i64, ctypes.POINTER(i32), ctypes.POINTER(i32),
                                             ctypes.POINTER(ctypes.c_float)]
    L.came_selftest_wait_timeout.restype = i32
    L.came_debug_bounds.argtypes = [i32, ctypes.POINTER(ctypes.c_uint32)]
    L.came_debug_bounds.restype = i32
    L.came_step_scaled.argtypes = [vp, ctypes.POINTER(came_hparams), ctypes.POINTER(vp), vp, vp]
    L.came_step_scaled.restype = i32
    L.came_clip_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(came_clip_tensor), i32, i32]
    L.came_clip_create.restype = i32
    L.came_clip_norm.argtypes = [vp, ctypes.POINTER(came_clip_params), ctypes.POINTER(vp), vp, vp]
    L.came_clip_norm.restype = i32
    L.came_clip_grads.argtypes = L.came_clip_norm.argtypes
    L.came_clip_grads.restype = i32
    L.came_clip_destroy.argtypes = [vp]
    L.came_clip_destroy.restype = i32
    L.came_embed_forward.argtypes = [ctypes.POINTER(came_embed), i32, vp]
    L.came_embed_forward.restype = i32
    L.came_embed_workspace.argtypes = [ctypes.POINTER(came_embed), ctypes.POINTER(i64)]
    L.came_embed_workspace.restype = i32
    L.came_embed_backward.argtypes = [ctypes.POINTER(came_embed), vp, i64, i32, vp]
    L.came_embed_backward.restype = i32
    return L


def _check(status: int, ctx=None) -> None:
    if status != CAME_OK:
        L = load()
        text = L.came_last_error(ctx).decode() or L.came_status_string(status).decode()
        raise CameError(status, f"{L.came_status_string(status).decode()}: {text}")


# --- the C entry points, same names ------------------------------------------------------

def came_create(tensors: Sequence[came_tensor], device: int = 0, flags: int = 0) -> ctypes.c_void_p:
    L = load()
    arr = (came_tensor * len(tensors))(*tensors)
    ctx = ctypes.c_void_p()
    _check(L.came_create(ctypes.byref(ctx), arr, len(tensors), device, flags))
    return ctx


def came_step(ctx, hp: came_hparams, grads: Optional[Sequence[int]] = None, stream: int = 0) -> None:
    L = load()
    garr = None
    if grads is not None:
        garr = (ctypes.c_void_p * len(grads))(*grads)
    _check(L.came_step(ctx, ctypes.byref(hp), garr, ctypes.c_void_p(stream)), ctx)


def came_step_scaled(ctx, hp: came_hparams, grads: Optional[Sequence[int]], device_scale: int,
                     stream: int = 0) -> None:
    """came_step with a further gradient pre-scale read from device memory (address of one fp32)."""
    L = load()
    garr = None
    if grads is not None:
        garr = (ctypes.c_void_p * len(grads))(*grads)
    _check(L.came_step_scaled(ctx, ctypes.byref(hp), garr, ctypes.c_void_p(device_scale),
                              ctypes.c_void_p(stream)), ctx)


def came_step_host(ctx, hp: came_hparams, host_grads: Sequence[int],
                   host_params_out: Optional[Sequence[Optional[int]]] = None, stream: int = 0) -> None:
    L = load()
    garr = (ctypes.c_void_p * len(host_grads))(*host_grads)
    parr = None
    if host_params_out is not None:
        parr = (ctypes.c_void_p * len(host_params_out))(*host_params_out)
    _check(L.came_step_host(ctx, ctypes.byref(hp), garr, parr, ctypes.c_void_p(stream)), ctx)


def came_destroy(ctx) -> None:
    _check(load().came_destroy(ctx))


def came_last_error(ctx=None) -> str:
    return load().came_last_error(ctx).decode()


def came_status_string(status: int) -> str:
    return load().came_status_string(status).decode()


def came_query(ctx, what: int) -> int:
    out = ctypes.c_int64()
    _check(load().came_query(ctx, what, ctypes.byref(out)), ctx)
    return int(out.value)


def came_set_profiling(ctx, enabled: bool) -> None:
    _check(load().came_set_profiling(ctx, int(enabled)), ctx)


def came_get_phase_ms(ctx) -> List[float]:
    buf = (ctypes.c_float * 8)()
    cnt = ctypes.c_int32()
    _check(load().came_get_phase_ms(ctx, buf, 8, ctypes.byref(cnt)), ctx)
    return [float(buf[i]) for i in range(cnt.value)]


def came_phase_name(ctx, phase: int) -> str:
    return load().came_phase_name(ctx, phase).decode()


def came_plan_tensor(rows: int, cols: int, ndim: int, grad_dtype: int, aligned32: bool = True,
                     tile_elems_target: int = 0) -> dict:
    o = [ctypes.c_int32() for _ in range(5)]
    _check(load().came_plan_tensor(rows, cols, ndim, grad_dtype, int(aligned32), tile_elems_target,
                                   *[ctypes.byref(x) for x in o]))
    return dict(zip(("vec", "threads_x", "tile_rows", "n_rb", "n_cb"), (int(x.value) for x in o)))


def came_tune(key: int, value: int) -> None:
    _check(load().came_tune(key, value))


CAME_STATIC_SCRATCH_BYTES = 8 << 20


def came_factor_update_static(grad: int, grad_dtype: int, rows: int, cols: int, r: int, c: int,
                              beta2: float, eps1: float, out_sqrt_sum_r: Optional[int] = None,
                              device: int = 0, stream: int = 0) -> None:
    """r, c <- the first two lines of Algorithm 2 for one matrix, without any allocation.

    For callers that may not allocate device memory (an allocator that owns the device
    heap, a no-synchronisation loop, an audited memory budget): the partial sums use a
    fixed array inside the library instead of a context's workspace.  All pointer
    arguments are device addresses (ints).  Calls share that array: keep them on one stream.
    """
    _check(load().came_factor_update_static(grad, grad_dtype, rows, cols, r, c, float(beta2),
                                            float(eps1), out_sqrt_sum_r, device,
                                            ctypes.c_void_p(stream)))


def came_factor_update_static_plan(grad: int, grad_dtype: int, rows: int, cols: int, r: int, c: int,
                                   beta2: float = 0.999, eps1: float = 1e-30, device: int = 0) -> dict:
    """Host-only: what came_factor_update_static would plan for these arguments (no GPU work)."""
    vec, nbytes = ctypes.c_int32(), ctypes.c_int64()
    _check(load().came_factor_update_static_plan(grad, grad_dtype, rows, cols, r, c, float(beta2),
                                                 float(eps1), device, ctypes.byref(vec),
                                                 ctypes.byref(nbytes)))
    return {"vec": int(vec.value), "scratch_bytes": int(nbytes.value)}


def came_required_grad_alignment(grad_dtype: int, vec: int) -> int:
    return int(load().came_required_grad_alignment(grad_dtype, vec))


def came_device_status(context_device: int, current_device: int) -> int:
    return int(load().came_device_status(context_device, current_device))


def came_lr_warmup(lr_peak: float, lr_start: float, step: int, warmup_steps: int) -> float:
    return float(load().came_lr_warmup(lr_peak, lr_start, step, warmup_steps))


def came_clear_device_error(ctx, stream: int = 0) -> None:
    _check(load().came_clear_device_error(ctx, ctypes.c_void_p(stream)), ctx)


def came_selftest_wait_timeout(device: int = 0, limit_ns: int = 1_000_000) -> dict:
    a, b, ms = ctypes.c_int32(), ctypes.c_int32(), ctypes.c_float()
    _check(load().came_selftest_wait_timeout(device, limit_ns, ctypes.byref(a), ctypes.byref(b),
                                             ctypes.byref(ms)))
    return {"timed_out": int(a.value), "error_word": int(b.value), "elapsed_ms": float(ms.value)}


def came_debug_bounds(device: int = 0) -> dict:
    """The device-side record of the bounds-checking build (raises CAME_ERR_UNSUPPORTED, status
    11, on the ordinary build)."""
    out = (ctypes.c_uint32 * 6)()
    _check(load().came_debug_bounds(device, out))
    return dict(zip(("code", "rb", "cb", "rows", "cols", "threads"), (int(x) for x in out)))


def came_clip_create(tensors: Sequence[came_clip_tensor], device: int = 0) -> ctypes.c_void_p:
    ctx = ctypes.c_void_p()
    arr = tensors if isinstance(tensors, ctypes.Array) else (came_clip_tensor * len(tensors))(*tensors)
    _check(load().came_clip_create(ctypes.byref(ctx), arr, len(tensors), device))
    return ctx


def came_clip_norm(ctx, params: came_clip_params, results: int, grads: Optional[Sequence[int]] = None,
                   stream: int = 0) -> None:
    garr = None if grads is None else (ctypes.c_void_p * len(grads))(*grads)
    _check(load().came_clip_norm(ctx, params, garr, results, stream))


def came_clip_grads(ctx, params: came_clip_params, results: int, grads: Optional[Sequence[int]] = None,
                    stream: int = 0) -> None:
    garr = None if grads is None else (ctypes.c_void_p * len(grads))(*grads)
    _check(load().came_clip_grads(ctx, params, garr, results, stream))


def came_clip_destroy(ctx) -> None:
    _check(load().came_clip_destroy(ctx))


def came_embed_forward(e: came_embed, device: int = 0, stream: int = 0) -> None:
    status = (_lib or load()).came_embed_forward(e, device, stream)
    if status:
        _check(status)


def came_embed_workspace(e: came_embed) -> int:
    out = ctypes.c_int64()
    status = (_lib or load()).came_embed_workspace(e, out)
    if status:
        _check(status)
    return out.value


def came_embed_backward(e: came_embed, workspace: int, workspace_bytes: int, device: int = 0,
                        stream: int = 0) -> None:
    status = (_lib or load()).came_embed_backward(e, workspace, workspace_bytes, device, stream)
    if status:
        _check(status)


def make_hparams(step: int, **kw) -> came_hparams:
    return came_hparams(float(kw["lr"]), float(kw["beta1"]), float(kw["beta2"]), float(kw["beta3"]),
                        float(kw["eps1"]), float(kw["eps2"]), float(kw["clip_d"]),
                        float(kw.get("weight_decay", 0.0)), int(step),
                        float(kw.get("grad_scale", 1.0)))


# --- what the operators' wrappers share ------------------------------------------------------

_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch
        _torch_module = torch
    return _torch_module


def _call_on(index, call, *args) -> None:
    """``call(*args, index, stream)`` with device ``index`` current; ``stream``: its current stream's
    address (asked for directly: a Stream object costs more than a launch)."""
    C = _torch()._C
    before = C._cuda_getDevice()
    if before == index:
        call(*args, index, C._cuda_getCurrentRawStream(index))
        return
    with _torch().cuda.device(index):
        call(*args, index, C._cuda_getCurrentRawStream(index))


# --- gradient norm and clipping ------------------------------------------------------------

def _cuda_tensor(x, name, dtype=None, device=None) -> None:
    if not x.is_cuda or (device is not None and x.device != device):
        raise CameError(CAME_ERR_DEVICE, f"{name} must be a CUDA tensor on {device or 'a GPU'}")
    if dtype is not None and x.dtype != dtype:
        raise CameError(CAME_ERR_DTYPE, f"{name} must be {dtype}, got {x.dtype}")


_DTYPE_CODES = {}       # torch dtype -> came_dtype


def _dtype_code(x, name) -> int:
    if not _DTYPE_CODES:
        _DTYPE_CODES.update({_torch().float32: CAME_F32, _torch().bfloat16: CAME_BF16})
    code = _DTYPE_CODES.get(x.dtype)
    if code is None:
        raise CameError(CAME_ERR_DTYPE, f"{name} must be fp32 or bf16, got {x.dtype}")
    return code


class GradClip:
    """The global norm of a list of gradients, and clipping by it.  To be made once for a list and
    kept: creation plans the tiles, allocates, and waits for a copy.

    ``grads``: contiguous fp32 or bf16 CUDA tensors of any shape, read by every call (their
    storage may be refilled; tensors with new memory are handed to a call).  ``outs``: where ``clip`` writes, tensors of the same sizes (``grads``
    itself clips in place), fp32 or bf16; None: norm only.  After a call ``total_norm``, ``coef``
    (CUDA scalars) and ``tensor_norms`` (one per tensor) hold its results, until the next call.
    """

    def __init__(self, grads, outs=None):
        import torch
        self.ctx = None
        self.grads = list(grads)
        self.outs = None if outs is None else list(outs)
        if not self.grads:
            raise CameError(CAME_ERR_SHAPE, "need at least one tensor")
        if self.outs is not None and len(self.outs) != len(self.grads):
            raise CameError(CAME_ERR_SHAPE, "outs must be as many as grads")
        first = self.grads[0]
        _cuda_tensor(first, "grads[0]")
        self.device = first.device
        self._codes = [self._check_tensor(g, "grads", i) for i, g in enumerate(self.grads)]
        packed = []
        if self.outs is None:
            for g, code in zip(self.grads, self._codes):
                packed += (g.data_ptr(), 0, g.numel(), code, 0)
        else:
            for i, (g, o, code) in enumerate(zip(self.grads, self.outs, self._codes)):
                out_code = self._check_tensor(o, "outs", i)
                if o.numel() != g.numel():
                    raise CameError(CAME_ERR_SHAPE, f"outs[{i}] has another size than grads[{i}]")
                packed += (g.data_ptr(), o.data_ptr(), g.numel(), code, out_code)
        n = len(self.grads)
        descs = (came_clip_tensor * n).from_buffer_copy(struct.pack("PPqii" * n, *packed))
        self.results = torch.empty(2 + n, dtype=torch.float32, device=self.device)
        self.total_norm, self.coef, self.tensor_norms = self.results[0], self.results[1], self.results[2:]
        self._results_at = self.results.data_ptr()
        self._params = came_clip_params()
        with torch.cuda.device(self.device):
            self.ctx = came_clip_create(descs, self.device.index)

    def _check_tensor(self, x, name, i) -> int:
        """The dtype code of a tensor that may be in the list."""
        if x.device != self.device:
            raise CameError(CAME_ERR_DEVICE, f"{name}[{i}] must be on {self.device}")
        if not x.is_contiguous():
            raise CameError(CAME_ERR_UNSUPPORTED, f"{name}[{i}] must be contiguous")
        return _dtype_code(x, name)

    def _run(self, call, max_norm, eps, grad_scale, grads):
        at = None
        if grads is not None:
            grads = list(grads)
            if len(grads) != len(self.grads):
                raise CameError(CAME_ERR_SHAPE, "grads must be as many as at creation")
            for i, (g, old) in enumerate(zip(grads, self.grads)):
                if self._check_tensor(g, "grads", i) != self._codes[i] or g.numel() != old.numel():
                    raise CameError(CAME_ERR_SHAPE, f"grads[{i}] must keep its size and dtype")
            at = [g.data_ptr() for g in grads]
        p = self._params
        p.max_norm, p.eps, p.grad_scale = max_norm, eps, grad_scale
        _call_on(self.device.index, call, self.ctx, p, self._results_at, at)
        if grads is not None:
            self.grads = grads
        return self.total_norm, self.coef, self.tensor_norms

    @staticmethod
    def _norm_call(ctx, p, results, at, index, stream):
        came_clip_norm(ctx, p, results, at, stream)

    @staticmethod
    def _clip_call(ctx, p, results, at, index, stream):
        came_clip_grads(ctx, p, results, at, stream)

    def norm(self, max_norm: float = float("inf"), eps: float = 1e-6, grad_scale: float = 1.0,
             grads=None):
        """``(total_norm, coef, tensor_norms)``; ``grads`` replaces the tensors of earlier calls
        (not inside a stream capture)."""
        return self._run(self._norm_call, max_norm, eps, grad_scale, grads)

    def clip(self, max_norm: float, eps: float = 1e-6, grad_scale: float = 1.0, grads=None):
        """``norm``, and ``outs = grads * (grad_scale * coef)``."""
        return self._run(self._clip_call, max_norm, eps, grad_scale, grads)

    def close(self) -> None:
        if self.ctx is not None:
            import torch
            torch.cuda.synchronize(self.device)
            came_clip_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# --- embedding lookup and its gradient -------------------------------------------------------

# (Written for small calls, whose time is the host's: one look at each attribute.)

_ID_CODES = {}          # torch dtype -> came_id_dtype


def _embed_table(table, name):
    """(rows, columns, row stride, dtype code, device index) of the table or its gradient."""
    if not _ID_CODES:
        torch = _torch()
        _DTYPE_CODES.update({torch.float32: CAME_F32, torch.bfloat16: CAME_BF16})
        _ID_CODES.update({torch.int32: CAME_I32, torch.int64: CAME_I64})
    shape, index = table.shape, table.get_device()
    if len(shape) != 2:
        raise CameError(CAME_ERR_SHAPE, f"{name} must be a matrix")
    if index < 0:
        raise CameError(CAME_ERR_DEVICE, f"{name} must be a CUDA tensor")
    rows, cols = shape
    ld, one = table.stride()
    if one != 1 and cols > 1:
        raise CameError(CAME_ERR_UNSUPPORTED, f"the rows of {name} must be contiguous")
    code = _DTYPE_CODES.get(table.dtype)
    if code is None:
        raise CameError(CAME_ERR_DTYPE, f"{name} must be fp32 or bf16, got {table.dtype}")
    return rows, cols, ld if rows > 1 else cols, code, index       # (the stride of a single row says nothing)


def _embed_ids(ids, index) -> int:
    """The ids' type code."""
    if ids.get_device() != index:
        raise CameError(CAME_ERR_DEVICE, "ids must be on the table's GPU")
    code = _ID_CODES.get(ids.dtype)
    if code is None:
        raise CameError(CAME_ERR_DTYPE, f"ids must be int32 or int64, got {ids.dtype}")
    if not ids.is_contiguous():
        raise CameError(CAME_ERR_UNSUPPORTED, "ids must be contiguous")
    return code


def _embed_data(data, name, ids, cols, index):
    """(row stride, dtype code) of the tokens' rows."""
    shape = data.shape
    if not shape or shape[:-1] != ids.shape or shape[-1] != cols:
        raise CameError(CAME_ERR_SHAPE, f"{name} must have the shape of ids and the columns of the table")
    if data.get_device() != index:
        raise CameError(CAME_ERR_DEVICE, f"{name} must be on the table's GPU")
    code = _DTYPE_CODES.get(data.dtype)
    if code is None:
        raise CameError(CAME_ERR_DTYPE, f"{name} must be fp32 or bf16, got {data.dtype}")
    if len(shape) != 2:
        try:
            data = data.view(ids.numel(), cols)
        except RuntimeError:
            raise CameError(CAME_ERR_UNSUPPORTED, f"the rows of {name} must lie at one stride") from None
    ld, one = data.stride()
    if one != 1 and cols > 1:
        raise CameError(CAME_ERR_UNSUPPORTED, f"the rows of {name} must be contiguous")
    return ld if data.shape[0] > 1 else cols, code


_lookup_class = None


def _lookup_function():
    """The lookup as an autograd function."""
    global _lookup_class
    if _lookup_class is None:
        torch = _torch()

        class Lookup(torch.autograd.Function):
            @staticmethod
            def forward(ctx, table, ids, scale, out_dtype):
                ctx.save_for_backward(ids)
                ctx.shape, ctx.dtype, ctx.scale = table.shape, table.dtype, scale
                return embed_forward(table, ids, scale, out_dtype=out_dtype)      # (grad mode is off here)

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, grad_out):
                (ids,) = ctx.saved_tensors
                grad = grad_out.new_empty(ctx.shape, dtype=ctx.dtype)
                return embed_backward(grad_out.contiguous(), ids, grad, ctx.scale), None, None, None

        _lookup_class = Lookup
    return _lookup_class


def embed_forward(table, ids, scale: float = 1.0, out=None, out_dtype=None):
    """``out[t] = scale * table[ids[t]]``, zero where an id is not a row of the table.

    ``table``: fp32 or bf16 CUDA matrix with contiguous rows; ``ids``: contiguous int32 or int64
    CUDA tensor of any shape; ``out``: tensor of shape ``(*ids.shape, cols)``, fp32 or bf16, made
    here when it is None (of type ``out_dtype``, the table's when that is None too).

    When autograd records and the table requires grad, the result carries the graph: the table's
    gradient is ``embed_backward``'s, a whole matrix of its type (once differentiable).  ``out``
    must be None then; ``embed_backward`` itself adds to a buffer of the caller's."""
    if table.requires_grad and _torch().is_grad_enabled():
        if out is not None:
            raise CameError(CAME_ERR_UNSUPPORTED, "a table that requires grad takes no out: detach it, or disable grad mode")
        return _lookup_function().apply(table, ids, scale, out_dtype)
    rows, cols, table_ld, table_code, index = _embed_table(table, "table")
    id_code = _embed_ids(ids, index)
    if out is None:
        out = table.new_empty((*ids.shape, cols), dtype=out_dtype)
        ld, code = cols, _DTYPE_CODES.get(out.dtype)
        if code is None:
            raise CameError(CAME_ERR_DTYPE, f"out must be fp32 or bf16, got {out.dtype}")
    else:
        if out_dtype is not None and out.dtype != out_dtype:
            raise CameError(CAME_ERR_DTYPE, f"out is {out.dtype}, not {out_dtype}")
        ld, code = _embed_data(out, "out", ids, cols, index)
    e = came_embed(table.data_ptr(), out.data_ptr(), ids.data_ptr(), rows, cols, ids.numel(), table_ld, ld,
                   0, scale, table_code, code, id_code, 0, 0)
    _call_on(index, came_embed_forward, e)
    return out


def embed_backward(grad_out, ids, grad, scale: float = 1.0, padding_row: Optional[int] = None,
                   accumulate: bool = False):
    """``grad[v] = scale * (sum of grad_out[t] over the tokens with ids[t] == v)``; with
    ``accumulate`` the sums are added to ``grad`` (a table tied to the output head).

    ``grad_out``: fp32 or bf16, shape ``(*ids.shape, cols)``; ``grad``: fp32 or bf16 matrix, every
    row of it written unless ``accumulate``; tokens of ``padding_row`` add nothing.  Returns
    ``grad``.  Bit-reproducible: a row's tokens are added in an order fixed by the ids."""
    rows, cols, grad_ld, grad_code, index = _embed_table(grad, "grad")
    id_code = _embed_ids(ids, index)
    ld, code = _embed_data(grad_out, "grad_out", ids, cols, index)
    flags = CAME_EMBED_ACCUMULATE if accumulate else 0
    if padding_row is not None:
        flags |= CAME_EMBED_PADDING_ROW
    e = came_embed(grad.data_ptr(), grad_out.data_ptr(), ids.data_ptr(), rows, cols, ids.numel(), grad_ld, ld,
                   padding_row or 0, scale, grad_code, code, id_code, flags, 0)
    size = came_embed_workspace(e)
    # from torch's allocator, for the device's current stream: not reused before the call is done
    ws = grad.new_empty((size + 3) // 4, dtype=_torch().float32)
    _call_on(index, came_embed_backward, e, ws.data_ptr(), size)
    return grad


# --- convenience wrapper -------------------------------------------------------------------

class CameOptimizer:
    """Owns the CAME state for a list of torch CUDA parameter tensors and steps them.

    ``params``: fp32 CUDA tensors (contiguous), updated in place.  1-D tensors take the vector
    path, 2-D tensors the matrix path; a tensor of rank >= 3 is handed to the library as the
    matrix (product of the leading dims) x (last dim), since the paper defines the method for
    matrices only.
    ``grads``: CUDA tensors of the same shapes, fp32 or bf16, read every step
    (their storage may be refilled between steps; pointers are fixed at creation).
    torch is used for allocation and the stream only.
    """

    def __init__(self, params, grads, flags: Optional[Sequence[int]] = None, device: int = 0,
                 create_flags: int = 0, bf16_copy: bool = False):
        import torch
        self.torch = torch
        self.params, self.grads = list(params), list(grads)
        self.m, self.r, self.c, self.R, self.C = [], [], [], [], []
        self.p_bf16 = []
        descs = []
        for i, (p, g) in enumerate(zip(self.params, self.grads)):
            assert p.is_cuda and p.dtype == torch.float32 and p.is_contiguous()
            assert g.is_cuda and g.is_contiguous() and g.shape == p.shape
            assert p.dim() >= 1
            ndim = 1 if p.dim() == 1 else 2
            cols = p.shape[-1] if ndim == 2 else 1
            rows = p.numel() // cols
            z = lambda n: torch.empty(n, dtype=torch.float32, device=p.device)
            self.m.append(torch.empty_like(p))
            self.r.append(z(rows)); self.R.append(z(rows))
            self.c.append(z(cols) if ndim == 2 else None)
            self.C.append(z(cols) if ndim == 2 else None)
            gd = CAME_BF16 if g.dtype == torch.bfloat16 else CAME_F32
            assert g.dtype in (torch.bfloat16, torch.float32)
            ptr = lambda t: t.data_ptr() if t is not None else None
            self.p_bf16.append(torch.empty_like(p, dtype=torch.bfloat16) if bf16_copy else None)
            descs.append(came_tensor(ptr(p), ptr(g), ptr(self.m[i]), ptr(self.r[i]), ptr(self.c[i]),
                                     ptr(self.R[i]), ptr(self.C[i]), rows, cols, ndim, gd,
                                     0 if flags is None else int(flags[i]), 0, ptr(self.p_bf16[i])))
        self.ctx = came_create(descs, device=device, flags=create_flags)
        self.step_count = 0

    def step(self, device_scale=None, **hp) -> None:
        """``device_scale``: an fp32 CUDA scalar that multiplies every gradient (``GradClip.coef``:
        the step then takes clipped gradients that nothing has to write)."""
        if device_scale is not None:
            _cuda_tensor(device_scale, "device_scale", self.torch.float32, self.params[0].device)
            if device_scale.numel() != 1:
                raise CameError(CAME_ERR_SHAPE, "device_scale must hold one value")
        self.step_count += 1
        stream = self.torch.cuda.current_stream().cuda_stream
        came_step_scaled(self.ctx, make_hparams(self.step_count, **hp), None,
                         0 if device_scale is None else device_scale.data_ptr(), stream)

    def query(self, what: int) -> int:
        return came_query(self.ctx, what)

    def close(self) -> None:
        if self.ctx is not None:
            self.torch.cuda.synchronize()
            came_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
