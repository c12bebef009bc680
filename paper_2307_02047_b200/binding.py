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
import operator
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
CAME_LAYERNORM_ACCUMULATE = 1
CAME_POSBIAS_BIDIRECTIONAL, CAME_POSBIAS_ACCUMULATE = 1, 2
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
            "came_embed_forward", "came_embed_workspace", "came_embed_backward",
            "came_adamw_create", "came_adamw_step", "came_adamw_destroy",
            "came_layernorm_forward", "came_layernorm_workspace", "came_layernorm_backward",
            "came_posbias_forward", "came_posbias_workspace", "came_posbias_backward", "came_posbias_bucket"]


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


class came_adamw_tensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("m", ctypes.c_void_p),
                ("v", ctypes.c_void_p), ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("param_bf16", ctypes.c_void_p), ("numel", ctypes.c_int64), ("grad_dtype", ctypes.c_int32),
                ("state_bits", ctypes.c_int32), ("flags", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]


class came_adamw_hparams(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double), ("grad_scale", ctypes.c_double),
                ("step", ctypes.c_int64), ("seed", ctypes.c_uint64)]


class came_layernorm(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in ("x", "weight", "bias", "y", "dy", "dx", "dweight", "dbias", "mean", "rstd")] + \
               [(k, ctypes.c_int64) for k in ("rows", "cols", "x_ld", "y_ld", "dx_ld")] + [("eps", ctypes.c_double)] + \
               [(k, ctypes.c_int32) for k in ("x_dtype", "y_dtype", "dx_dtype", "weight_dtype")] + \
               [("flags", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]


class came_posbias(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in ("table", "data", "device_offset")] + \
               [(k, ctypes.c_int64) for k in ("offset", "q_len", "k_len", "batch", "table_ld", "batch_stride", "head_stride", "q_stride")] + \
               [(k, ctypes.c_int32) for k in ("heads", "buckets", "max_distance", "table_dtype", "data_dtype")] + [("flags", ctypes.c_uint32)]


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
    L.came_adamw_create.argtypes = [ctypes.POINTER(vp), ctypes.POINTER(came_adamw_tensor), i32, i32, u32]
    L.came_adamw_create.restype = i32
    L.came_adamw_step.argtypes = [vp, ctypes.POINTER(came_adamw_hparams), ctypes.POINTER(vp), vp, vp, vp]
    L.came_adamw_step.restype = i32
    L.came_adamw_destroy.argtypes = [vp]
    L.came_adamw_destroy.restype = i32
    L.came_layernorm_forward.argtypes = [ctypes.POINTER(came_layernorm), i32, vp]
    L.came_layernorm_forward.restype = i32
    L.came_layernorm_workspace.argtypes = [ctypes.POINTER(came_layernorm), ctypes.POINTER(i64)]
    L.came_layernorm_workspace.restype = i32
    L.came_layernorm_backward.argtypes = [ctypes.POINTER(came_layernorm), vp, i64, i32, vp]
    L.came_layernorm_backward.restype = i32
    L.came_posbias_forward.argtypes = [ctypes.POINTER(came_posbias), i32, vp]
    L.came_posbias_forward.restype = i32
    L.came_posbias_workspace.argtypes = [ctypes.POINTER(came_posbias), ctypes.POINTER(i64)]
    L.came_posbias_workspace.restype = i32
    L.came_posbias_backward.argtypes = [ctypes.POINTER(came_posbias), vp, i64, i32, vp]
    L.came_posbias_backward.restype = i32
    L.came_posbias_bucket.argtypes = [ctypes.POINTER(came_posbias), i64, ctypes.POINTER(i32)]
    L.came_posbias_bucket.restype = i32
    # the same functions for descriptors that are packed bytes (a third of a structure's time to make)
    for name in ("came_layernorm_forward", "came_layernorm_workspace", "came_layernorm_backward",
                 "came_posbias_forward", "came_posbias_workspace", "came_posbias_backward"):
        packed, known = L[name], getattr(L, name)
        packed.argtypes, packed.restype = [ctypes.c_char_p, *known.argtypes[1:]], known.restype
        setattr(L, name + "_packed", packed)
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


def came_adamw_create(tensors: Sequence[came_adamw_tensor], device: int = 0, flags: int = 0) -> ctypes.c_void_p:
    ctx = ctypes.c_void_p()
    arr = (came_adamw_tensor * len(tensors))(*tensors)
    _check(load().came_adamw_create(ctypes.byref(ctx), arr, len(tensors), device, flags))
    return ctx


def came_adamw_step(ctx, hp: came_adamw_hparams, grads: Optional[Sequence[int]] = None, device_scale: int = 0,
                    device_step: int = 0, stream: int = 0) -> None:
    garr = None if grads is None else (ctypes.c_void_p * len(grads))(*grads)
    status = (_lib or load()).came_adamw_step(ctx, hp, garr, device_scale, device_step, stream)
    if status:
        _check(status)


def came_adamw_destroy(ctx) -> None:
    _check(load().came_adamw_destroy(ctx))


def came_layernorm_forward(l: came_layernorm, device: int = 0, stream: int = 0) -> None:
    status = (_lib or load()).came_layernorm_forward(l, device, stream)
    if status:
        _check(status)


def came_layernorm_workspace(l: came_layernorm) -> int:
    out = ctypes.c_int64()
    status = (_lib or load()).came_layernorm_workspace(l, out)
    if status:
        _check(status)
    return out.value


def came_layernorm_backward(l: came_layernorm, workspace: int, workspace_bytes: int, device: int = 0,
                            stream: int = 0) -> None:
    status = (_lib or load()).came_layernorm_backward(l, workspace, workspace_bytes, device, stream)
    if status:
        _check(status)


def came_posbias_forward(p: came_posbias, device: int = 0, stream: int = 0) -> None:
    _check(load().came_posbias_forward(p, device, stream))


def came_posbias_workspace(p: came_posbias) -> int:
    out = ctypes.c_int64()
    _check(load().came_posbias_workspace(p, out))
    return out.value


def came_posbias_backward(p: came_posbias, workspace: int, workspace_bytes: int, device: int = 0, stream: int = 0) -> None:
    _check(load().came_posbias_backward(p, workspace, workspace_bytes, device, stream))


def came_posbias_bucket(p: came_posbias, relative: int) -> int:
    out = ctypes.c_int32()
    _check(load().came_posbias_bucket(p, relative, out))
    return out.value


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


_forward_ad = None


def _refuse_tangents(*tensors) -> None:
    """Forward-mode differentiation has no formulas here, and a result without a tangent would count as constant."""
    global _forward_ad
    if _forward_ad is None:
        _forward_ad = _torch().autograd.forward_ad
    if _forward_ad._current_level < 0:       # (looked at first: unpacking takes a microsecond for each tensor)
        return
    for t in tensors:
        if t is not None and _forward_ad.unpack_dual(t).tangent is not None:
            raise CameError(CAME_ERR_UNSUPPORTED, "a tensor carries a tangent: no forward-mode differentiation here")


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
    _refuse_tangents(table)
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
    _refuse_tangents(grad_out)
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


# --- AdamW ---------------------------------------------------------------------------------------

CAME_ADAMW_BLOCK = 256      # consecutive elements that share a scale where states have 8 bits


class AdamWOptimizer:
    """AdamW over a list of torch CUDA parameter tensors: one launch steps them all (one for each type
    of state and gradient in the list).

    ``params``: fp32 CUDA tensors of any shape, contiguous, updated in place.  ``grads``: tensors of the same
    shapes, fp32 or bf16, read by every step (their storage may be refilled; tensors with new memory are
    handed to ``step``).  ``state_bits``: 32 (fp32 states) or 8, one for all or one per tensor.  With 8, ``m[i]``
    is ``torch.float8_e4m3fn``, ``v[i]`` is ``torch.float8_e5m2``, both in the shape of the parameter, and each 256
    consecutive elements share a power of two in ``m_scale[i]``, ``v_scale[i]`` (``torch.float8_e8m0fnu``):
    the state's value is code times scale.  States are rounded up or down at random, with bits that
    ``seed`` and the number of the step determine (see ``include/came_b200.h``).

    ``m``, ``v``, ``m_scale``, ``v_scale``: lists of the states to go on with (None: new ones, zero);
    ``step_count`` goes with them.  ``flags``: one per tensor, ``CAME_T_NO_WEIGHT_DECAY`` or 0.  ``bf16_copy``: True,
    or the list of bf16 tensors that every step fills with the new parameters (``p_bf16``)."""

    def __init__(self, params, grads, state_bits=32, flags: Optional[Sequence[int]] = None, bf16_copy=False,
                 m=None, v=None, m_scale=None, v_scale=None, seed: int = 0, step_count: int = 0):
        torch = _torch()
        self.ctx = None
        self.params, self.grads = list(params), list(grads)
        n = len(self.params)
        if not n or len(self.grads) != n:
            raise CameError(CAME_ERR_SHAPE, "need at least one parameter, and as many grads")
        self.state_bits = [state_bits] * n if isinstance(state_bits, int) else list(state_bits)
        if not 0 <= seed < 1 << 64:
            raise CameError(CAME_ERR_HPARAM, "seed must lie in [0, 2^64)")
        given = {"state_bits": self.state_bits, "m": m, "v": v, "m_scale": m_scale, "v_scale": v_scale, "flags": flags,
                 "bf16_copy": None if isinstance(bf16_copy, bool) or bf16_copy is None else bf16_copy}
        for name, x in given.items():
            if x is not None and len(x) != n:
                raise CameError(CAME_ERR_SHAPE, f"{name} must be as many as params")
        if (m is None) != (v is None) or (m is None and (m_scale is not None or v_scale is not None)):
            raise CameError(CAME_ERR_NULL, "m and v belong together, and scales to them")
        first = self.params[0]
        _cuda_tensor(first, "params[0]")
        self.device, self.seed, self.step_count = first.device, seed, step_count
        self.m, self.v, self.m_scale, self.v_scale, self.p_bf16 = [], [], [], [], []
        descs, self._codes = [], []
        at = lambda x: 0 if x is None else x.data_ptr()  # noqa: E731
        for i, (p, g, bits) in enumerate(zip(self.params, self.grads, self.state_bits)):
            self._check_tensor(p, f"params[{i}]", (torch.float32,), p.numel())
            self._codes.append(_dtype_code(g, f"grads[{i}]"))
            self._check_tensor(g, f"grads[{i}]", None, p.numel())
            if bits not in (32, 8):
                raise CameError(CAME_ERR_DTYPE, f"state_bits of tensor {i} must be 32 or 8")
            blocks = -(-p.numel() // CAME_ADAMW_BLOCK)
            e8m0 = torch.float8_e8m0fnu
            for name, mine, theirs, dtype, shape in (
                    ("m", self.m, m, torch.float32 if bits == 32 else torch.float8_e4m3fn, p.shape),
                    ("v", self.v, v, torch.float32 if bits == 32 else torch.float8_e5m2, p.shape),
                    ("m_scale", self.m_scale, m_scale, e8m0 if bits == 8 else None, (blocks,)),
                    ("v_scale", self.v_scale, v_scale, e8m0 if bits == 8 else None, (blocks,))):
                if dtype is None:
                    mine.append(None)
                elif m is None:
                    zeros = torch.zeros(shape, dtype=torch.float32 if dtype == torch.float32 else torch.uint8, device=self.device)
                    mine.append(zeros if dtype == torch.float32 else zeros.view(dtype))
                else:
                    if theirs is None or theirs[i] is None:
                        raise CameError(CAME_ERR_NULL, f"{name}[{i}] is required with 8-bit states")
                    self._check_tensor(theirs[i], f"{name}[{i}]", (dtype,), p.numel() if len(shape) != 1 or name in "mv" else blocks)
                    mine.append(theirs[i])
            if given["bf16_copy"] is not None:
                self._check_tensor(bf16_copy[i], f"bf16_copy[{i}]", (torch.bfloat16,), p.numel())
                self.p_bf16.append(bf16_copy[i])
            else:
                self.p_bf16.append(torch.empty_like(p, dtype=torch.bfloat16, requires_grad=False) if bf16_copy else None)
            descs.append(came_adamw_tensor(at(p), at(g), at(self.m[i]), at(self.v[i]), at(self.m_scale[i]), at(self.v_scale[i]),
                                           at(self.p_bf16[i]), p.numel(), self._codes[i], bits, 0 if flags is None else int(flags[i]), 0))
        self._hp = came_adamw_hparams()
        with torch.cuda.device(self.device):
            self.ctx = came_adamw_create(descs, self.device.index, CAME_CREATE_KEEP_STATE)

    def _check_tensor(self, x, name, dtypes, numel) -> None:
        if x.device != self.device:
            raise CameError(CAME_ERR_DEVICE, f"{name} must be on {self.device}")
        if dtypes is not None and x.dtype not in dtypes:
            raise CameError(CAME_ERR_DTYPE, f"{name} must be {dtypes[0]}, got {x.dtype}")
        if x.numel() != numel:
            raise CameError(CAME_ERR_SHAPE, f"{name} must have {numel} elements")
        if not x.is_contiguous():
            raise CameError(CAME_ERR_UNSUPPORTED, f"{name} must be contiguous")

    def step(self, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.0,
             grad_scale: float = 1.0, device_scale=None, device_step=None, grads=None) -> None:
        """One step on the current stream.

        ``device_scale``: an fp32 CUDA scalar that multiplies every gradient (``GradClip.coef``).  ``device_step``: an
        int64 CUDA scalar that holds the number of the step, counted by the caller: for steps that are captured
        into a graph (``step_count`` is not used then).  ``grads``: tensors that this call reads in place
        of the ones given at creation."""
        torch = _torch()
        scale_at = step_at = 0
        if device_scale is not None:
            _cuda_tensor(device_scale, "device_scale", torch.float32, self.device)
            if device_scale.numel() != 1:
                raise CameError(CAME_ERR_SHAPE, "device_scale must hold one value")
            scale_at = device_scale.data_ptr()
        if device_step is not None:
            _cuda_tensor(device_step, "device_step", torch.int64, self.device)
            if device_step.numel() != 1:
                raise CameError(CAME_ERR_SHAPE, "device_step must hold one value")
            step_at = device_step.data_ptr()
        moved = None
        if grads is not None:
            grads = list(grads)
            if len(grads) != len(self.params):
                raise CameError(CAME_ERR_SHAPE, "grads must be as many as params")
            for i, (g, p) in enumerate(zip(grads, self.params)):
                self._check_tensor(g, f"grads[{i}]", None, p.numel())
                if _dtype_code(g, f"grads[{i}]") != self._codes[i]:
                    raise CameError(CAME_ERR_DTYPE, f"grads[{i}] must keep its dtype")
            moved = [g.data_ptr() for g in grads]
        hp = self._hp
        hp.lr, hp.beta1, hp.beta2, hp.eps, hp.weight_decay, hp.grad_scale = lr, beta1, beta2, eps, weight_decay, grad_scale
        hp.step, hp.seed = self.step_count + 1, self.seed
        _call_on(self.device.index, self._step_call, self.ctx, hp, moved, scale_at, step_at)
        if device_step is None:
            self.step_count += 1

    @staticmethod
    def _step_call(ctx, hp, grads, scale_at, step_at, index, stream):
        came_adamw_step(ctx, hp, grads, scale_at, step_at, stream)

    def close(self) -> None:
        if self.ctx is not None:
            _torch().cuda.synchronize(self.device)
            came_adamw_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# --- layer norm ----------------------------------------------------------------------------------


# (Written for small calls, whose time is the host's: packed descriptors, one look at each attribute.)

_pack_layernorm = struct.Struct("10P5qd4iII").pack


def _rows_of(x, name, shape, index):
    """(rows, row stride, dtype code) of a tensor whose last dimension is normalised."""
    if x.get_device() != index:
        raise CameError(CAME_ERR_DEVICE, f"{name} must be on the GPU of x")
    code = _DTYPE_CODES.get(x.dtype)
    if code is None:
        code = _dtype_code(x, name)
    mine = x.shape
    if shape is not None and mine != shape:
        raise CameError(CAME_ERR_SHAPE, f"{name} must have the shape of x")
    if not mine or not mine[-1]:
        raise CameError(CAME_ERR_SHAPE, f"{name} must have a last dimension of at least one element")
    cols = mine[-1]
    if x.is_contiguous():
        return x.numel() // cols, cols, code
    if len(mine) != 2:
        try:
            x = x.view(x.numel() // cols, cols)
        except RuntimeError:
            raise CameError(CAME_ERR_UNSUPPORTED, f"the rows of {name} must lie at one stride") from None
    rows = x.shape[0]
    ld, one = x.stride()
    if one != 1 and cols > 1:
        raise CameError(CAME_ERR_UNSUPPORTED, f"the rows of {name} must be contiguous")
    return rows, ld if rows > 1 else cols, code           # (the stride of a single row says nothing)


def _norm_param(p, name, cols, index, code):
    """Address of a parameter (or gradient) of a row's length, and its dtype code; `code`: the one that it must have."""
    if p.get_device() != index:
        raise CameError(CAME_ERR_DEVICE, f"{name} must be on the GPU of x")
    mine = _DTYPE_CODES.get(p.dtype)
    if mine is None:
        mine = _dtype_code(p, name)
    if code is not None and mine != code:
        raise CameError(CAME_ERR_DTYPE, f"{name} must have the dtype of the parameters before it")
    if p.shape != (cols,):
        raise CameError(CAME_ERR_SHAPE, f"{name} must have {cols} elements")
    if not p.is_contiguous():
        raise CameError(CAME_ERR_UNSUPPORTED, f"{name} must be contiguous")
    return p.data_ptr(), mine


def _norm_stats(s, name, rows, index):
    """Address of the rows' means or reciprocal deviations."""
    if s.get_device() != index:
        raise CameError(CAME_ERR_DEVICE, f"{name} must be on the GPU of x")
    if s.dtype != _torch().float32:
        raise CameError(CAME_ERR_DTYPE, f"{name} must be fp32")
    if s.numel() != rows or not s.is_contiguous():
        raise CameError(CAME_ERR_SHAPE, f"{name} must be contiguous and have one element per row")
    return s.data_ptr()


def _layernorm_forward_call(l, index, stream):
    status = _lib.came_layernorm_forward_packed(l, index, stream)
    if status:
        _check(status)


def _layernorm_backward_call(l, workspace, size, index, stream):
    status = _lib.came_layernorm_backward_packed(l, workspace, size, index, stream)
    if status:
        _check(status)


def layer_norm_forward(x, weight=None, bias=None, eps: float = 1e-5, out=None, out_dtype=None, stats: bool = True):
    """``(y, mean, rstd)`` with ``y = (x - mean) * rstd * weight + bias`` over the last dimension, ``rstd`` =
    1 / sqrt(variance + eps).

    ``x``: fp32 or bf16 CUDA tensor of any shape whose rows (the last dimension) are contiguous and lie at one stride;
    ``weight``, ``bias``: contiguous, as long as a row, fp32 or bf16 (both the same), or None.  ``out``: tensor of x's
    shape, made here (of type ``out_dtype``, x's when that is None too) when it is None.  ``mean`` and ``rstd`` are fp32,
    one for each row, in the shape of x without its last dimension; with ``stats`` false they are not written and
    ``y`` alone is returned (inference).  No autograd: see ``layer_norm``."""
    _refuse_tangents(x, weight, bias)
    torch = _torch()
    if _lib is None:
        load()
    index = x.get_device()
    if index < 0:
        raise CameError(CAME_ERR_DEVICE, "x must be a CUDA tensor")
    rows, x_ld, x_code = _rows_of(x, "x", None, index)
    shape = x.shape
    cols = shape[-1]
    w_at = b_at = 0
    w_code = None
    if weight is not None:
        w_at, w_code = _norm_param(weight, "weight", cols, index, None)
    if bias is not None:
        b_at, w_code = _norm_param(bias, "bias", cols, index, w_code)
    if out is None:
        out = x.new_empty(shape, dtype=out_dtype)
        y_ld, y_code = cols, _DTYPE_CODES.get(out.dtype)
        if y_code is None:
            y_code = _dtype_code(out, "out")
    else:
        if out_dtype is not None and out.dtype != out_dtype:
            raise CameError(CAME_ERR_DTYPE, f"out is {out.dtype}, not {out_dtype}")
        _, y_ld, y_code = _rows_of(out, "out", shape, index)
    if stats:
        mean, rstd = x.new_empty(shape[:-1], dtype=torch.float32), x.new_empty(shape[:-1], dtype=torch.float32)
        mean_at, rstd_at = mean.data_ptr(), rstd.data_ptr()
    else:
        mean_at = rstd_at = 0
    l = _pack_layernorm(x.data_ptr(), w_at, b_at, out.data_ptr(), 0, 0, 0, 0, mean_at, rstd_at, rows, cols, x_ld, y_ld, 0, eps,
                        x_code, y_code, 0, w_code or 0, 0, 0)
    _call_on(index, _layernorm_forward_call, l)
    return (out, mean, rstd) if stats else out


def layer_norm_backward(grad_out, x, mean, rstd, weight=None, grad_x=None, grad_weight=None, grad_bias=None,
                        accumulate: bool = False, need_x: bool = True):
    """The gradient of x, in ``grad_x`` (made here, of x's type, when it is None; nothing with ``need_x`` false).

    ``grad_out``, ``x``: fp32 or bf16, of the same shape; ``mean``, ``rstd``: as ``layer_norm_forward`` gave
    them.  ``grad_weight``, ``grad_bias``: buffers of a row's length, in the weight's type (without a weight: fp32 or bf16,
    both the same), which receive the sums over all rows, or to which these are added with ``accumulate``; None: not
    wanted.  Returns ``grad_x``.  Bit-reproducible."""
    _refuse_tangents(grad_out, x, mean, rstd, weight)
    torch = _torch()
    if _lib is None:
        load()
    index = x.get_device()
    if index < 0:
        raise CameError(CAME_ERR_DEVICE, "x must be a CUDA tensor")
    rows, x_ld, x_code = _rows_of(x, "x", None, index)
    shape = x.shape
    cols = shape[-1]
    _, y_ld, y_code = _rows_of(grad_out, "grad_out", shape, index)
    mean_at, rstd_at = _norm_stats(mean, "mean", rows, index), _norm_stats(rstd, "rstd", rows, index)
    w_at = dw_at = db_at = dx_at = dx_ld = dx_code = 0
    w_code = None
    if weight is not None:
        w_at, w_code = _norm_param(weight, "weight", cols, index, None)
    if grad_weight is not None:
        dw_at, w_code = _norm_param(grad_weight, "grad_weight", cols, index, w_code)
    if grad_bias is not None:
        db_at, w_code = _norm_param(grad_bias, "grad_bias", cols, index, w_code)
    if grad_x is not None:
        _, dx_ld, dx_code = _rows_of(grad_x, "grad_x", shape, index)
        dx_at = grad_x.data_ptr()
    elif need_x:
        grad_x = x.new_empty(shape)
        dx_at, dx_ld, dx_code = grad_x.data_ptr(), cols, x_code
    l = _pack_layernorm(x.data_ptr(), w_at, 0, 0, grad_out.data_ptr(), dx_at, dw_at, db_at, mean_at, rstd_at, rows, cols,
                        x_ld, y_ld, dx_ld, 0.0, x_code, y_code, dx_code, w_code or 0, CAME_LAYERNORM_ACCUMULATE if accumulate else 0, 0)
    out = ctypes.c_int64()
    status = _lib.came_layernorm_workspace_packed(l, out)
    if status:
        _check(status)
    size = out.value
    # from torch's allocator, for the device's current stream: not reused before the call is done
    ws = x.new_empty((size + 3) // 4, dtype=torch.float32)
    _call_on(index, _layernorm_backward_call, l, ws.data_ptr(), size)
    return grad_x


_layer_norm_class = None


def _layer_norm_function():
    """Layer norm as an autograd function."""
    global _layer_norm_class
    if _layer_norm_class is None:
        torch = _torch()

        class LayerNorm(torch.autograd.Function):
            @staticmethod
            def forward(ctx, x, weight, bias, eps, out_dtype):
                y, mean, rstd = layer_norm_forward(x, weight, bias, eps, out_dtype=out_dtype)
                ctx.save_for_backward(x, weight, mean, rstd)
                ctx.bias_like = None if bias is None else (bias.shape, bias.dtype)
                return y

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, grad_out):
                x, weight, mean, rstd = ctx.saved_tensors
                need_x, need_w, need_b = ctx.needs_input_grad[:3]
                new = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=x.device)  # noqa: E731
                dw = new(weight.shape, weight.dtype) if need_w else None
                db = new(*ctx.bias_like) if need_b else None
                dx = layer_norm_backward(grad_out.contiguous(), x, mean, rstd, weight, grad_weight=dw, grad_bias=db, need_x=need_x)
                return dx, dw, db, None, None

        _layer_norm_class = LayerNorm
    return _layer_norm_class


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5, out_dtype=None):
    """``layer_norm_forward``'s y as part of autograd's graph (once differentiable): gradients of ``x``, ``weight`` and
    ``bias``, each in its own type.  When nothing requires grad, or grad mode is off, y alone is computed.

    (Of autograd in general: before a backward pass is captured into a CUDA graph, eager graphs of the same leaves
    have to be gone; torch ends the process otherwise.)"""
    if _torch().is_grad_enabled() and (x.requires_grad or (weight is not None and weight.requires_grad) or (bias is not None and bias.requires_grad)):
        _refuse_tangents(x, weight, bias)
        return _layer_norm_function().apply(x, weight, bias, eps, out_dtype)
    return layer_norm_forward(x, weight, bias, eps, out_dtype=out_dtype, stats=False)


# --- relative position bias ----------------------------------------------------------------------

_pack_posbias = struct.Struct("3P8q5iI").pack
_posbias_class = None


def _posbias_forward_call(p, index, stream):
    status = _lib.came_posbias_forward_packed(p, index, stream)
    if status:
        _check(status)


def _posbias_backward_call(p, workspace, size, index, stream):
    status = _lib.came_posbias_backward_packed(p, workspace, size, index, stream)
    if status:
        _check(status)


def _offset_of(offset, index):
    """(address of an offset on the device, offset on the host)."""
    if isinstance(offset, int):
        if not -1 << 40 <= offset <= 1 << 40:
            raise CameError(CAME_ERR_SHAPE, "offset must lie in [-2^40, 2^40]")
        return 0, offset
    torch = _torch()
    if not isinstance(offset, torch.Tensor) or offset.dtype != torch.int64 or offset.numel() != 1:
        raise CameError(CAME_ERR_DTYPE, "offset must be a whole number, or a CUDA tensor of one int64")
    if offset.get_device() != index:
        raise CameError(CAME_ERR_DEVICE, "offset must be on the table's GPU")
    return offset.data_ptr(), 0


def _check_distance(max_distance) -> None:
    """What the packed descriptor can hold (the library looks at the rest)."""
    try:
        fits = 0 <= operator.index(max_distance) <= 1 << 29
    except TypeError:
        fits = False
    if not fits:
        raise CameError(CAME_ERR_HPARAM, "max_distance must be a whole number, up to 2^29")


def _position_bias_function():
    """The bias as an autograd function."""
    global _posbias_class
    if _posbias_class is None:
        torch = _torch()

        class PositionBias(torch.autograd.Function):
            @staticmethod
            def forward(ctx, table, q_len, k_len, offset, bidirectional, max_distance, out_dtype):
                # (an offset on the device is copied: the caller may have counted on when the gradient is computed)
                ctx.offset = offset if isinstance(offset, int) else offset.clone()
                ctx.bidirectional, ctx.max_distance, ctx.shape, ctx.dtype = bidirectional, max_distance, table.shape, table.dtype
                return position_bias_forward(table, q_len, k_len, offset, bidirectional, max_distance, out_dtype=out_dtype)

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, grad_out):
                if grad_out.stride(-1) != 1:
                    grad_out = grad_out.contiguous()
                grad = grad_out.new_empty(ctx.shape, dtype=ctx.dtype)
                return (position_bias_backward(grad_out, grad, ctx.offset, ctx.bidirectional, ctx.max_distance),) + (None,) * 6

        _posbias_class = PositionBias
    return _posbias_class


def position_bias_forward(table, q_len: int, k_len: int, offset=0, bidirectional: bool = True, max_distance: int = 128,
                          out=None, out_dtype=None):
    """``out[h, i, j] = table[bucket(j - i - offset), h]``, shape ``(heads, q_len, k_len)``: a number to add to the scores
    of query i and key j (the buckets: see ``include/came_b200.h``).

    ``table``: fp32 or bf16 CUDA matrix ``(buckets, heads)`` with contiguous rows.  ``offset``: the position of query 0 among
    the keys, a whole number or a CUDA tensor of one int64 that the kernel reads (captured decoding).  ``bidirectional``: half
    of the buckets for keys behind the query; else such keys count as distance 0.  ``out``: contiguous, fp32 or bf16,
    made here (of type ``out_dtype``, the table's when that is None too) when it is None.

    When autograd records and the table requires grad, the result carries the graph: the table's gradient is
    ``position_bias_backward``'s, in its type (once differentiable).  ``out`` must be None then."""
    _refuse_tangents(table)
    if _lib is None:
        load()
    if table.requires_grad and _torch().is_grad_enabled():
        if out is not None:
            raise CameError(CAME_ERR_UNSUPPORTED, "a table that requires grad takes no out: detach it, or disable grad mode")
        return _position_bias_function().apply(table, q_len, k_len, offset, bidirectional, max_distance, out_dtype)
    buckets, heads, ld, code, index = _embed_table(table, "table")
    offset_at, offset = _offset_of(offset, index)
    _check_distance(max_distance)
    if out is None:
        if not (0 <= q_len <= 1 << 30 and 0 <= k_len <= 1 << 30) or heads * q_len * k_len > 1 << 40:
            raise CameError(CAME_ERR_SHAPE, "q_len and k_len must lie in [0, 2^30], all elements together 2^40")
        out = table.new_empty((heads, q_len, k_len), dtype=out_dtype)
    else:
        if out_dtype is not None and out.dtype != out_dtype:
            raise CameError(CAME_ERR_DTYPE, f"out is {out.dtype}, not {out_dtype}")
        if out.get_device() != index:
            raise CameError(CAME_ERR_DEVICE, "out must be on the table's GPU")
        if out.shape != (heads, q_len, k_len):
            raise CameError(CAME_ERR_SHAPE, f"out must have the shape {(heads, q_len, k_len)}")
        if not out.is_contiguous():
            raise CameError(CAME_ERR_UNSUPPORTED, "out must be contiguous")
    out_code = _DTYPE_CODES.get(out.dtype)
    if out_code is None:
        raise CameError(CAME_ERR_DTYPE, f"out must be fp32 or bf16, got {out.dtype}")
    p = _pack_posbias(table.data_ptr(), out.data_ptr(), offset_at, offset, q_len, k_len, 0, ld, 0, 0, 0, heads, buckets,
                      max_distance, code, out_code, CAME_POSBIAS_BIDIRECTIONAL if bidirectional else 0)
    _call_on(index, _posbias_forward_call, p)
    return out


def position_bias_backward(grad_out, grad, offset=0, bidirectional: bool = True, max_distance: int = 128,
                           accumulate: bool = False):
    """``grad[b, h]`` = the sum of ``grad_out`` over all queries and keys (and the batch) of head h with bucket b; with
    ``accumulate`` the sums are added to ``grad``.

    ``grad_out``: fp32 or bf16, ``(heads, q_len, k_len)`` or ``(batch, heads, q_len, k_len)`` (a bias that was added to a
    batch of scores), with any strides but a contiguous last dimension; ``grad``: fp32 or bf16 ``(buckets, heads)``.
    Returns ``grad``.  Bit-reproducible."""
    _refuse_tangents(grad_out)
    if _lib is None:
        load()
    buckets, heads, ld, code, index = _embed_table(grad, "grad")
    offset_at, offset = _offset_of(offset, index)
    _check_distance(max_distance)
    if grad_out.get_device() != index:
        raise CameError(CAME_ERR_DEVICE, "grad_out must be on the table's GPU")
    data_code = _DTYPE_CODES.get(grad_out.dtype)
    if data_code is None:
        raise CameError(CAME_ERR_DTYPE, f"grad_out must be fp32 or bf16, got {grad_out.dtype}")
    shape, strides = grad_out.shape, grad_out.stride()
    if len(shape) == 3:
        shape, strides = (1, *shape), (0, *strides)
    if len(shape) != 4 or shape[1] != heads:
        raise CameError(CAME_ERR_SHAPE, "grad_out must be (heads, q_len, k_len) or (batch, heads, q_len, k_len), with the heads of grad")
    if strides[3] != 1 and shape[3] > 1:
        raise CameError(CAME_ERR_UNSUPPORTED, "the last dimension of grad_out must be contiguous")
    flags = (CAME_POSBIAS_BIDIRECTIONAL if bidirectional else 0) | (CAME_POSBIAS_ACCUMULATE if accumulate else 0)
    p = _pack_posbias(grad.data_ptr(), grad_out.data_ptr(), offset_at, offset, shape[2], shape[3], shape[0], ld, *strides[:3], heads, buckets,
                      max_distance, code, data_code, flags)
    out = ctypes.c_int64()
    status = _lib.came_posbias_workspace_packed(p, out)
    if status:
        _check(status)
    size = out.value
    # from torch's allocator, for the device's current stream: not reused before the call is done
    ws = grad.new_empty((size + 3) // 4, dtype=_torch().float32)
    _call_on(index, _posbias_backward_call, p, ws.data_ptr(), size)
    return grad
