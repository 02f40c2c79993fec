"""ctypes binding of libddp_gfx950.so.

One Python function per C entry point of include/ddp_gfx950.h, with the same
name.  The functions only marshal arguments (lists / numpy arrays -> C arrays)
and turn negative status codes into DdpError; every step of the path runs in
the library's HIP kernels.  There is no fallback: if the shared library has not
been built, importing this module raises.
"""
from __future__ import annotations

import ctypes as C
import os
from operator import index as _index
from typing import Optional, Sequence

import numpy as np

# The process must hold a single HIP runtime.  PyTorch ships its own copy of
# libamdhip64 under the same SONAME; importing torch first makes the dynamic
# linker resolve this library's dependency to that already-loaded copy, so that
# the stream handles torch hands out are valid inside the library.
try:  # pragma: no cover - torch is present wherever a GPU is used
    import torch  # noqa: F401
except Exception:  # torch missing: the system runtime is used
    pass

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libddp_gfx950.so")

DDP_OK = 0
DDP_ERR_ARG, DDP_ERR_STATE, DDP_ERR_ALREADY_READY = -1, -2, -3
DDP_ERR_HIP, DDP_ERR_NO_DEVICE, DDP_ERR_UNSUPPORTED = -4, -5, -6
DDP_FP32, DDP_FP16, DDP_BF16 = 0, 1, 2
DDP_MAX_REPLICAS = 64
DDP_DEVICE_NONE = -1
DDP_CAP_WHOLE_MODEL = (1 << 64) - 1
DDP_OPT_PIPELINE, DDP_OPT_WRITE_ALL, DDP_OPT_TIMING = 1, 2, 3
DDP_OPT_NONTEMPORAL = 5
DDP_OPT_EMIT_BUSY_BLOCKS = 8
DDP_OPT_COALESCE, DDP_OPT_FIND_UNUSED, DDP_OPT_REDUCE_STREAMS = 10, 11, 12
DDP_OPT_REDUCE_BLOCKS_PER_CU, DDP_OPT_REDUCE_CAP_MIN_BYTES = 13, 14
DDP_OPT_ACCUMULATE_BLOCKS_PER_CU, DDP_OPT_TAIL_ON_BACKWARD = 16, 17
DDP_OPT_FLAG_ORDER, DDP_OPT_GATE_WAIT_US, DDP_OPT_LAUNCH_HOLD, DDP_OPT_CHAIN_LAUNCHES = 18, 19, 21, 22
DDP_STAT_REPAIRED_LAUNCHES, DDP_STAT_EARLY_LAUNCHES = 100, 101
DDP_PIPELINE_STAGED, DDP_PIPELINE_FUSED = 0, 1
DDP_STATIC_SCRATCH_BYTES = 32 << 20
DDP_STATE_FP32, DDP_STATE_8BIT = 0, 1
DDP_SCORE_SOFTMAX, DDP_SCORE_SIGMOID = 0, 1
DDP_K_PACK, DDP_K_REDUCE, DDP_K_UNPACK, DDP_K_ACCUMULATE, DDP_K_ITERATION = 0, 1, 2, 3, 4

EXPORTS = [
    "ddp_version", "ddp_last_error", "ddp_create", "ddp_destroy", "ddp_set_option", "ddp_get_option",
    "ddp_register_params", "ddp_set_outputs", "ddp_build_buckets", "ddp_rebuild_buckets", "ddp_get_ready_order",
    "ddp_get_assignment",
    "ddp_get_bucket_info", "ddp_get_bucket_ptr", "ddp_mark_ready", "ddp_mark_ready_local",
    "ddp_get_global_used",
    "ddp_mark_ready_many", "ddp_finalize_backward", "ddp_synchronize",
    "ddp_get_launch_log", "ddp_no_sync_accumulate", "ddp_get_used_map",
    "ddp_synth_backward", "ddp_get_kernel_times", "ddp_sync_static",
    "ddp_opt_state_layout", "ddp_opt_create", "ddp_opt_destroy", "ddp_opt_last_error", "ddp_opt_register",
    "ddp_opt_set_groups", "ddp_opt_set_copies", "ddp_opt_set_state", "ddp_opt_grad_norm", "ddp_opt_adamw_step",
    "ddp_opt_read_state",
    "ddp_embedding_create", "ddp_embedding_destroy", "ddp_embedding_last_error", "ddp_embedding_lookup",
    "ddp_embedding_grad",
    "ddp_layernorm_create", "ddp_layernorm_destroy", "ddp_layernorm_last_error", "ddp_layernorm_forward",
    "ddp_layernorm_backward",
    "ddp_position_bias_create", "ddp_position_bias_destroy", "ddp_position_bias_last_error", "ddp_position_bias_buckets",
    "ddp_position_bias_apply", "ddp_position_bias_grad",
    "ddp_router_create", "ddp_router_destroy", "ddp_router_last_error", "ddp_router_route", "ddp_router_grad",
    "ddp_router_balance",
]


class DdpError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"ddp error {code}: {message}")
        self.code = code


if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python paper_2006_15704_amd/build.py` "
        "(there is no fallback implementation)")

_lib = C.CDLL(LIB_PATH)


def _refuse_stale_library() -> None:
    """The library carries a digest of the sources it was compiled from; if the
    sources next to it have changed since, results would silently describe old
    code."""
    from . import build as _build
    _lib.ddp_version.restype = C.c_char_p
    have = _lib.ddp_version().decode().rsplit("ddp-src-hash:", 1)[-1]
    want = _build.source_hash()
    if have != want:
        raise ImportError(
            f"{LIB_PATH} was built from other sources (digest {have}, sources on disk {want}): "
            "rebuild it with `python paper_2006_15704_amd/build.py`")


_refuse_stale_library()

_vp, _i32, _i64, _u64 = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64
_lib.ddp_version.restype = C.c_char_p
_lib.ddp_last_error.restype = C.c_char_p
_lib.ddp_last_error.argtypes = [_vp]
_lib.ddp_create.argtypes = [C.POINTER(_vp), _i32, _i32, _vp, _vp]
_lib.ddp_destroy.argtypes = [_vp]
_lib.ddp_set_option.argtypes = [_vp, _i32, _i64]
_lib.ddp_get_option.argtypes = [_vp, _i32, C.POINTER(_i64)]
_lib.ddp_register_params.argtypes = [_vp, _i32, C.POINTER(_i64), C.POINTER(_i32), C.POINTER(_vp)]
_lib.ddp_set_outputs.argtypes = [_vp, C.POINTER(_vp)]
_lib.ddp_build_buckets.argtypes = [_vp, _u64]
_lib.ddp_rebuild_buckets.argtypes = [_vp, _u64]
_lib.ddp_get_ready_order.argtypes = [_vp, _i32, C.POINTER(_i32), _i32, C.POINTER(_i32)]
_lib.ddp_get_assignment.argtypes = [_vp, C.POINTER(_i32), C.POINTER(_i64)]
_lib.ddp_get_bucket_info.argtypes = [_vp, _i32, C.POINTER(_i64), C.POINTER(_i32), C.POINTER(_i32)]
_lib.ddp_get_bucket_ptr.argtypes = [_vp, _i32, _i32, C.POINTER(_vp)]
_lib.ddp_mark_ready.argtypes = [_vp, _i32]
_lib.ddp_mark_ready_local.argtypes = [_vp, _i32, C.POINTER(C.c_uint8)]
_lib.ddp_get_global_used.argtypes = [_vp, C.POINTER(C.c_uint8)]
_lib.ddp_mark_ready_many.argtypes = [_vp, C.POINTER(_i32), _i32]
_lib.ddp_finalize_backward.argtypes = [_vp]
_lib.ddp_synchronize.argtypes = [_vp]
_lib.ddp_get_launch_log.argtypes = [_vp, _i32, C.POINTER(_i32), C.POINTER(_i32), _i32, C.POINTER(_i32)]
_lib.ddp_no_sync_accumulate.argtypes = [_vp, C.POINTER(_vp)]
_lib.ddp_get_used_map.argtypes = [_vp, _i32, C.POINTER(C.c_uint8)]
_lib.ddp_synth_backward.argtypes = [_vp, C.POINTER(_i32), _i32, C.POINTER(_i64), C.POINTER(_vp), _i32]
_lib.ddp_get_kernel_times.argtypes = [_vp, _i32, C.POINTER(C.c_float), C.POINTER(_i32), _i32, C.POINTER(_i32)]
_lib.ddp_sync_static.argtypes = [_i32, _i32, _vp, _i32, C.POINTER(_i64), C.POINTER(_i32), C.POINTER(_vp), _u64]
_f32, _f64 = C.c_float, C.c_double
_lib.ddp_opt_last_error.restype = C.c_char_p
_lib.ddp_opt_last_error.argtypes = [_vp]
_lib.ddp_opt_state_layout.argtypes = [_i32, C.POINTER(_i64), _i32, C.POINTER(_i64), C.POINTER(_i64)]
_lib.ddp_opt_create.argtypes = [C.POINTER(_vp), _i32, _vp]
_lib.ddp_opt_destroy.argtypes = [_vp]
_lib.ddp_opt_register.argtypes = [_vp, _i32, C.POINTER(_i64), C.POINTER(_i32), C.POINTER(_vp), C.POINTER(_i32),
                                  C.POINTER(_vp)]
_lib.ddp_opt_set_groups.argtypes = [_vp, C.POINTER(_f32), C.POINTER(_f32)]
_lib.ddp_opt_set_copies.argtypes = [_vp, C.POINTER(_i32), C.POINTER(_vp)]
_lib.ddp_opt_set_state.argtypes = [_vp, _i32, _vp, _i64]
_lib.ddp_opt_grad_norm.argtypes = [_vp, _f64, C.POINTER(C.c_uint8), _vp]
_lib.ddp_opt_adamw_step.argtypes = [_vp] + [_f64] * 7 + [_i32, C.POINTER(C.c_uint8)]
_lib.ddp_opt_read_state.argtypes = [_vp, _vp, _vp]
_lib.ddp_embedding_last_error.restype = C.c_char_p
_lib.ddp_embedding_last_error.argtypes = [_vp]
_lib.ddp_embedding_create.argtypes = [C.POINTER(_vp), _i32, _vp, _i64, _i64, _i64]
_lib.ddp_embedding_destroy.argtypes = [_vp]
_lib.ddp_embedding_lookup.argtypes = [_vp, _i64, _vp, _i32, _vp, _i32, _i64, _f32, _vp, _i32, _i64]
_lib.ddp_embedding_grad.argtypes = [_vp, _i64, _vp, _i32, _vp, _i32, _i64, _f32, _i64, _i32, _vp, _i32, _i64]
_lib.ddp_layernorm_last_error.restype = C.c_char_p
_lib.ddp_layernorm_last_error.argtypes = [_vp]
_lib.ddp_layernorm_create.argtypes = [C.POINTER(_vp), _i32, _vp, _i64]
_lib.ddp_layernorm_destroy.argtypes = [_vp]
_lib.ddp_layernorm_forward.argtypes = [_vp, _i64, _vp, _i32, _i64, _vp, _i64, _vp, _vp, _i32, _f32, _vp, _i64, _vp, _i32, _i64, _vp, _vp]
_lib.ddp_layernorm_backward.argtypes = [_vp, _i64, _vp, _i32, _i64, _vp, _i32, _i64, _vp, _vp, _vp, _i32, _vp, _i64, _vp, _i64, _i32,
                                        _vp, _vp, _i32]
_lib.ddp_position_bias_last_error.restype = C.c_char_p
_lib.ddp_position_bias_last_error.argtypes = [_vp]
_lib.ddp_position_bias_create.argtypes = [C.POINTER(_vp), _i32, _vp, _i32, _i32, _i32, _i64, _i32]
_lib.ddp_position_bias_destroy.argtypes = [_vp]
_lib.ddp_position_bias_buckets.argtypes = [_vp, C.POINTER(_i32)]
_lib.ddp_position_bias_apply.argtypes = [_vp, _i64, _i64, _i64, _i64, _vp, _i32, _i64, _f32, _vp, _i32, _f32, _i32, _vp, _i32, _i64,
                                         _i64, _i64]
_lib.ddp_position_bias_grad.argtypes = [_vp, _i64, _i64, _i64, _i64, _vp, _i32, _i64, _i64, _i64, _f32, _vp, _vp, _i32, _i32, _vp, _i32,
                                        _i64]
_lib.ddp_router_last_error.restype = C.c_char_p
_lib.ddp_router_last_error.argtypes = [_vp]
_lib.ddp_router_create.argtypes = [C.POINTER(_vp), _i32, _vp] + [_i32] * 7 + [_f32]
_lib.ddp_router_destroy.argtypes = [_vp]
_lib.ddp_router_route.argtypes = [_vp, _i64, _vp, _i32, _i64, _vp, _vp, _vp, _i32, _vp, _i32]
_lib.ddp_router_grad.argtypes = [_vp, _i64, _vp, _i32, _i64, _vp, _vp, _i32, _vp, _i64]
_lib.ddp_router_balance.argtypes = [_vp, _i32, _vp, _f32, _vp, _vp]
for _name in EXPORTS:
    if not _name.endswith("_last_error") and _name != "ddp_version":
        getattr(_lib, _name).restype = _i32


def _check(ctx, status: int) -> int:
    if status < 0:
        msg = _lib.ddp_last_error(ctx)
        raise DdpError(status, msg.decode() if msg else "")
    return status


def _i32_array(values) -> np.ndarray:
    return np.ascontiguousarray(values, dtype=np.int32)


def _i64_array(values) -> np.ndarray:
    return np.ascontiguousarray(values, dtype=np.int64)


def _ptr_array(values) -> np.ndarray:
    """Device addresses (ints, None = NULL) -> contiguous uint64 array."""
    return np.ascontiguousarray([0 if v is None else int(v) for v in values], dtype=np.uint64)


def _as(arr: np.ndarray, ctype):
    return arr.ctypes.data_as(C.POINTER(ctype))


def ddp_version() -> str:
    return _lib.ddp_version().decode()


def ddp_last_error(ctx) -> str:
    msg = _lib.ddp_last_error(ctx)
    return msg.decode() if msg else ""


_replicas = {}      # context address -> R, for checking array lengths before they cross the C ABI
_nparams = {}       # context address -> n


def ddp_create(R: int, device: int, reduce_stream: int = 0, backward_stream: int = 0):
    """Returns the opaque context handle.  Streams are raw hipStream_t values
    (torch.cuda.Stream.cuda_stream)."""
    handle = _vp()
    _check(None, _lib.ddp_create(C.byref(handle), R, device, _vp(reduce_stream or None),
                                 _vp(backward_stream or None)))
    _replicas[handle.value] = int(R)
    _nparams.pop(handle.value, None)
    return handle


def ddp_destroy(ctx) -> None:
    _replicas.pop(ctx.value, None)
    _nparams.pop(ctx.value, None)
    _check(ctx, _lib.ddp_destroy(ctx))


def ddp_set_option(ctx, option: int, value: int) -> None:
    _check(ctx, _lib.ddp_set_option(ctx, option, value))


def ddp_get_option(ctx, option: int) -> int:
    value = _i64()
    _check(ctx, _lib.ddp_get_option(ctx, option, C.byref(value)))
    return value.value


def ddp_register_params(ctx, numel: Sequence[int], dtype: Sequence[int],
                        grad_ptrs: Optional[Sequence[int]]) -> None:
    """grad_ptrs: flat sequence of R*n device addresses, [r][i] row-major."""
    ne, dt = _i64_array(numel), _i32_array(dtype)
    if grad_ptrs is None:
        gp = None
    else:
        arr = _ptr_array(grad_ptrs)
        gp = _as(arr, _vp)
    _check(ctx, _lib.ddp_register_params(ctx, len(ne), _as(ne, _i64), _as(dt, _i32), gp))
    _nparams[ctx.value] = len(ne)


def ddp_set_outputs(ctx, out_ptrs: Optional[Sequence[int]]) -> None:
    """out_ptrs: n device addresses of binary32 tensors that receive the averages."""
    if out_ptrs is None:
        _check(ctx, _lib.ddp_set_outputs(ctx, None))
        return
    arr = _ptr_array(out_ptrs)
    if len(arr) != _nparams.get(ctx.value, len(arr)):      # the library reads exactly n pointers
        raise ValueError(f"out_ptrs has {len(arr)} entries, {_nparams[ctx.value]} parameters are registered")
    _check(ctx, _lib.ddp_set_outputs(ctx, _as(arr, _vp)))


def ddp_build_buckets(ctx, cap_bytes: int) -> int:
    return _check(ctx, _lib.ddp_build_buckets(ctx, cap_bytes))


def ddp_get_assignment(ctx, n: int):
    bucket_of = np.zeros(n, dtype=np.int32)
    offset = np.zeros(n, dtype=np.int64)
    _check(ctx, _lib.ddp_get_assignment(ctx, _as(bucket_of, _i32), _as(offset, _i64)))
    return bucket_of, offset


def ddp_get_bucket_info(ctx, b: int):
    elems, npar, dt = _i64(), _i32(), _i32()
    _check(ctx, _lib.ddp_get_bucket_info(ctx, b, C.byref(elems), C.byref(npar), C.byref(dt)))
    return elems.value, npar.value, dt.value


def ddp_get_bucket_ptr(ctx, b: int, r: int) -> int:
    p = _vp()
    _check(ctx, _lib.ddp_get_bucket_ptr(ctx, b, r, C.byref(p)))
    return p.value or 0


# The calls made once per parameter, and those that take a list with an entry per
# parameter or tensor, go through a small CPython module (plain argument passing, a
# tenth of the interpreter time of numpy and a ctypes call); it is built together with
# the library.  A list it does not take (anything but plain ints) it leaves to the
# conversions below, by returning None.
import importlib.util as _ilu

_fast_path = os.path.join(_HERE, "_ddp_fastcall.so")
if not os.path.exists(_fast_path):
    raise ImportError(f"{_fast_path} is missing: build it with `python paper_2006_15704_amd/build.py`")
_spec = _ilu.spec_from_file_location("_ddp_fastcall", _fast_path)
_fast = _ilu.module_from_spec(_spec)
_spec.loader.exec_module(_fast)
_mark, _finalize, _mark_local, _many, _accumulate, _static = (
    C.cast(f, _vp).value for f in (_lib.ddp_mark_ready, _lib.ddp_finalize_backward, _lib.ddp_mark_ready_local,
                                   _lib.ddp_mark_ready_many, _lib.ddp_no_sync_accumulate, _lib.ddp_sync_static))
_fast.bind(_mark, _finalize, _mark_local, _i32, _many, _accumulate, _static)
_fast_mark, _fast_finalize, _fast_mark_local = _fast.mark_ready, _fast.finalize_backward, _fast.mark_ready_local
_fast_many, _fast_accumulate, _fast_static = _fast.mark_ready_many, _fast.no_sync_accumulate, _fast.sync_static
_fast.bind_around(*(C.cast(f, _vp).value for f in (_lib.ddp_embedding_lookup, _lib.ddp_embedding_grad,
                                                   _lib.ddp_opt_grad_norm, _lib.ddp_opt_adamw_step)))
_fast_lookup, _fast_grad = _fast.embedding_lookup, _fast.embedding_grad
_fast_norm, _fast_step = _fast.opt_grad_norm, _fast.opt_adamw_step
_fast.bind_layer(*(C.cast(f, _vp).value for f in (
    _lib.ddp_layernorm_forward, _lib.ddp_layernorm_backward, _lib.ddp_position_bias_apply, _lib.ddp_position_bias_grad,
    _lib.ddp_router_route, _lib.ddp_router_grad, _lib.ddp_router_balance)))


def _address(ctx):
    return ctx.value if type(ctx) is _vp else None


def ddp_mark_ready(ctx, param_id: int) -> None:
    status = _fast_mark(ctx.value, param_id)
    if status < 0:
        _check(ctx, status)


def ddp_mark_ready_local(ctx, param_id: int, used) -> None:
    """used: R flags, non-zero = that replica produced a gradient for the parameter."""
    status = _fast_mark_local(ctx.value, param_id, used, _replicas)
    if status < 0:
        _check(ctx, status)


def ddp_get_global_used(ctx, n: int) -> np.ndarray:
    used = np.zeros(n, dtype=np.uint8)
    _check(ctx, _lib.ddp_get_global_used(ctx, _as(used, C.c_uint8)))
    return used


def ddp_mark_ready_many(ctx, ids) -> None:
    status = _fast_many(_address(ctx), ids)
    if status is not None:
        if status < 0:
            _check(ctx, status)
        return
    arr = _i32_array(ids)
    _check(ctx, _lib.ddp_mark_ready_many(ctx, _as(arr, _i32), len(arr)))


def ddp_finalize_backward(ctx) -> None:
    status = _fast_finalize(ctx.value)
    if status < 0:
        _check(ctx, status)


def ddp_synchronize(ctx) -> None:
    _check(ctx, _lib.ddp_synchronize(ctx))


def ddp_rebuild_buckets(ctx, cap_bytes: int) -> int:
    """New number of buckets; the mapping follows the closed iteration's ready order."""
    return _check(ctx, _lib.ddp_rebuild_buckets(ctx, cap_bytes))


def ddp_get_ready_order(ctx, which: int = 1):
    """Parameters in the order of their ready marks: running (0) or last closed (1) iteration."""
    n = _i32()
    _check(ctx, _lib.ddp_get_ready_order(ctx, which, None, 0, C.byref(n)))
    ids = np.zeros(max(n.value, 1), dtype=np.int32)
    _check(ctx, _lib.ddp_get_ready_order(ctx, which, _as(ids, _i32), n.value, C.byref(n)))
    return [int(x) for x in ids[: n.value]]


def ddp_get_launch_log(ctx, which: int = 1):
    """[(bucket, after_call)] of the running (0) or last closed (1) iteration."""
    n = _i32()
    _check(ctx, _lib.ddp_get_launch_log(ctx, which, None, None, 0, C.byref(n)))
    ids = np.zeros(max(n.value, 1), dtype=np.int32)
    calls = np.zeros(max(n.value, 1), dtype=np.int32)
    _check(ctx, _lib.ddp_get_launch_log(ctx, which, _as(ids, _i32), _as(calls, _i32), n.value, C.byref(n)))
    return [(int(ids[i]), int(calls[i])) for i in range(n.value)]


def ddp_no_sync_accumulate(ctx, micro_grad_ptrs: Sequence[Optional[int]]) -> None:
    address = _address(ctx)
    need = _replicas.get(address, 0) * _nparams.get(address, 0)      # the library reads that many pointers
    status = _fast_accumulate(address, micro_grad_ptrs, need)
    if status is not None:
        if status < 0:
            _check(ctx, status)
        return
    arr = _ptr_array(micro_grad_ptrs)
    if len(arr) < need:
        raise ValueError(f"micro_grad_ptrs has {len(arr)} entries, expected R*n = {need}")
    _check(ctx, _lib.ddp_no_sync_accumulate(ctx, _as(arr, _vp)))


def ddp_get_used_map(ctx, n: int, which: int = 1) -> np.ndarray:
    used = np.zeros(n, dtype=np.uint8)
    _check(ctx, _lib.ddp_get_used_map(ctx, which, _as(used, C.c_uint8)))
    return used


def ddp_synth_backward(ctx, order, delay_ns=None, src_ptrs=None, mark: bool = True) -> None:
    o = _i32_array(order)
    d = None if delay_ns is None else _i64_array(delay_ns)
    s = None if src_ptrs is None else _ptr_array(src_ptrs)
    _check(ctx, _lib.ddp_synth_backward(ctx, _as(o, _i32), len(o),
                                        None if d is None else _as(d, _i64),
                                        None if s is None else _as(s, _vp), 1 if mark else 0))


def ddp_get_kernel_times(ctx, kind: int):
    """(ms[], bucket_id[]) of the timed launches of `kind`."""
    n = _i32()
    _check(ctx, _lib.ddp_get_kernel_times(ctx, kind, None, None, 0, C.byref(n)))
    ms = np.zeros(max(n.value, 1), dtype=np.float32)
    ids = np.zeros(max(n.value, 1), dtype=np.int32)
    _check(ctx, _lib.ddp_get_kernel_times(ctx, kind, _as(ms, C.c_float), _as(ids, _i32), n.value, C.byref(n)))
    return ms[:n.value].copy(), ids[:n.value].copy()


def ddp_sync_static(R: int, device: int, stream: int, numel: Sequence[int], dtype: Sequence[int],
                    grad_ptrs: Sequence[int], cap_bytes: int) -> int:
    """One whole synchronization without a context and without device-memory
    allocation; returns the number of buckets."""
    status = _fast_static(R, device, stream, numel, dtype, grad_ptrs, cap_bytes)
    if status is not None:
        return _check(None, status)
    ne, dt, gp = _i64_array(numel), _i32_array(dtype), _ptr_array(grad_ptrs)
    if len(gp) != R * len(ne):
        raise ValueError(f"grad_ptrs has {len(gp)} entries, expected R*n = {R * len(ne)}")
    return _check(None, _lib.ddp_sync_static(R, device, _vp(stream or None), len(ne), _as(ne, _i64),
                                             _as(dt, _i32), _as(gp, _vp), cap_bytes))


# ---- around the synchronization: the optimizer ----

_opt_n = {}      # handle address -> number of tensors, for checking array lengths before they cross the C ABI


def _check_opt(opt, status: int) -> int:
    if status < 0:
        raise DdpError(status, ddp_opt_last_error(opt))
    return status


def _sized(values, n: int, what: str, convert):
    """An array of exactly n entries (the library reads that many), or None."""
    if values is None:
        return None
    arr = convert(values)
    if arr.ndim != 1 or len(arr) != n:
        raise ValueError(f"{what} has {arr.size} entries, expected {n}")
    return arr


def _pointer(address):
    return _vp(None if address is None else _index(address) or None)


def _f32_array(values) -> np.ndarray:
    return np.ascontiguousarray(values, dtype=np.float32)


def _flags(used, opt):
    if used is None:
        return None
    return _sized(used, _opt_n.get(opt.value, 0), "used", lambda u: np.ascontiguousarray(np.asarray(u) != 0, dtype=np.uint8))


def _or_null(arr, ctype):
    return None if arr is None else _as(arr, ctype)


def ddp_opt_last_error(opt) -> str:
    msg = _lib.ddp_opt_last_error(opt)
    return msg.decode() if msg else ""


def ddp_opt_state_layout(numel: Sequence[int], kind: int):
    """(element offset of every tensor, {"m", "v", "m_top", "v_top": byte offsets, "elems", "bytes"})."""
    ne = _i64_array(numel)
    offset, where = np.zeros(len(ne), dtype=np.int64), np.zeros(6, dtype=np.int64)
    _check_opt(None, _lib.ddp_opt_state_layout(len(ne), _as(ne, _i64), kind, _as(offset, _i64), _as(where, _i64)))
    return offset, dict(zip(("m", "v", "m_top", "v_top", "elems", "bytes"), (int(x) for x in where)))


def ddp_opt_create(device: int, stream: int = 0):
    """Returns the opaque handle.  stream: a raw hipStream_t value."""
    handle = _vp()
    _check_opt(None, _lib.ddp_opt_create(C.byref(handle), device, _vp(stream or None)))
    return handle


def ddp_opt_destroy(opt) -> None:
    _opt_n.pop(opt.value, None)
    _check_opt(None, _lib.ddp_opt_destroy(opt))


def ddp_opt_register(opt, numel: Sequence[int], param_dtype: Sequence[int], param_ptrs: Optional[Sequence[int]],
                     grad_dtype: Sequence[int], grad_ptrs: Optional[Sequence[int]]) -> None:
    ne = _i64_array(numel)
    n = len(ne)
    pt, gt = _sized(param_dtype, n, "param_dtype", _i32_array), _sized(grad_dtype, n, "grad_dtype", _i32_array)
    pp, gp = _sized(param_ptrs, n, "param_ptrs", _ptr_array), _sized(grad_ptrs, n, "grad_ptrs", _ptr_array)
    _check_opt(opt, _lib.ddp_opt_register(opt, n, _as(ne, _i64), _as(pt, _i32), _or_null(pp, _vp), _as(gt, _i32),
                                          _or_null(gp, _vp)))
    _opt_n[opt.value] = n


def ddp_opt_set_groups(opt, lr_scale: Optional[Sequence[float]] = None,
                       decay_scale: Optional[Sequence[float]] = None) -> None:
    n = _opt_n.get(opt.value, 0)
    lr, decay = _sized(lr_scale, n, "lr_scale", _f32_array), _sized(decay_scale, n, "decay_scale", _f32_array)
    _check_opt(opt, _lib.ddp_opt_set_groups(opt, _or_null(lr, _f32), _or_null(decay, _f32)))


def ddp_opt_set_copies(opt, copy_dtype: Sequence[int], copy_ptrs: Sequence[Optional[int]]) -> None:
    n = _opt_n.get(opt.value, 0)
    ct, cp = _sized(copy_dtype, n, "copy_dtype", _i32_array), _sized(copy_ptrs, n, "copy_ptrs", _ptr_array)
    _check_opt(opt, _lib.ddp_opt_set_copies(opt, _or_null(ct, _i32), _or_null(cp, _vp)))


def ddp_opt_set_state(opt, kind: int, state: int, nbytes: int) -> None:
    _check_opt(opt, _lib.ddp_opt_set_state(opt, kind, _vp(state or None), nbytes))


def ddp_opt_grad_norm(opt, grad_scale: float = 1.0, norm_out: int = 0, used=None) -> None:
    status = _fast_norm(_address(opt), grad_scale, norm_out) if used is None else None
    if status is None:
        flags = _flags(used, opt)
        status = _lib.ddp_opt_grad_norm(opt, float(grad_scale), _or_null(flags, C.c_uint8), _pointer(norm_out))
    if status < 0:
        _check_opt(opt, status)


def ddp_opt_adamw_step(opt, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
                       weight_decay: float = 0.0, grad_scale: float = 1.0, max_norm: float = 0.0,
                       skip_nonfinite: bool = False, used=None) -> None:
    status = None
    if used is None:
        status = _fast_step(_address(opt), lr, beta1, beta2, eps, weight_decay, grad_scale, max_norm, skip_nonfinite)
    if status is None:
        flags = _flags(used, opt)
        hyper = [float(x) for x in (lr, beta1, beta2, eps, weight_decay, grad_scale, max_norm)]
        status = _lib.ddp_opt_adamw_step(opt, *hyper, 1 if skip_nonfinite else 0, _or_null(flags, C.c_uint8))
    if status < 0:
        _check_opt(opt, status)


def ddp_opt_read_state(opt, m_out: int, v_out: int) -> None:
    _check_opt(opt, _lib.ddp_opt_read_state(opt, m_out or None, v_out or None))


# ---- around the synchronization: the embedding ----

def _check_embedding(emb, status: int) -> int:
    if status < 0:
        raise DdpError(status, ddp_embedding_last_error(emb))
    return status


def ddp_embedding_last_error(emb) -> str:
    msg = _lib.ddp_embedding_last_error(emb)
    return msg.decode() if msg else ""


def ddp_embedding_create(device: int, stream: int, rows: int, width: int, max_tokens: int):
    """Returns the opaque handle.  max_tokens: of a ddp_embedding_grad call (0: lookups only)."""
    handle = _vp()
    _check_embedding(None, _lib.ddp_embedding_create(C.byref(handle), device, _vp(stream or None), rows, width, max_tokens))
    return handle


def ddp_embedding_destroy(emb) -> None:
    _check_embedding(None, _lib.ddp_embedding_destroy(emb))


def ddp_embedding_lookup(emb, tokens: int, ids: int, id_bits: int, table: int, table_dtype: int, table_stride: int,
                         scale: float, out: int, out_dtype: int, out_stride: int) -> None:
    status = _fast_lookup(_address(emb), tokens, ids, id_bits, table, table_dtype, table_stride, scale, out,
                          out_dtype, out_stride)
    if status is None:
        status = _lib.ddp_embedding_lookup(emb, _index(tokens), _pointer(ids), _index(id_bits), _pointer(table),
                                           _index(table_dtype), _index(table_stride), float(scale), _pointer(out),
                                           _index(out_dtype), _index(out_stride))
    if status < 0:
        _check_embedding(emb, status)


def ddp_embedding_grad(emb, tokens: int, ids: int, id_bits: int, dout: int, dout_dtype: int, dout_stride: int,
                       scale: float, padding_row: int, accumulate: bool, grad: int, grad_dtype: int,
                       grad_stride: int) -> None:
    status = _fast_grad(_address(emb), tokens, ids, id_bits, dout, dout_dtype, dout_stride, scale, padding_row,
                        accumulate, grad, grad_dtype, grad_stride)
    if status is None:
        status = _lib.ddp_embedding_grad(emb, _index(tokens), _pointer(ids), _index(id_bits), _pointer(dout),
                                         _index(dout_dtype), _index(dout_stride), float(scale), _index(padding_row),
                                         1 if accumulate else 0, _pointer(grad), _index(grad_dtype), _index(grad_stride))
    if status < 0:
        _check_embedding(emb, status)


# ---- inside a layer: norm, relative position bias, routing to experts ----
# (addresses are ints, 0 or None: NULL; binding checks as for the embedding)

def _check_layer(last_error, handle, status: int) -> int:
    if status < 0:
        raise DdpError(status, last_error(handle))
    return status


def ddp_layernorm_last_error(norm) -> str:
    msg = _lib.ddp_layernorm_last_error(norm)
    return msg.decode() if msg else ""


def ddp_layernorm_create(device: int, stream: int, width: int):
    """Returns the opaque handle."""
    handle = _vp()
    _check_layer(ddp_layernorm_last_error, None, _lib.ddp_layernorm_create(C.byref(handle), device, _vp(stream or None), width))
    return handle


def ddp_layernorm_destroy(norm) -> None:
    _check_layer(ddp_layernorm_last_error, None, _lib.ddp_layernorm_destroy(norm))


def ddp_layernorm_forward(norm, rows: int, x: int, x_dtype: int, x_stride: int, residual: int, residual_stride: int, gamma: int, beta: int,
                          param_dtype: int, eps: float, sum_: int, sum_stride: int, y: int, y_dtype: int, y_stride: int, mean: int = 0,
                          rstd: int = 0) -> None:
    status = _fast.layernorm_forward(_address(norm), rows, x, x_dtype, x_stride, residual, residual_stride, gamma, beta, param_dtype,
                                     eps, sum_, sum_stride, y, y_dtype, y_stride, mean, rstd)
    if status is None:
        status = _lib.ddp_layernorm_forward(norm, _index(rows), _pointer(x), _index(x_dtype), _index(x_stride), _pointer(residual),
                                            _index(residual_stride), _pointer(gamma), _pointer(beta), _index(param_dtype), float(eps),
                                            _pointer(sum_), _index(sum_stride), _pointer(y), _index(y_dtype), _index(y_stride),
                                            _pointer(mean), _pointer(rstd))
    if status < 0:
        _check_layer(ddp_layernorm_last_error, norm, status)


def ddp_layernorm_backward(norm, rows: int, dy: int, dy_dtype: int, dy_stride: int, x: int, x_dtype: int, x_stride: int, mean: int, rstd: int,
                           gamma: int, param_dtype: int, dsum: int, dsum_stride: int, dx: int, dx_stride: int, accumulate: bool,
                           dgamma: int, dbeta: int, grad_dtype: int) -> None:
    status = _fast.layernorm_backward(_address(norm), rows, dy, dy_dtype, dy_stride, x, x_dtype, x_stride, mean, rstd, gamma,
                                      param_dtype, dsum, dsum_stride, dx, dx_stride, accumulate, dgamma, dbeta, grad_dtype)
    if status is None:
        status = _lib.ddp_layernorm_backward(norm, _index(rows), _pointer(dy), _index(dy_dtype), _index(dy_stride), _pointer(x),
                                             _index(x_dtype), _index(x_stride), _pointer(mean), _pointer(rstd), _pointer(gamma),
                                             _index(param_dtype), _pointer(dsum), _index(dsum_stride), _pointer(dx), _index(dx_stride),
                                             1 if accumulate else 0, _pointer(dgamma), _pointer(dbeta), _index(grad_dtype))
    if status < 0:
        _check_layer(ddp_layernorm_last_error, norm, status)


def ddp_position_bias_last_error(bias) -> str:
    msg = _lib.ddp_position_bias_last_error(bias)
    return msg.decode() if msg else ""


def ddp_position_bias_create(device: int, stream: int, heads: int, buckets: int, exact: int, max_distance: int, both: bool):
    """Returns the opaque handle.  both: keys behind the query have buckets of their own."""
    handle = _vp()
    _check_layer(ddp_position_bias_last_error, None, _lib.ddp_position_bias_create(
        C.byref(handle), device, _vp(stream or None), heads, buckets, exact, max_distance, 1 if both else 0))
    return handle


def ddp_position_bias_destroy(bias) -> None:
    _check_layer(ddp_position_bias_last_error, None, _lib.ddp_position_bias_destroy(bias))


def ddp_position_bias_buckets(bias) -> np.ndarray:
    """The smallest distance of every bucket of one direction."""
    first = np.zeros(1024, dtype=np.int32)
    n = _check_layer(ddp_position_bias_last_error, bias, _lib.ddp_position_bias_buckets(bias, _as(first, _i32)))
    return first[:n]


def ddp_position_bias_apply(bias, batch: int, queries: int, keys: int, offset: int, table: int, table_dtype: int, table_stride: int,
                            scale: float, key_lengths: int, causal: bool, masked: float, accumulate: bool, out: int, out_dtype: int,
                            batch_stride: int, head_stride: int, query_stride: int) -> None:
    status = _fast.position_bias_apply(_address(bias), batch, queries, keys, offset, table, table_dtype, table_stride, scale,
                                       key_lengths, causal, masked, accumulate, out, out_dtype, batch_stride, head_stride,
                                       query_stride)
    if status is None:
        status = _lib.ddp_position_bias_apply(bias, _index(batch), _index(queries), _index(keys), _index(offset), _pointer(table),
                                              _index(table_dtype), _index(table_stride), float(scale), _pointer(key_lengths),
                                              1 if causal else 0, float(masked), 1 if accumulate else 0, _pointer(out), _index(out_dtype),
                                              _index(batch_stride), _index(head_stride), _index(query_stride))
    if status < 0:
        _check_layer(ddp_position_bias_last_error, bias, status)


def ddp_position_bias_grad(bias, batch: int, queries: int, keys: int, offset: int, dscores: int, dtype: int, batch_stride: int,
                           head_stride: int, query_stride: int, scale: float, key_lengths: int, query_lengths: int, causal: bool,
                           accumulate: bool, grad: int, grad_dtype: int, grad_stride: int) -> None:
    status = _fast.position_bias_grad(_address(bias), batch, queries, keys, offset, dscores, dtype, batch_stride, head_stride,
                                      query_stride, scale, key_lengths, query_lengths, causal, accumulate, grad, grad_dtype,
                                      grad_stride)
    if status is None:
        status = _lib.ddp_position_bias_grad(bias, _index(batch), _index(queries), _index(keys), _index(offset), _pointer(dscores),
                                             _index(dtype), _index(batch_stride), _index(head_stride), _index(query_stride), float(scale),
                                             _pointer(key_lengths), _pointer(query_lengths), 1 if causal else 0, 1 if accumulate else 0,
                                             _pointer(grad), _index(grad_dtype), _index(grad_stride))
    if status < 0:
        _check_layer(ddp_position_bias_last_error, bias, status)


def ddp_router_last_error(router) -> str:
    msg = _lib.ddp_router_last_error(router)
    return msg.decode() if msg else ""


def ddp_router_create(device: int, stream: int, experts: int, chosen: int, groups: int = 1, kept: int = 1, top: int = 1,
                      score: int = DDP_SCORE_SOFTMAX, renormalise: bool = True, scale: float = 1.0):
    """Returns the opaque handle."""
    handle = _vp()
    _check_layer(ddp_router_last_error, None, _lib.ddp_router_create(C.byref(handle), device, _vp(stream or None), experts, chosen, groups,
                                                                     kept, top, score, 1 if renormalise else 0, scale))
    return handle


def ddp_router_destroy(router) -> None:
    _check_layer(ddp_router_last_error, None, _lib.ddp_router_destroy(router))


def ddp_router_route(router, tokens: int, logits: int, dtype: int, stride: int, bias: int, experts_out: int, weights: int,
                     weights_dtype: int, counts: int = 0, accumulate: bool = False) -> None:
    status = _fast.router_route(_address(router), tokens, logits, dtype, stride, bias, experts_out, weights, weights_dtype, counts,
                                accumulate)
    if status is None:
        status = _lib.ddp_router_route(router, _index(tokens), _pointer(logits), _index(dtype), _index(stride), _pointer(bias),
                                       _pointer(experts_out), _pointer(weights), _index(weights_dtype), _pointer(counts),
                                       1 if accumulate else 0)
    if status < 0:
        _check_layer(ddp_router_last_error, router, status)


def ddp_router_grad(router, tokens: int, logits: int, dtype: int, stride: int, experts_in: int, dweights: int, dweights_dtype: int,
                    dlogits: int, dlogits_stride: int) -> None:
    status = _fast.router_grad(_address(router), tokens, logits, dtype, stride, experts_in, dweights, dweights_dtype, dlogits,
                               dlogits_stride)
    if status is None:
        status = _lib.ddp_router_grad(router, _index(tokens), _pointer(logits), _index(dtype), _index(stride), _pointer(experts_in),
                                      _pointer(dweights), _index(dweights_dtype), _pointer(dlogits), _index(dlogits_stride))
    if status < 0:
        _check_layer(ddp_router_last_error, router, status)


def ddp_router_balance(router, replicas: int, counts: int, rate: float, bias: int, bias_out: int) -> None:
    status = _fast.router_balance(_address(router), replicas, counts, rate, bias, bias_out)
    if status is None:
        status = _lib.ddp_router_balance(router, _index(replicas), _pointer(counts), float(rate), _pointer(bias), _pointer(bias_out))
    if status < 0:
        _check_layer(ddp_router_last_error, router, status)
