"""ctypes binding of the C ABI in ``include/rtopk.h`` (same names, same
argument order). Tensors are passed as raw device pointers; no arithmetic of
the method happens here."""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "librtopk.so")
_LIB: Optional[ctypes.CDLL] = None

# what include/rtopk.h declares ...
EXPORTS = ("rtopk_encode_workspace_bytes", "rtopk_aggregate_workspace_bytes", "rtopk_encode",
           "rtopk_encode_batch", "rtopk_encode_batch_device_step",
           "rtopk_aggregate", "rtopk_aggregate_update", "rtopk_aggregate_update_workspace_bytes",
           "rtopk_aggregate_update_momentum", "rtopk_aggregate_update_static",
           "rtopk_quantize_i8_workspace_bytes", "rtopk_quantize_i8",
           "rtopk_matmul_i8_workspace_bytes", "rtopk_matmul_i8",
           "rtopk_linear_i8_workspace_bytes", "rtopk_linear_i8",
           "rtopk_linear_i8_backward_workspace_bytes", "rtopk_linear_i8_backward",
           "rtopk_orthogonalize_workspace_bytes", "rtopk_orthogonalize",
           "rtopk_aggregate_update_orthogonal_workspace_bytes", "rtopk_aggregate_update_orthogonal",
           "rtopk_strerror", "rtopk_version")
# ... and include/rtopk_diag.h
DIAG_EXPORTS = ("rtopk_encode_stats", "rtopk_trace_next_encode", "rtopk_force_next_encode",
                "rtopk_diag_stream_add", "rtopk_product_plan", "rtopk_orthogonalize_plan", "rtopk_debug_checks")


class RtopkError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} (code {code})")


class EncodeStats(ctypes.Structure):
    _fields_ = [("error_flags", ctypes.c_uint32), ("path", ctypes.c_uint32),
                ("threshold_bits", ctypes.c_uint32), ("boundary_list_size", ctypes.c_uint32),
                ("count_greater", ctypes.c_uint64), ("ties_taken", ctypes.c_uint64),
                ("superset_size", ctypes.c_uint64), ("key_list_size", ctypes.c_uint64)]


class ProductPlan(ctypes.Structure):
    _fields_ = [(name, ctypes.c_uint32) for name in ("edge", "tiles", "runs")]


class OrthogonalizePlan(ctypes.Structure):
    _fields_ = [(name, ctypes.c_uint32) for name in ("narrow", "gram_edge", "gram_runs", "joined", "square_edge", "next_edge",
                                                     "two_at_a_time")]


def library_path() -> str:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Load ``librtopk.so``. There is no fallback: a missing library is an error."""
    global _LIB
    if _LIB is not None:
        return _LIB
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2005_10761_amd.build` "
            "(hipcc, gfx950). The rTop-k path has no CPU or PyTorch fallback.")
    L = ctypes.CDLL(_LIB_PATH)
    u64, u32, vp = ctypes.c_uint64, ctypes.c_uint32, ctypes.c_void_p
    L.rtopk_encode_workspace_bytes.argtypes = [u64, u64, u64, ctypes.POINTER(u64)]
    L.rtopk_encode_workspace_bytes.restype = ctypes.c_int
    L.rtopk_aggregate_workspace_bytes.argtypes = [u64, u32, u64, ctypes.POINTER(u64)]
    L.rtopk_aggregate_workspace_bytes.restype = ctypes.c_int
    L.rtopk_encode.argtypes = [vp, vp, u64, u64, u64, u64, u64, vp, vp, vp, u64, vp]
    L.rtopk_encode.restype = ctypes.c_int
    L.rtopk_encode_batch.argtypes = [u32, vp, vp, u64, u64, u64, vp, u64, vp, vp, vp, u64, vp]
    L.rtopk_encode_batch.restype = ctypes.c_int
    L.rtopk_encode_batch_device_step.argtypes = [u32, vp, vp, u64, u64, u64, vp, vp, vp, vp, vp,
                                                 u64, vp]
    L.rtopk_encode_batch_device_step.restype = ctypes.c_int
    L.rtopk_diag_stream_add.argtypes = [vp, vp, u64, vp]
    L.rtopk_diag_stream_add.restype = ctypes.c_int
    L.rtopk_debug_checks.argtypes = []
    L.rtopk_debug_checks.restype = ctypes.c_int
    L.rtopk_aggregate.argtypes = [vp, vp, u32, u64, u64, vp, vp, u64, vp]
    L.rtopk_aggregate.restype = ctypes.c_int
    L.rtopk_aggregate_update_workspace_bytes.argtypes = [u64, u32, u64, ctypes.POINTER(u64)]
    L.rtopk_aggregate_update_workspace_bytes.restype = ctypes.c_int
    L.rtopk_aggregate_update.argtypes = [vp, vp, u32, u64, u64, ctypes.c_float, ctypes.c_float,
                                         vp, vp, u64, vp]
    L.rtopk_aggregate_update.restype = ctypes.c_int
    L.rtopk_aggregate_update_static.argtypes = [vp, vp, u32, u64, u64, ctypes.c_float,
                                                ctypes.c_float, vp, vp]
    L.rtopk_aggregate_update_static.restype = ctypes.c_int
    L.rtopk_aggregate_update_momentum.argtypes = [vp, vp, u32, u64, u64, ctypes.c_float,
                                                  ctypes.c_float, ctypes.c_float, vp, vp, vp]
    L.rtopk_aggregate_update_momentum.restype = ctypes.c_int
    L.rtopk_encode_stats.argtypes = [vp, vp, ctypes.POINTER(EncodeStats)]
    L.rtopk_encode_stats.restype = ctypes.c_int
    L.rtopk_trace_next_encode.argtypes = [ctypes.c_int, vp, vp]
    L.rtopk_trace_next_encode.restype = ctypes.c_int
    L.rtopk_force_next_encode.argtypes = [ctypes.c_uint]
    L.rtopk_force_next_encode.restype = ctypes.c_int
    i32, f32, pu64 = ctypes.c_int, ctypes.c_float, ctypes.POINTER(u64)
    for name, args in {
            "rtopk_quantize_i8_workspace_bytes": [u64, u64, i32, pu64],
            "rtopk_quantize_i8": [vp, i32, u64, u64, u64, i32, vp, u64, vp, vp, u64, vp],
            "rtopk_matmul_i8_workspace_bytes": [u64, u64, u64, pu64],
            "rtopk_matmul_i8": [vp, vp, vp, vp, vp, u64, u64, u64, u64, u64, vp, i32, u64, vp, u64, vp],
            "rtopk_linear_i8_workspace_bytes": [u64, u64, u64, pu64],
            "rtopk_linear_i8": [vp, i32, u64, u64, u64, vp, vp, u64, u64, vp, vp, i32, u64, vp, u64, vp],
            "rtopk_linear_i8_backward_workspace_bytes": [u64, u64, u64, pu64],
            "rtopk_linear_i8_backward": [vp, vp, i32, u64, u64, u64, u64, u64, vp, vp, u64, vp, u64,
                                         vp, u64, vp, vp, u64, vp],
            "rtopk_orthogonalize_workspace_bytes": [u32, u64, u64, i32, pu64],
            "rtopk_orthogonalize": [u32, vp, i32, u64, u64, u64, u32, vp, f32, i32, vp, i32, u64, vp,
                                    u64, vp],
            "rtopk_aggregate_update_orthogonal_workspace_bytes": [u32, u64, u64, i32, pu64],
            "rtopk_aggregate_update_orthogonal": [u32, vp, vp, u32, u64, u64, u64, f32, f32, f32, i32, f32,
                                                  f32, u32, vp, f32, i32, vp, vp, vp, u64, vp],
            "rtopk_product_plan": [u64, u64, u64, i32, vp],
            "rtopk_orthogonalize_plan": [u32, u64, u64, i32, u32, vp, vp]}.items():
        getattr(L, name).argtypes = args
        getattr(L, name).restype = i32
    L.rtopk_strerror.argtypes = [ctypes.c_int]
    L.rtopk_strerror.restype = ctypes.c_char_p
    L.rtopk_version.argtypes = []
    L.rtopk_version.restype = ctypes.c_int
    _LIB = L
    return L


def strerror(code: int) -> str:
    return load_library().rtopk_strerror(int(code)).decode()


def version() -> int:
    return int(load_library().rtopk_version())


def encode_workspace_bytes(d: int, r: int, k: int) -> int:
    out = ctypes.c_uint64(0)
    rc = load_library().rtopk_encode_workspace_bytes(d, r, k, ctypes.byref(out))
    if rc:
        raise RtopkError(rc, "rtopk_encode_workspace_bytes")
    return int(out.value)


def aggregate_workspace_bytes(d: int, n: int, k: int) -> int:
    out = ctypes.c_uint64(0)
    rc = load_library().rtopk_aggregate_workspace_bytes(d, n, k, ctypes.byref(out))
    if rc:
        raise RtopkError(rc, "rtopk_aggregate_workspace_bytes")
    return int(out.value)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# the current stream's handle without a Stream object around it (2.8 us less in every call), where torch has it
_RAW_STREAM = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_handle(stream) -> Optional[int]:
    if stream is None:
        if _RAW_STREAM is not None:
            return _RAW_STREAM(torch.cuda.current_device()) or None
        stream = torch.cuda.current_stream()
    h = stream.cuda_stream
    return h if h else None


def _need(t: torch.Tensor, dtype, name: str) -> None:
    if not t.is_cuda or t.dtype != dtype or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous {dtype} tensor on the GPU")


def encode(grad: torch.Tensor, residual: torch.Tensor, r: int, k: int, seed: int, step: int,
           out_idx: torch.Tensor, out_val: torch.Tensor, workspace: torch.Tensor,
           stream=None) -> None:
    """rtopk_encode: enqueue one node-side step of Algorithm 1. ``residual`` is
    updated in place; ``out_idx`` (int32 storage holding uint32 values) and
    ``out_val`` receive the message."""
    _need(grad, torch.float32, "grad")
    _need(residual, torch.float32, "residual")
    _need(out_idx, torch.int32, "out_idx")
    _need(out_val, torch.float32, "out_val")
    d = grad.numel()
    if residual.numel() != d or out_idx.numel() < k or out_val.numel() < k:
        raise ValueError("residual must have d elements, out_idx/out_val at least k")
    rc = load_library().rtopk_encode(
        _ptr(grad), _ptr(residual), d, r, k, seed & (2**64 - 1), step & (2**64 - 1),
        _ptr(out_idx), _ptr(out_val), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream_handle(stream))
    if rc:
        raise RtopkError(rc, "rtopk_encode")


def encode_batch(grads, residuals, r: int, k: int, seeds, step: int, out_idx, out_val,
                 workspace: torch.Tensor, stream=None) -> None:
    """rtopk_encode_batch: one node-side step of Algorithm 1 for every member of
    a list of equally sized vectors, in shared kernel launches. ``grads``,
    ``residuals``, ``out_idx``, ``out_val`` are sequences of tensors (as for
    :func:`encode`), ``seeds`` a sequence of ints; ``workspace`` holds
    ``len(grads)`` slices of ``encode_workspace_bytes(d, r, k)`` bytes."""
    n = len(grads)
    if n < 1 or not (len(residuals) == len(seeds) == len(out_idx) == len(out_val) == n):
        raise ValueError("grads, residuals, seeds, out_idx, out_val must have the same length >= 1")
    d = grads[0].numel()
    for g, m, oi, ov in zip(grads, residuals, out_idx, out_val):
        _need(g, torch.float32, "grad")
        _need(m, torch.float32, "residual")
        _need(oi, torch.int32, "out_idx")
        _need(ov, torch.float32, "out_val")
        if g.numel() != d or m.numel() != d or oi.numel() < k or ov.numel() < k:
            raise ValueError("every member needs d gradient and residual elements and k outputs")
    vp_arr = ctypes.c_void_p * n
    seeds_arr = (ctypes.c_uint64 * n)(*[s & (2**64 - 1) for s in seeds])
    rc = load_library().rtopk_encode_batch(
        n, vp_arr(*[_ptr(t) for t in grads]), vp_arr(*[_ptr(t) for t in residuals]), d, r, k,
        seeds_arr, step & (2**64 - 1), vp_arr(*[_ptr(t) for t in out_idx]),
        vp_arr(*[_ptr(t) for t in out_val]), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream_handle(stream))
    if rc:
        raise RtopkError(rc, "rtopk_encode_batch")


def encode_batch_device_step(grads, residuals, r: int, k: int, seeds, step_device: torch.Tensor,
                             out_idx, out_val, workspace: torch.Tensor, stream=None) -> None:
    """rtopk_encode_batch_device_step: as :func:`encode_batch`, with the step
    number read from ``step_device`` (one int64 on the GPU) when the kernels run."""
    n = len(grads)
    if n < 1 or not (len(residuals) == len(seeds) == len(out_idx) == len(out_val) == n):
        raise ValueError("grads, residuals, seeds, out_idx, out_val must have the same length >= 1")
    _need(step_device, torch.int64, "step_device")
    d = grads[0].numel()
    for g, m, oi, ov in zip(grads, residuals, out_idx, out_val):
        _need(g, torch.float32, "grad")
        _need(m, torch.float32, "residual")
        _need(oi, torch.int32, "out_idx")
        _need(ov, torch.float32, "out_val")
        if g.numel() != d or m.numel() != d or oi.numel() < k or ov.numel() < k:
            raise ValueError("every member needs d gradient and residual elements and k outputs")
    vp_arr = ctypes.c_void_p * n
    seeds_arr = (ctypes.c_uint64 * n)(*[s & (2**64 - 1) for s in seeds])
    rc = load_library().rtopk_encode_batch_device_step(
        n, vp_arr(*[_ptr(t) for t in grads]), vp_arr(*[_ptr(t) for t in residuals]), d, r, k,
        seeds_arr, _ptr(step_device), vp_arr(*[_ptr(t) for t in out_idx]),
        vp_arr(*[_ptr(t) for t in out_val]), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _stream_handle(stream))
    if rc:
        raise RtopkError(rc, "rtopk_encode_batch_device_step")


def diag_stream_add(grad: torch.Tensor, residual: torch.Tensor, stream=None) -> None:
    """rtopk_diag_stream_add: residual += grad, streamed as the encoder's dominant kernel streams."""
    _need(grad, torch.float32, "grad")
    _need(residual, torch.float32, "residual")
    if grad.numel() != residual.numel():
        raise ValueError("grad and residual must have the same length")
    rc = load_library().rtopk_diag_stream_add(_ptr(grad), _ptr(residual), grad.numel(),
                                              _stream_handle(stream))
    if rc:
        raise RtopkError(rc, "rtopk_diag_stream_add")


def aggregate(idx: torch.Tensor, val: torch.Tensor, n: int, k: int, out: torch.Tensor,
              workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """rtopk_aggregate: enqueue the master's averaging step. ``idx``/``val`` hold
    the n messages back to back; ``out`` (d elements) is fully overwritten."""
    _need(idx, torch.int32, "idx")
    _need(val, torch.float32, "val")
    _need(out, torch.float32, "out")
    if idx.numel() < n * k or val.numel() < n * k:
        raise ValueError("idx/val must hold n*k entries")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    rc = load_library().rtopk_aggregate(_ptr(idx), _ptr(val), n, k, out.numel(), _ptr(out),
                                        _ptr(workspace), ws_bytes, _stream_handle(stream))
    if rc:
        raise RtopkError(rc, "rtopk_aggregate")


def aggregate_update_workspace_bytes(d: int, n: int, k: int) -> int:
    out = ctypes.c_uint64(0)
    rc = load_library().rtopk_aggregate_update_workspace_bytes(d, n, k, ctypes.byref(out))
    if rc:
        raise RtopkError(rc, "rtopk_aggregate_update_workspace_bytes")
    return out.value


def aggregate_update(idx: torch.Tensor, val: torch.Tensor, n: int, k: int, eta: float,
                     scale: float, omega: torch.Tensor, workspace: torch.Tensor,
                     stream=None) -> None:
    """rtopk_aggregate_update: enqueue omega -= eta * scale * (average of the n
    messages), in place on ``omega`` (d elements)."""
    _need(idx, torch.int32, "idx")
    _need(val, torch.float32, "val")
    _need(omega, torch.float32, "omega")
    if idx.numel() < n * k or val.numel() < n * k:
        raise ValueError("idx/val must hold n*k entries")
    rc = load_library().rtopk_aggregate_update(_ptr(idx), _ptr(val), n, k, omega.numel(),
                                               eta, scale, _ptr(omega), _ptr(workspace),
                                               workspace.numel() * workspace.element_size(),
                                               _stream_handle(stream))
    if rc:
        raise RtopkError(rc, "rtopk_aggregate_update")


STATIC_SCRATCH_BYTES = 16 << 20


def aggregate_update_static(idx: torch.Tensor, val: torch.Tensor, n: int, k: int, eta: float,
                            scale: float, omega: torch.Tensor, stream=None) -> None:
    """rtopk_aggregate_update_static: as :func:`aggregate_update`, with the
    library's built-in scratch array in place of a workspace."""
    _need(idx, torch.int32, "idx")
    _need(val, torch.float32, "val")
    _need(omega, torch.float32, "omega")
    if idx.numel() < n * k or val.numel() < n * k:
        raise ValueError("idx/val must hold n*k entries")
    rc = load_library().rtopk_aggregate_update_static(_ptr(idx), _ptr(val), n, k, omega.numel(),
                                                      eta, scale, _ptr(omega),
                                                      _stream_handle(stream))
    if rc:
        raise RtopkError(rc, "rtopk_aggregate_update_static")


def aggregate_update_momentum(idx: torch.Tensor, val: torch.Tensor, n: int, k: int, eta: float,
                              scale: float, mu: float, omega: torch.Tensor,
                              velocity: torch.Tensor, stream=None) -> None:
    """rtopk_aggregate_update_momentum: enqueue velocity = mu * velocity + scale *
    (average of the n messages); omega -= eta * velocity, both in place."""
    _need(idx, torch.int32, "idx")
    _need(val, torch.float32, "val")
    _need(omega, torch.float32, "omega")
    _need(velocity, torch.float32, "velocity")
    if idx.numel() < n * k or val.numel() < n * k or velocity.numel() != omega.numel():
        raise ValueError("idx/val must hold n*k entries; omega and velocity the same d")
    rc = load_library().rtopk_aggregate_update_momentum(
        _ptr(idx), _ptr(val), n, k, omega.numel(), eta, scale, mu, _ptr(omega), _ptr(velocity),
        _stream_handle(stream))
    if rc:
        raise RtopkError(rc, "rtopk_aggregate_update_momentum")


STAGES = {"prepare": 1, "fused": 2, "classify": 3, "finalize": 4, "emit": 5, "all": 100}


def trace_next_encode(stage: int, ev_begin: int, ev_end: int) -> None:
    """rtopk_trace_next_encode: raw hipEvent_t handles, recorded around ``stage``
    of the next encode issued from this thread."""
    rc = load_library().rtopk_trace_next_encode(stage, ev_begin, ev_end)
    if rc:
        raise RtopkError(rc, "rtopk_trace_next_encode")


FORCE_ESTIMATE_MISS = 1
FORCE_KEY_WINDOW_MISS = 2
FORCE_CHECK_IN_ABORT = 4
FORCE_BRACKET_LOW = 8
FORCE_BARRIER_TIMEOUT = 16


def force_next_encode(flags: int) -> None:
    """rtopk_force_next_encode: make the next encode from this thread take an
    exact fallback path (test hook)."""
    rc = load_library().rtopk_force_next_encode(flags)
    if rc:
        raise RtopkError(rc, "rtopk_force_next_encode")


def encode_stats(workspace: torch.Tensor, stream=None) -> dict:
    st = EncodeStats()
    rc = load_library().rtopk_encode_stats(_ptr(workspace), _stream_handle(stream),
                                           ctypes.byref(st))
    if rc:
        raise RtopkError(rc, "rtopk_encode_stats")
    return {name: int(getattr(st, name)) for name, _ in EncodeStats._fields_}


# ---- matrix parameters: a layer's products in 8-bit integers, orthogonalised updates ----------
# (As in all calls of this module outputs are written where they lie and nothing is recorded for autograd: a layer's gradients
# come from linear_i8_backward.)

_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_INT8 = (torch.int8,)
_ALONG = {"rows": 0, "columns": 1}
_PRODUCTS = {"pairs": 0, "halves": 1}
#: (a, b, c) of every step, in common use for updates of neural networks
QUINTIC = (3.4445, -4.7750, 2.0315)


def _matrix(t: torch.Tensor, name: str, types) -> int:
    """Refuses what is not a matrix of one of ``types`` on the GPU with its rows one after the other; the distance of
    its rows in elements."""
    if not t.is_cuda or t.dtype not in types or t.dim() != 2:
        raise TypeError(f"{name} must be a matrix on the GPU of {' or '.join(map(str, types))}")
    (rows, cols), (ld, one) = t.size(), t.stride()
    if rows < 2:
        ld = cols or 1
    if cols > 1 and one != 1 or ld < cols:
        raise TypeError(f"the elements of {name}'s rows must be neighbours, and its rows must not overlap")
    return ld


def _ld(t: torch.Tensor) -> int:
    """Distance of a matrix's rows in elements."""
    return t.stride(0) if t.size(0) > 1 else max(t.size(1), 1)


def _vector(t: torch.Tensor, length: int, name: str) -> None:
    _need(t, torch.float32, name)
    if t.numel() != length:
        raise ValueError(f"{name} must have {length} elements")


def _bytes(name: str, *args) -> int:
    out = ctypes.c_uint64(0)
    rc = getattr(load_library(), name)(*args, ctypes.byref(out))
    if rc:
        raise RtopkError(rc, name)
    return out.value


def _workspace(workspace: Optional[torch.Tensor], need: int, device, stream):
    """The caller's workspace, or memory of torch's allocator on the call's stream: (pointer, bytes, what holds it)."""
    if workspace is not None:
        if not workspace.is_cuda or not workspace.is_contiguous():
            raise TypeError("workspace must be a contiguous tensor on the GPU")
        return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace
    if not need:
        return None, 0, None
    if stream is None:
        held = torch.empty(need + 256, dtype=torch.uint8, device=device)
    else:
        with torch.cuda.stream(stream):
            held = torch.empty(need + 256, dtype=torch.uint8, device=device)
    at = held.data_ptr()
    return at + -at % 256, need, held


@functools.lru_cache(maxsize=1024)
def quantize_i8_workspace_bytes(rows: int, cols: int, along: str = "rows") -> int:
    return _bytes("rtopk_quantize_i8_workspace_bytes", rows, cols, _ALONG[along])


def quantize_i8(x: torch.Tensor, q: torch.Tensor, scale: torch.Tensor, along: str = "rows",
                workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """rtopk_quantize_i8: ``q`` (int8) and ``scale`` of the matrix ``x``, a scale for each row, or
    (``along="columns"``) for each column, ``q`` then holding ``x`` turned over. Give ``q`` rows that start on
    16 bytes (a multiple of 16 between them) where the product is to read it fast. ``workspace``: None
    takes it from torch's allocator, here and in the calls below."""
    ldx, ldq = _matrix(x, "x", _TYPES), _matrix(q, "q", _INT8)
    rows, cols = x.size()
    if q.size() != ((rows, cols) if along == "rows" else (cols, rows)):
        raise ValueError("q must have the shape of x, or of x turned over along columns")
    _vector(scale, q.size(0), "scale")
    need = 0 if along == "rows" or workspace is not None else quantize_i8_workspace_bytes(rows, cols, along)
    ws, ws_bytes, held = _workspace(workspace, need, x.device, stream)
    rc = load_library().rtopk_quantize_i8(x.data_ptr(), _TYPES[x.dtype], rows, cols, ldx, _ALONG[along], q.data_ptr(), ldq,
                                          scale.data_ptr(), ws, ws_bytes, _stream_handle(stream))
    if rc:
        raise RtopkError(rc, "rtopk_quantize_i8")


@functools.lru_cache(maxsize=1024)
def matmul_i8_workspace_bytes(m: int, n: int, k: int) -> int:
    return _bytes("rtopk_matmul_i8_workspace_bytes", m, n, k)


def matmul_i8(a: torch.Tensor, a_scale: torch.Tensor, b: torch.Tensor, b_scale: torch.Tensor, out: torch.Tensor,
              bias: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """rtopk_matmul_i8: out[i, j] = a_scale[i] b_scale[j] sum_k a[i, k] b[j, k] (+ bias[j])."""
    lda, ldb, ldo = _matrix(a, "a", _INT8), _matrix(b, "b", _INT8), _matrix(out, "out", _TYPES)
    (m, k), (n, b_k) = a.size(), b.size()
    if b_k != k or out.size() != (m, n):
        raise ValueError("a is [m, k], b [n, k], out [m, n]")
    _vector(a_scale, m, "a_scale")
    _vector(b_scale, n, "b_scale")
    if bias is not None:
        _vector(bias, n, "bias")
    need = 0 if workspace is not None else matmul_i8_workspace_bytes(m, n, k)
    ws, ws_bytes, held = _workspace(workspace, need, a.device, stream)
    rc = load_library().rtopk_matmul_i8(a.data_ptr(), a_scale.data_ptr(), b.data_ptr(), b_scale.data_ptr(), _ptr(bias), m, n, k, lda, ldb,
                                        out.data_ptr(), _TYPES[out.dtype], ldo, ws, ws_bytes, _stream_handle(stream))
    if rc:
        raise RtopkError(rc, "rtopk_matmul_i8")


@functools.lru_cache(maxsize=1024)
def linear_i8_workspace_bytes(m: int, k: int, n: int) -> int:
    return _bytes("rtopk_linear_i8_workspace_bytes", m, k, n)


def linear_i8(x: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, out: torch.Tensor, bias: Optional[torch.Tensor] = None,
              workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """rtopk_linear_i8: out = x w^T + bias, ``x`` [m, k] quantised by token on the way, ``w`` [n, k] int8 with
    ``w_scale`` [n] as :func:`quantize_i8` leaves them."""
    # (a token's call is as long as what the host does for it: 8 us of checks and conversions in its first form)
    ldx, ldw, ldo = _matrix(x, "x", _TYPES), _matrix(w, "w", _INT8), _matrix(out, "out", _TYPES)
    (m, k), (n, w_k) = x.size(), w.size()
    if w_k != k or out.size() != (m, n):
        raise ValueError("x is [m, k], w [n, k], out [m, n]")
    _vector(w_scale, n, "w_scale")
    if bias is not None:
        _vector(bias, n, "bias")
    need = 0 if workspace is not None else linear_i8_workspace_bytes(m, k, n)
    ws, ws_bytes, held = _workspace(workspace, need, x.device, stream)
    rc = load_library().rtopk_linear_i8(x.data_ptr(), _TYPES[x.dtype], m, k, ldx, w.data_ptr(), w_scale.data_ptr(), n, ldw, _ptr(bias),
                                        out.data_ptr(), _TYPES[out.dtype], ldo, ws, ws_bytes, _stream_handle(stream))
    if rc:
        raise RtopkError(rc, "rtopk_linear_i8")


@functools.lru_cache(maxsize=1024)
def linear_i8_backward_workspace_bytes(m: int, k: int, n: int) -> int:
    return _bytes("rtopk_linear_i8_backward_workspace_bytes", m, k, n)


def linear_i8_backward(dy: torch.Tensor, x: Optional[torch.Tensor], w_turned: Optional[torch.Tensor],
                       w_turned_scale: Optional[torch.Tensor], dx: Optional[torch.Tensor], dw: Optional[torch.Tensor],
                       db: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """rtopk_linear_i8_backward: the gradients of :func:`linear_i8`'s input, weights (binary32, [n, k]) and bias from
    ``dy`` [m, n]. ``w_turned`` [k, n] and its scales: the weights quantised along columns. ``dx`` or ``dw`` may be
    None, and then what only they need too."""
    if dx is None and dw is None:
        raise ValueError("neither dx nor dw is asked for")
    if dx is not None and (w_turned is None or w_turned_scale is None) or dw is not None and x is None:
        raise ValueError("dx needs w_turned and its scales, dw needs x")
    if db is not None and dw is None:
        raise ValueError("db comes with dw")
    _matrix(dy, "dy", _TYPES)
    m, n = dy.shape
    k = (dx if dx is not None else dw).size(1)
    if dx is not None:
        _matrix(dx, "dx", (dy.dtype,))
        _matrix(w_turned, "w_turned", _INT8)
        _vector(w_turned_scale, k, "w_turned_scale")
        if tuple(dx.shape) != (m, k) or tuple(w_turned.shape) != (k, n):
            raise ValueError("dy is [m, n], dx [m, k], w_turned [k, n]")
    if dw is not None:
        _matrix(x, "x", (dy.dtype,))
        _matrix(dw, "dw", (torch.float32,))
        if tuple(x.shape) != (m, k) or tuple(dw.shape) != (n, k):
            raise ValueError("dy is [m, n], x [m, k], dw [n, k]")
    if db is not None:
        _vector(db, n, "db")
    ws, ws_bytes, held = _workspace(workspace, 0 if workspace is not None else linear_i8_backward_workspace_bytes(m, k, n),
                                    dy.device, stream)
    ld = lambda t: 0 if t is None else _ld(t)   # noqa: E731
    rc = load_library().rtopk_linear_i8_backward(
        _ptr(dy), _ptr(x), _TYPES[dy.dtype], m, k, n, _ld(dy), ld(x), _ptr(w_turned), _ptr(w_turned_scale), ld(w_turned),
        _ptr(dx), ld(dx), _ptr(dw), ld(dw), _ptr(db), ws, ws_bytes, _stream_handle(stream))
    if rc:
        raise RtopkError(rc, "rtopk_linear_i8_backward")


def _coefficients(coefficients, steps: Optional[int]):
    """(number of steps, their coefficients as binary32): one triple for all of 5 or ``steps``, or a triple for each."""
    rows = [tuple(c) for c in coefficients] if not isinstance(coefficients[0], (int, float)) else \
        [tuple(coefficients)] * (5 if steps is None else steps)
    if not rows or any(len(c) != 3 for c in rows) or (steps is not None and len(rows) != steps):
        raise ValueError("coefficients: three numbers, or three for each step")
    return len(rows), (ctypes.c_float * (3 * len(rows)))(*[v for c in rows for v in c])


@functools.lru_cache(maxsize=1024)
def orthogonalize_workspace_bytes(count: int, rows: int, cols: int, products: str = "pairs") -> int:
    return _bytes("rtopk_orthogonalize_workspace_bytes", count, rows, cols, _PRODUCTS[products])


def orthogonalize(xs, outs, steps: Optional[int] = None, coefficients=QUINTIC, eps: float = 1e-7,
                  products: Optional[str] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """rtopk_orthogonalize: Newton-Schulz orthogonalisation of every matrix of the list ``xs`` (equal shapes, types and
    row distances) into ``outs`` (which may be ``xs``). ``products``: "pairs" (None too: 22 bits between the
    products, about as exact as binary32), or "halves" (11 bits, down to a third of the time), whose error grows with what the strongest directions
    have over the others: beyond a bfloat16 result's own rounding from about 30 times in each element on."""
    count = len(xs)
    if count < 1 or len(outs) != count:
        raise ValueError("xs and outs must have the same length >= 1")
    x, out = xs[0], outs[0]
    for a, b in zip(xs, outs):
        _matrix(a, "x", (x.dtype,) if x.dtype in _TYPES else _TYPES)
        _matrix(b, "out", (out.dtype,) if out.dtype in _TYPES else _TYPES)
        if a.shape != x.shape or b.shape != x.shape or _ld(a) != _ld(x) or _ld(b) != _ld(out):
            raise ValueError("all matrices must have one shape, and one distance of their rows")
    products = products or "pairs"
    rows, cols = x.shape
    number, abc = _coefficients(coefficients, steps)
    ws, ws_bytes, held = _workspace(workspace, 0 if workspace is not None else
                                    orthogonalize_workspace_bytes(count, rows, cols, products), x.device, stream)
    vp_arr = ctypes.c_void_p * count
    rc = load_library().rtopk_orthogonalize(
        count, vp_arr(*[_ptr(t) for t in xs]), _TYPES[x.dtype], rows, cols, _ld(x), number, abc, eps, _PRODUCTS[products],
        vp_arr(*[_ptr(t) for t in outs]), _TYPES[out.dtype], _ld(out), ws, ws_bytes, _stream_handle(stream))
    if rc:
        raise RtopkError(rc, "rtopk_orthogonalize")


@functools.lru_cache(maxsize=1024)
def aggregate_update_orthogonal_workspace_bytes(count: int, rows: int, cols: int, products: str = "pairs") -> int:
    return _bytes("rtopk_aggregate_update_orthogonal_workspace_bytes", count, rows, cols, _PRODUCTS[products])


def aggregate_update_orthogonal(idx, val, n: int, k: int, eta: float, scale: float, mu: float, omega, velocity,
                                nesterov: bool = True, decay: float = 0.0, gain: float = 1.0, steps: Optional[int] = None,
                                coefficients=QUINTIC, eps: float = 1e-7, products: str = "pairs",
                                workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """rtopk_aggregate_update_orthogonal: for every matrix of the list ``omega`` (with its ``velocity`` and its n
    messages ``idx``, ``val`` back to back): velocity = mu velocity + scale average, and omega = (1 - eta decay)
    omega - eta gain orthogonalised(mu velocity + scale average, or velocity without ``nesterov``), in place."""
    count = len(omega)
    if count < 1 or not (len(idx) == len(val) == len(velocity) == count):
        raise ValueError("idx, val, omega and velocity must have the same length >= 1")
    if n < 1 or k < 1:
        raise ValueError("n and k must be at least 1")
    if omega[0].dim() != 2:
        raise ValueError("omega must hold matrices")
    rows, cols = omega[0].shape
    for i, v, w, m in zip(idx, val, omega, velocity):
        _need(i, torch.int32, "idx")
        _need(v, torch.float32, "val")
        _need(w, torch.float32, "omega")
        _need(m, torch.float32, "velocity")
        if tuple(w.shape) != (rows, cols) or m.numel() != rows * cols:
            raise ValueError("all of omega must have one shape, and velocity as many elements")
        if i.numel() < n * k or v.numel() < n * k:
            raise ValueError("idx/val must hold n*k entries")
    number, abc = _coefficients(coefficients, steps)
    ws, ws_bytes, held = _workspace(workspace, 0 if workspace is not None else
                                    aggregate_update_orthogonal_workspace_bytes(count, rows, cols, products), omega[0].device, stream)
    vp_arr = ctypes.c_void_p * count
    pointers = lambda ts: vp_arr(*[_ptr(t) for t in ts])   # noqa: E731
    rc = load_library().rtopk_aggregate_update_orthogonal(
        count, pointers(idx), pointers(val), n, k, rows, cols, eta, scale, mu, int(bool(nesterov)), decay, gain, number, abc, eps,
        _PRODUCTS[products], pointers(omega), pointers(velocity), ws, ws_bytes, _stream_handle(stream))
    if rc:
        raise RtopkError(rc, "rtopk_aggregate_update_orthogonal")


def product_plan(m: int, n: int, k: int, on_lines: bool = True) -> dict:
    """rtopk_product_plan: the tiles and runs that the 8-bit product of these sizes takes."""
    plan = ProductPlan()
    rc = load_library().rtopk_product_plan(m, n, k, int(on_lines), ctypes.byref(plan))
    if rc:
        raise RtopkError(rc, "rtopk_product_plan")
    return {name: int(getattr(plan, name)) for name, _ in plan._fields_}


def orthogonalize_plan(count: int, rows: int, cols: int, products: str = "pairs", steps: Optional[int] = None,
                       coefficients=QUINTIC) -> dict:
    """rtopk_orthogonalize_plan: the tiles, runs and form of steps that the orthogonalisation of these sizes takes."""
    number, abc = _coefficients(coefficients, steps)
    plan = OrthogonalizePlan()
    rc = load_library().rtopk_orthogonalize_plan(count, rows, cols, _PRODUCTS[products], number, abc, ctypes.byref(plan))
    if rc:
        raise RtopkError(rc, "rtopk_orthogonalize_plan")
    return {name: int(getattr(plan, name)) for name, _ in plan._fields_}
