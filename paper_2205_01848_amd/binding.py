"""ctypes binding of libmoe.so: the same names as the C entry points in
include/moe.h, taking torch tensors (device memory) and ints.  This module
only marshals arguments; every step runs in the HIP kernels of libmoe.  If
the library is missing it raises - there is no fallback path.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import Optional

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libmoe.so")

MOE_F32, MOE_BF16 = 0, 1
MOE_RELU, MOE_GELU_TANH, MOE_SWIGLU = 0, 1, 2
ACTS = {"relu": MOE_RELU, "gelu_tanh": MOE_GELU_TANH, "swiglu": MOE_SWIGLU}
STATUS_BAD_ID, STATUS_DUP_ID, STATUS_REGION, STATUS_BAD_TARGET = 1, 2, 4, 8

_c_int, _c_i64, _c_size, _p = ctypes.c_int, ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p


class _stream_p(ctypes.c_void_p):
    """The stream of the calls around the layer (norm, vocabulary loss, AdamW)."""


class LayerFwdArgs(ctypes.Structure):
    """moe_layer_fwd_args."""
    _fields_ = ([(n, _c_int) for n in ("dtype", "act", "T", "d", "E", "k", "f", "renorm",
                                       "dynamic", "num", "den", "cap_min", "row_align")] +
                [("rows_alloc", _c_i64)] +
                [(n, _p) for n in ("x", "w_g", "bias", "w1", "w3", "w2", "cached_ids", "logits",
                                   "weights", "ids", "capacity", "offsets", "counts", "fill",
                                   "dest_row", "src", "status", "x_disp", "h_save", "y_disp",
                                   "y")] +
                [("route_ws", _p), ("route_ws_bytes", _c_size), ("ffn_ws", _p),
                 ("ffn_ws_bytes", _c_size)])


class AdamWTensorArgs(ctypes.Structure):
    """moe_adamw_tensor."""
    _fields_ = ([(n, _p) for n in ("p", "g", "master", "m", "v", "m_exp", "v_exp")] +
                [("n", _c_i64), ("weight_decay", ctypes.c_double), ("p_dtype", _c_int), ("g_dtype", _c_int)])


# name -> (restype, argtypes)
SIGNATURES = {
    "moe_status_string": (ctypes.c_char_p, [_c_int]),
    "moe_abi_version": (_c_int, []),
    "moe_gate_topk": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int,
                               _p, _p, _p, _p, _p, _p]),
    "moe_count": (_c_int, [_p, _c_int, _c_int, _c_int, _p, _p, _p]),
    "moe_update_capacity": (_c_int, [_p, _c_int, _c_int, _c_int, _p, _c_int, _c_int, _c_int,
                                     _c_int, _p, _p]),
    "moe_dispatch_workspace_bytes": (_c_size, [_c_int, _c_int, _c_int]),
    "moe_dispatch": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _c_int, _p, _p, _p, _p,
                              _c_i64, _p, _p, _p, _p, _p, _p, _p, _c_size]),
    "moe_route_workspace_bytes": (_c_size, [_c_int, _c_int, _c_int]),
    "moe_route": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _c_int, _p, _p, _c_int, _c_int,
                           _c_int, _c_int, _c_int, _c_i64, _p, _p, _p, _p, _p, _p, _p, _p, _p,
                           _c_size]),
    "moe_layer_fwd": (_c_int, [_p, ctypes.POINTER(LayerFwdArgs)]),
    "moe_dispatch_noalloc": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _c_int, _p, _p, _p,
                                      _p, _c_i64, _p, _p, _p, _p, _p, _p]),
    "moe_dispatch_noalloc_max_assignments": (_c_size, []),
    "moe_ffn_fwd_workspace_bytes": (_c_size, [_c_int, _c_int, _c_int, _c_int, _c_int, _c_i64]),
    "moe_ffn_bwd_workspace_bytes": (_c_size, [_c_int, _c_int, _c_int, _c_int, _c_int, _c_i64]),
    "moe_expert_ffn_fwd": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _c_int, _p, _p,
                                    _c_i64, _p, _p, _p, _p, _p, _p, _p, _c_size]),
    "moe_zero_pad_rows": (_c_int, [_p, _c_int, _c_int, _c_int, _p, _p, _p, _c_i64, _p]),
    "moe_combine": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _c_i64, _p, _p, _p, _p]),
    "moe_combine_bwd": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _c_i64, _p, _p, _p,
                                 _p, _p, _p]),
    "moe_expert_ffn_bwd": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _c_int, _p, _p,
                                    _c_i64, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p, _p,
                                    _c_size]),
    "moe_gate_bwd_workspace_bytes": (_c_size, [_c_int, _c_int, _c_int]),
    "moe_gate_bwd": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _p, _p,
                              _p, _p, _p, _p, _p, _p, _c_size]),
    "moe_dispatch_bwd": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _c_int, _c_i64, _p,
                                  _p, _p, _p, _p]),
    "moe_balance_workspace_bytes": (_c_size, [_c_int, _c_int]),
    "moe_balance_fwd": (_c_int, [_p, _c_int, _c_int, _c_int, ctypes.c_float, _p, _p, _p, _p,
                                 _p, _c_size]),
    "moe_aggregate_spec": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _p, _p, _c_i64, _p]),
    "moe_spec_loss_workspace_bytes": (_c_size, [_c_int]),
    "moe_spec_loss": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _p, _p, _p, _p, _c_i64, _p,
                               _p, _p, _p, _c_size]),
    "moe_vocab_loss_workspace_bytes": (_c_size, [_c_int] * 6),
    "moe_vocab_loss": (_c_int, [_stream_p, _c_int, _c_int, _c_int, _c_int, _p, _c_i64, _p, _p,
                                ctypes.c_float, _p, _p, _p, _p, _c_i64, _c_int, _p, _p, _p, _c_size]),
    "moe_cache_update": (_c_int, [_p, _c_int, _c_int, _p, _p, _p, _p]),
    "moe_cached_weights": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _p, _p, _p]),
    "moe_caching_decision": (_c_int, [_c_int, _c_i64, _c_i64, _c_int, _c_int, _c_int, _c_int,
                                      _c_int, _c_int]),
    "moe_capacity_trigger": (_c_int, [_c_int, _c_int, _p, _p, _c_int, _c_int, _c_int, _c_int,
                                      _c_int]),
    "moe_policy_create": (_c_int, [_c_int, _c_int, _c_int, _c_int, _c_int, _c_int, _c_int,
                                   _c_int, _c_int, _c_int, _p, _p]),
    "moe_policy_destroy": (None, [_p]),
    "moe_policy_begin": (_c_int, [_p, _p, _p, _p, _p, _p]),
    "moe_policy_end": (_c_int, [_p, _p, _p]),
    "moe_policy_state": (_c_int, [_p, _p, _p, _p, _p]),
    "moe_quantized_width": (_c_int, [_c_int]),
    "moe_quantize_rows": (_c_int, [_p, _c_int, _c_i64, _c_int, _p, _c_i64, _p, _p]),
    "moe_rms_norm_fwd": (_c_int, [_stream_p, _c_int, _c_i64, _c_int, _p, _c_i64, _p, _c_i64, _p,
                                  ctypes.c_float, _p, _c_i64, _p, _c_i64, _p, _p, _p]),
    "moe_rms_norm_bwd_workspace_bytes": (_c_size, [_c_i64, _c_int]),
    "moe_rms_norm_bwd": (_c_int, [_stream_p, _c_int, _c_i64, _c_int, _p, _c_i64, _p, _p, _p, _c_i64, _p,
                                  _c_i64, _p, _c_i64, _c_int, _p, _p, _c_size]),
    "moe_expert_matmul_i8_workspace_bytes": (_c_size, [_c_int, _c_int, _c_i64]),
    "moe_expert_matmul_i8": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _p, _p, _c_i64, _p, _p,
                                      _p, _c_int, _c_int, _p, _p, _p, _p, _c_size]),
    "moe_ffn_fwd_i8_workspace_bytes": (_c_size, [_c_int, _c_int, _c_int, _c_int, _c_int, _c_i64]),
    "moe_expert_ffn_fwd_i8": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _c_int, _p, _p, _c_i64,
                                       _p, _p, _p, _c_int, _c_int, _p, _p, _p, _p, _p, _p, _p,
                                       _p, _c_size]),
    "moe_gated_ffn_fwd_workspace_bytes": (_c_size, [_c_int, _c_int, _c_int, _c_int]),
    "moe_gated_ffn_bwd_workspace_bytes": (_c_size, [_c_int, _c_int, _c_int, _c_int]),
    "moe_gated_ffn_fwd": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _c_int, _p, _c_i64, _p, _p,
                                   _p, _p, _c_i64, _p, _p, _c_i64, _p, _c_size]),
    "moe_gated_ffn_bwd": (_c_int, [_p, _c_int, _c_int, _c_int, _c_int, _c_int, _p, _c_i64, _p, _p,
                                   _p, _p, _p, _c_i64, _p, _c_i64, _p, _c_i64, _c_int, _p, _p, _p,
                                   _p, _c_size]),
    "moe_adamw_blocks": (_c_size, [_c_i64]),
    "moe_adamw": (_c_int, [_stream_p, _c_int, ctypes.POINTER(AdamWTensorArgs)] +
                  [ctypes.c_double] * 4 + [_c_i64, ctypes.c_uint32, _p, _p]),
    "moe_adamw_unpack": (_c_int, [_stream_p, _c_int, ctypes.POINTER(AdamWTensorArgs), _p, _p]),
    "moe_timing_enable": (_c_int, [_c_int]),
    "moe_set_gemm_tiles": (_c_int, [_c_int]),
    "moe_set_dx_weight_copy": (_c_int, [_c_int]),
    "moe_timing_report": (_c_int, [ctypes.c_char_p, _c_size]),
}

_lib = None


ABI_VERSION = 7   # moe_abi_version() of the library this binding is written for


class MoEError(RuntimeError):
    pass


def lib():
    """The loaded libmoe.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise MoEError(f"{LIB_PATH} is not built (python -m paper_2205_01848_amd.build); "
                           "the HIP library is required, there is no fallback")
        L = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        # buffer sizes here follow this ABI (h_save planes, argument lists):
        # a library of another version would read and write past them
        if L.moe_abi_version() != ABI_VERSION:
            raise MoEError(f"{LIB_PATH} has ABI version {L.moe_abi_version()}, this binding "
                           f"expects {ABI_VERSION}: rebuild it (python -m paper_2205_01848_amd.build)")
        _lib = L
    return _lib


def _check(st: int, what: str):
    if st != 0:
        raise MoEError(f"{what}: {lib().moe_status_string(st).decode()}")


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise MoEError("tensor must live in device memory")
    if not t.is_contiguous():
        raise MoEError("tensor must be contiguous")
    return t.data_ptr()


# Every call runs on the device of its tensors, on that device's current stream,
# whichever device is current.
def _stream():
    # (by index: without one, torch takes more than twice as long to find it)
    return torch.cuda.current_stream(torch.cuda.current_device()).cuda_stream


def _first_device(values) -> Optional[int]:
    for t in values:
        if isinstance(t, torch.Tensor):
            return t.get_device()           # -1: not in device memory, which the call refuses
    return None


def _on_its_device(fn):
    """fn with the device of its first tensor made current (the others are to live there too).
    Where it is current already (the usual case) torch's guard, which costs as much as a
    small launch, is left out."""
    @functools.wraps(fn)
    def call(*args, **kw):
        i = _first_device(args)
        if i is None:
            i = _first_device(kw.values())
        if i is None or i < 0 or i == torch.cuda.current_device():
            return fn(*args, **kw)
        with torch.cuda.device(i):
            return fn(*args, **kw)
    return call


def _device_of(*tensors) -> int:
    """Index of the one device all the call's tensors live on."""
    first = -1
    for t in tensors:
        if t is None:
            continue
        i = t.get_device()          # -1: not in device memory
        if i < 0:
            raise MoEError("tensor must live in device memory")
        if first < 0:
            first = i
        elif i != first:
            raise MoEError(f"tensors on devices {first} and {i}: one device is needed")
    return first


class _Here:
    """`with _Here(index) as stream`: on that device, with its current stream."""

    __slots__ = ("index", "guard")

    def __init__(self, index):
        self.index = index
        self.guard = None if index == torch.cuda.current_device() else torch.cuda.device(index)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()
        return torch.cuda.current_stream(self.index).cuda_stream

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return MOE_BF16
    if t.dtype == torch.float32:
        return MOE_F32
    raise MoEError(f"unsupported layer dtype {t.dtype}")


_I32, _F32 = torch.int32, torch.float32


def _need(t: Optional[torch.Tensor], n: int, name: str, dtype=None, optional=False):
    """Refuse a tensor with fewer than the n elements the entry point reads or
    writes, or of the wrong element type.  The C ABI takes bare pointers and
    cannot check sizes; an undersized buffer would be accessed past its end."""
    if t is None:
        if optional:
            return
        raise MoEError(f"{name} is required")
    if dtype is not None and t.dtype != dtype:
        raise MoEError(f"{name}: element type {t.dtype}, expected {dtype}")
    if t.numel() < n:
        raise MoEError(f"{name} holds {t.numel()} elements, the call needs {n}")


def _nbytes(t: torch.Tensor) -> int:
    return t.numel() * t.element_size()


def h_save_planes(act: int) -> int:
    """[rows_alloc, f] planes of h_save: A for ReLU, H and A for GELU, H1, H3
    and A for SwiGLU."""
    return 3 if act == MOE_SWIGLU else 2 if act == MOE_GELU_TANH else 1


def workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


# ---- entry points -----------------------------------------------------------
@_on_its_device
def moe_gate_topk(x, w_g, bias, k, renorm, logits, ids, weights):
    T, d = x.shape
    E = w_g.shape[0]
    _need(w_g, E * d, "w_g", x.dtype)
    _need(bias, E, "bias", _F32, optional=True)
    _need(logits, T * E, "logits", _F32)
    _need(ids, T * k, "ids", _I32)
    _need(weights, T * k, "weights", _F32)
    _check(lib().moe_gate_topk(_stream(), _dt(x), T, d, E, k, int(renorm), _ptr(x), _ptr(w_g),
                               _ptr(bias), _ptr(logits), _ptr(ids), _ptr(weights)),
           "moe_gate_topk")


@_on_its_device
def moe_count(ids, E, counts, status):
    T, k = ids.shape
    _need(ids, T * k, "ids", _I32)
    _need(counts, E, "counts", _I32)
    _need(status, 1, "status", _I32)
    _check(lib().moe_count(_stream(), T, E, k, _ptr(ids), _ptr(counts), _ptr(status)),
           "moe_count")


@_on_its_device
def moe_update_capacity(T, k, E, counts, num, den, cap_min, capacity, offsets, row_align=1):
    _need(counts, E, "counts", _I32, optional=True)
    _need(capacity, E, "capacity", _I32)
    _need(offsets, E + 1, "offsets", _I32)
    _check(lib().moe_update_capacity(_stream(), T, k, E, _ptr(counts), num, den, cap_min,
                                     row_align, _ptr(capacity), _ptr(offsets)),
           "moe_update_capacity")


def moe_dispatch_workspace_bytes(T, E, k) -> int:
    return lib().moe_dispatch_workspace_bytes(T, E, k)


@_on_its_device
def moe_dispatch(x, ids, E, capacity, offsets, rows_alloc, counts, fill, dest_row, src, x_disp,
                 status, ws):
    T, d = x.shape
    k = ids.shape[1]
    _need(ids, T * k, "ids", _I32)
    for t, n, name in ((capacity, E, "capacity"), (offsets, E + 1, "offsets"),
                       (counts, E, "counts"), (fill, E, "fill"), (dest_row, T * k, "dest_row"),
                       (src, rows_alloc, "src"), (status, 1, "status")):
        _need(t, n, name, _I32)
    _need(x_disp, rows_alloc * d, "x_disp", x.dtype)
    _check(lib().moe_dispatch(_stream(), _dt(x), T, d, E, k, _ptr(x), _ptr(ids), _ptr(capacity),
                              _ptr(offsets), rows_alloc, _ptr(counts), _ptr(fill),
                              _ptr(dest_row), _ptr(src), _ptr(x_disp), _ptr(status), _ptr(ws),
                              _nbytes(ws)), "moe_dispatch")


def moe_route_workspace_bytes(T, E, k) -> int:
    return lib().moe_route_workspace_bytes(T, E, k)


@_on_its_device
def moe_route(x, ids, E, dynamic, num, den, cap_min, rows_alloc, capacity, offsets, counts, fill,
              dest_row, src, x_disp, status, ws, row_align=1):
    """moe_count (dynamic), moe_update_capacity and moe_dispatch in one call."""
    T, d = x.shape
    k = ids.shape[1]
    _need(ids, T * k, "ids", _I32)
    for t, n, name in ((capacity, E, "capacity"), (offsets, E + 1, "offsets"),
                       (counts, E, "counts"), (fill, E, "fill"), (dest_row, T * k, "dest_row"),
                       (src, rows_alloc, "src"), (status, 1, "status")):
        _need(t, n, name, _I32)
    _need(x_disp, rows_alloc * d, "x_disp", x.dtype)
    _check(lib().moe_route(_stream(), _dt(x), T, d, E, k, _ptr(x), _ptr(ids), int(dynamic), num,
                           den, cap_min, row_align, rows_alloc, _ptr(capacity), _ptr(offsets),
                           _ptr(counts), _ptr(fill), _ptr(dest_row), _ptr(src), _ptr(x_disp),
                           _ptr(status), _ptr(ws), _nbytes(ws)), "moe_route")


@_on_its_device
def moe_layer_fwd(x, w_g, bias, w1, w3, w2, cached_ids, weights, *, act, k, renorm, dynamic, num,
                  den, rows_alloc, logits, ids, capacity, offsets, counts, fill, dest_row, src,
                  status, x_disp, h_save, y_disp, y, route_ws, ffn_ws, cap_min=0, row_align=1):
    """A whole layer forward in one call.  cached_ids None: the gate writes
    logits, ids and weights; else weights are the combine weights (None with
    y None: no combine)."""
    T, d = x.shape
    E, f, _ = w1.shape
    dt, R = x.dtype, rows_alloc
    a = LayerFwdArgs(_dt(x), act, T, d, E, k, f, int(renorm), int(dynamic), num, den, cap_min,
                     row_align, R)
    # every tensor the call reads or writes: (member, tensor, elements, type)
    need = [("x", x, T * d, dt), ("w1", w1, E * f * d, dt), ("w2", w2, E * d * f, dt),
            ("capacity", capacity, E, _I32), ("offsets", offsets, E + 1, _I32),
            ("counts", counts, E, _I32), ("fill", fill, E, _I32),
            ("dest_row", dest_row, T * k, _I32), ("src", src, R, _I32), ("status", status, 1, _I32),
            ("x_disp", x_disp, R * d, dt), ("y_disp", y_disp, R * d, dt)]
    if cached_ids is None:
        need += [("w_g", w_g, E * d, dt), ("logits", logits, T * E, _F32), ("ids", ids, T * k, _I32),
                 ("weights", weights, T * k, _F32)]
        if bias is not None:
            need.append(("bias", bias, E, _F32))
    else:
        need.append(("cached_ids", cached_ids, T * k, _I32))
        if y is not None:
            need.append(("weights", weights, T * k, _F32))
    if w3 is not None or act == MOE_SWIGLU:
        need.append(("w3", w3, E * f * d, dt))
    if h_save is not None:
        need.append(("h_save", h_save, h_save_planes(act) * R * f, dt))
    if y is not None:
        need.append(("y", y, T * d, dt))
    for name, t, n, dtype in need:
        if t is None or t.dtype != dtype or t.numel() < n or not t.is_cuda or not t.is_contiguous():
            _need(t, n, name, dtype)
            _ptr(t)
        setattr(a, name, t.data_ptr())
    for name, ws in (("route_ws", route_ws), ("ffn_ws", ffn_ws)):
        setattr(a, name, _ptr(ws))
        setattr(a, name + "_bytes", _nbytes(ws))
    _check(lib().moe_layer_fwd(_stream(), ctypes.byref(a)), "moe_layer_fwd")


def moe_dispatch_noalloc_max_assignments() -> int:
    return lib().moe_dispatch_noalloc_max_assignments()


@_on_its_device
def moe_dispatch_noalloc(x, ids, E, capacity, offsets, rows_alloc, counts, fill, dest_row, src,
                         x_disp, status):
    """moe_dispatch without a workspace (the library's fixed device scratch)."""
    T, d = x.shape
    k = ids.shape[1]
    _need(ids, T * k, "ids", _I32)
    for t, n, name in ((capacity, E, "capacity"), (offsets, E + 1, "offsets"),
                       (counts, E, "counts"), (fill, E, "fill"), (dest_row, T * k, "dest_row"),
                       (src, rows_alloc, "src"), (status, 1, "status")):
        _need(t, n, name, _I32)
    _need(x_disp, rows_alloc * d, "x_disp", x.dtype)
    _check(lib().moe_dispatch_noalloc(_stream(), _dt(x), T, d, E, k, _ptr(x), _ptr(ids),
                                      _ptr(capacity), _ptr(offsets), rows_alloc, _ptr(counts),
                                      _ptr(fill), _ptr(dest_row), _ptr(src), _ptr(x_disp),
                                      _ptr(status)), "moe_dispatch_noalloc")


def moe_ffn_fwd_workspace_bytes(dt, act, E, d, f, rows_alloc) -> int:
    return lib().moe_ffn_fwd_workspace_bytes(dt, act, E, d, f, rows_alloc)


def moe_ffn_bwd_workspace_bytes(dt, act, E, d, f, rows_alloc) -> int:
    return lib().moe_ffn_bwd_workspace_bytes(dt, act, E, d, f, rows_alloc)


@_on_its_device
def moe_expert_ffn_fwd(act, offsets, rows, x_disp, w1, w3, w2, h_save, y_disp, ws):
    E, f, d = w1.shape
    R, dt = x_disp.shape[0], w1.dtype
    _need(offsets, E + 1, "offsets", _I32)
    _need(rows, E, "rows", _I32)
    _need(x_disp, R * d, "x_disp", dt)
    _need(w3, E * f * d, "w3", dt, optional=act != MOE_SWIGLU)
    _need(w2, E * d * f, "w2", dt)
    _need(h_save, h_save_planes(act) * R * f, "h_save", dt, optional=True)
    _need(y_disp, R * d, "y_disp", dt)
    _check(lib().moe_expert_ffn_fwd(_stream(), _dt(w1), act, E, d, f, _ptr(offsets), _ptr(rows),
                                    x_disp.shape[0], _ptr(x_disp), _ptr(w1), _ptr(w3), _ptr(w2),
                                    _ptr(h_save), _ptr(y_disp), _ptr(ws), _nbytes(ws)),
           "moe_expert_ffn_fwd")


@_on_its_device
def moe_zero_pad_rows(offsets, fill, rows, buf):
    E = fill.shape[0]
    R, d = buf.shape
    _need(offsets, E + 1, "offsets", _I32)
    _need(fill, E, "fill", _I32)
    _need(rows, E, "rows", _I32)
    _check(lib().moe_zero_pad_rows(_stream(), _dt(buf), E, d, _ptr(offsets), _ptr(fill),
                                   _ptr(rows), R, _ptr(buf)), "moe_zero_pad_rows")


@_on_its_device
def moe_combine(y_disp, dest_row, weights, y):
    T, k = dest_row.shape
    d = y.shape[1]
    _need(y_disp, y_disp.shape[0] * d, "y_disp", y.dtype)
    _need(dest_row, T * k, "dest_row", _I32)
    _need(weights, T * k, "weights", _F32)
    _need(y, T * d, "y")
    _check(lib().moe_combine(_stream(), _dt(y), T, d, k, y_disp.shape[0], _ptr(y_disp),
                             _ptr(dest_row), _ptr(weights), _ptr(y)), "moe_combine")


@_on_its_device
def moe_combine_bwd(dy, y_disp, dest_row, weights, dy_disp, dweights):
    T, k = dest_row.shape
    d = dy.shape[1]
    R = y_disp.shape[0]
    _need(dy, T * d, "dy")
    _need(y_disp, R * d, "y_disp", dy.dtype)
    _need(dest_row, T * k, "dest_row", _I32)
    _need(weights, T * k, "weights", _F32)
    _need(dy_disp, R * d, "dy_disp", dy.dtype)
    _need(dweights, T * k, "dweights", _F32)
    _check(lib().moe_combine_bwd(_stream(), _dt(dy), T, d, k, y_disp.shape[0], _ptr(dy),
                                 _ptr(y_disp), _ptr(dest_row), _ptr(weights), _ptr(dy_disp),
                                 _ptr(dweights)), "moe_combine_bwd")


@_on_its_device
def moe_expert_ffn_bwd(act, offsets, rows, x_disp, h_save, w1, w3, w2, dy_disp, dx_disp, dw1,
                       dw3, dw2, ws):
    E, f, d = w1.shape
    R, dt, sw = x_disp.shape[0], w1.dtype, act == MOE_SWIGLU
    _need(offsets, E + 1, "offsets", _I32)
    _need(rows, E, "rows", _I32)
    _need(x_disp, R * d, "x_disp", dt)
    _need(h_save, h_save_planes(act) * R * f, "h_save", dt)
    _need(w3, E * f * d, "w3", dt, optional=not sw)
    _need(w2, E * d * f, "w2", dt)
    _need(dy_disp, R * d, "dy_disp", dt)
    _need(dx_disp, R * d, "dx_disp", dt)
    _need(dw1, E * f * d, "dw1", _F32)
    _need(dw3, E * f * d, "dw3", _F32, optional=not sw)
    _need(dw2, E * d * f, "dw2", _F32)
    _check(lib().moe_expert_ffn_bwd(_stream(), _dt(w1), act, E, d, f, _ptr(offsets), _ptr(rows),
                                    x_disp.shape[0], _ptr(x_disp), _ptr(h_save), _ptr(w1),
                                    _ptr(w3), _ptr(w2), _ptr(dy_disp), _ptr(dx_disp), _ptr(dw1),
                                    _ptr(dw3), _ptr(dw2), _ptr(ws), _nbytes(ws)),
           "moe_expert_ffn_bwd")


# ---- 8-bit integer products and the dense gated block ------------------------
def _rows(t: Optional[torch.Tensor], name, T, d, dtype, optional=False):
    """Row distance in elements of a [T, d] tensor whose rows are contiguous."""
    if t is None:
        if optional:
            return 0
        raise MoEError(f"{name} is required")
    if t.dtype is not dtype:
        raise MoEError(f"{name}: element type {t.dtype}, expected {dtype}")
    if t.shape != (T, d):
        raise MoEError(f"{name} has shape {tuple(t.shape)}, expected {(T, d)}")
    if T == 0:
        return d
    ld, one = t.stride()
    if one != 1 and d > 1:
        raise MoEError(f"{name}: the elements of a row must be contiguous")
    if T == 1:
        return d
    if ld < d or ld % 8:
        raise MoEError(f"{name}: rows are {ld} elements apart, a multiple of 8 not below "
                       f"{d} is needed")
    return ld


def _at(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def quantized_width(n: int) -> int:
    """Bytes between quantised rows of n values."""
    return (n + 15) // 16 * 16


def moe_quantize_rows(x, q, scale):
    """x [rows, n] (rows may be further apart) -> q [rows, quantized_width(n)], scale [rows]."""
    rows, n = x.shape
    ld = _rows(x, "x", rows, n, x.dtype)
    dt = _dt(x)
    _need(q, rows * quantized_width(n), "q", torch.int8)
    _need(scale, rows, "scale", _F32)
    with _Here(_device_of(x, q, scale)) as stream:
        _check(lib().moe_quantize_rows(stream, dt, rows, n, _at(x), ld, _ptr(q), _ptr(scale)),
               "moe_quantize_rows")


def moe_rms_norm_fwd(x, weight, eps, y=None, add=None, sum=None, rstd=None, q=None, scale=None):
    """s = x + add -> sum, y = s rsqrt(mean s^2 + eps) weight, and the same rows in 8 bits -> q
    [rows, quantized_width(d)], scale [rows]; x, add, sum, y [rows, d] may be rows of wider
    tensors."""
    (rows, d), dtype = x.shape, x.dtype
    dt = _dt(x)
    ldx = _rows(x, "x", rows, d, dtype)
    ldadd = 0 if add is None else _rows(add, "add", rows, d, dtype)
    ldsum = 0 if sum is None else _rows(sum, "sum", rows, d, dtype)
    ldy = 0 if y is None else _rows(y, "y", rows, d, dtype)
    _need(weight, d, "weight", dtype)
    if rstd is not None:
        _need(rstd, rows, "rstd", _F32)
    if q is not None:
        _need(q, rows * quantized_width(d), "q", torch.int8)
    if scale is not None:
        _need(scale, rows, "scale", _F32)
    with _Here(_device_of(x, weight, y, add, sum, rstd, q, scale)) as stream:
        _check(lib().moe_rms_norm_fwd(stream, dt, rows, d, _at(x), ldx, _at(add), ldadd, _ptr(weight),
                                      eps, _at(sum), ldsum, _at(y), ldy, _ptr(rstd), _ptr(q),
                                      _ptr(scale)), "moe_rms_norm_fwd")


def moe_rms_norm_bwd_workspace_bytes(rows, d) -> int:
    return lib().moe_rms_norm_bwd_workspace_bytes(rows, d)


def moe_rms_norm_bwd(s, weight, rstd, dy, dx, dw, ws, dsum=None):
    """Gradients of moe_rms_norm_fwd; dw (float32 or the layer's type) and ws None: dx alone."""
    (rows, d), dtype = s.shape, s.dtype
    dt = _dt(s)
    lds = _rows(s, "s", rows, d, dtype)
    lddy, lddx = _rows(dy, "dy", rows, d, dtype), _rows(dx, "dx", rows, d, dtype)
    lddsum = 0 if dsum is None else _rows(dsum, "dsum", rows, d, dtype)
    _need(weight, d, "weight", dtype)
    _need(rstd, rows, "rstd", _F32)
    if dw is not None and dw.dtype not in (dtype, _F32):
        raise MoEError(f"dw: a tensor of {dtype} or float32 is needed")
    _need(dw, d, "dw", optional=True)
    with _Here(_device_of(s, weight, rstd, dy, dx, dw, ws, dsum)) as stream:
        _check(lib().moe_rms_norm_bwd(stream, dt, rows, d, _at(s), lds, _ptr(weight), _ptr(rstd),
                                      _at(dy), lddy, _at(dsum), lddsum, _at(dx), lddx,
                                      dt if dw is None else _dt(dw), _ptr(dw), _ptr(ws),
                                      0 if ws is None else _nbytes(ws)), "moe_rms_norm_bwd")


def moe_expert_matmul_i8_workspace_bytes(E, N, rows_alloc) -> int:
    return lib().moe_expert_matmul_i8_workspace_bytes(E, N, rows_alloc)


def _need_scales(x_scale, src, k, R):
    """Elements of x_scale and src, and the number of tokens, of an int8 product."""
    if src is None:
        _need(x_scale, R, "x_scale", _F32)
        return 0
    _need(src, R, "src", _I32)
    _need(x_scale, 0, "x_scale", _F32)
    if k < 1:
        raise MoEError("k picks per token are needed with src")
    return x_scale.numel()


def moe_expert_matmul_i8(offsets, rows, xq, x_scale, wq, w_scale, y, ws, src=None, k=1):
    """xq [R, K] int8, wq [E, N, K] int8 -> y [R, N] over every expert's rows.  src (with k):
    moe_dispatch's, and x_scale holds one scale per token."""
    E, N, K = wq.shape
    R = xq.shape[0]
    dt = _dt(y)
    _need(offsets, E + 1, "offsets", _I32)
    _need(rows, E, "rows", _I32)
    _need(xq, R * K, "xq", torch.int8)
    _need(wq, E * N * K, "wq", torch.int8)
    _need(w_scale, E * N, "w_scale", _F32)
    _need(y, R * N, "y")
    T = _need_scales(x_scale, src, k, R)
    with _Here(_device_of(offsets, rows, xq, x_scale, wq, w_scale, y, ws, src)) as stream:
        _check(lib().moe_expert_matmul_i8(stream, dt, E, K, N, _ptr(offsets), _ptr(rows), R,
                                          _ptr(xq), _ptr(x_scale), _ptr(src), T, k, _ptr(wq),
                                          _ptr(w_scale), _ptr(y), _ptr(ws), _nbytes(ws)),
               "moe_expert_matmul_i8")


def moe_ffn_fwd_i8_workspace_bytes(dt, act, E, d, f, rows_alloc) -> int:
    return lib().moe_ffn_fwd_i8_workspace_bytes(dt, act, E, d, f, rows_alloc)


def moe_expert_ffn_fwd_i8(act, offsets, rows, xq, x_scale, w1q, w1_scale, w3q, w3_scale, w2q,
                          w2_scale, y_disp, ws, src=None, k=1):
    """The expert FFN on quantised tokens xq [R, quantized_width(d)] and weights
    (w1q, w3q [E, f, ..], w2q [E, d, ..])."""
    (E, f, kd), d, R = w1q.shape, w2q.shape[1], xq.shape[0]
    dt, sw = _dt(y_disp), act == MOE_SWIGLU
    if kd != quantized_width(d):
        raise MoEError(f"w1q: rows of {kd} bytes, expected {quantized_width(d)} for d = {d}")
    _need(offsets, E + 1, "offsets", _I32)
    _need(rows, E, "rows", _I32)
    _need(xq, R * kd, "xq", torch.int8)
    for name, t, n, dtype, opt in (
            ("w1q", w1q, E * f * kd, torch.int8, False), ("w1_scale", w1_scale, E * f, _F32, False),
            ("w3q", w3q, E * f * kd, torch.int8, not sw), ("w3_scale", w3_scale, E * f, _F32, not sw),
            ("w2q", w2q, E * d * quantized_width(f), torch.int8, False),
            ("w2_scale", w2_scale, E * d, _F32, False)):
        _need(t, n, name, dtype, optional=opt)
    _need(y_disp, R * d, "y_disp")
    T = _need_scales(x_scale, src, k, R)
    with _Here(_device_of(offsets, rows, xq, x_scale, w1q, w1_scale, w3q, w3_scale, w2q,
                                      w2_scale, y_disp, ws, src)) as stream:
        _check(lib().moe_expert_ffn_fwd_i8(
            stream, dt, act, E, d, f, _ptr(offsets), _ptr(rows), R, _ptr(xq), _ptr(x_scale),
            _ptr(src), T, k, _ptr(w1q), _ptr(w1_scale), _ptr(w3q), _ptr(w3_scale), _ptr(w2q),
            _ptr(w2_scale), _ptr(y_disp), _ptr(ws), _nbytes(ws)), "moe_expert_ffn_fwd_i8")


def moe_gated_ffn_fwd_workspace_bytes(dt, T, d, f) -> int:
    return lib().moe_gated_ffn_fwd_workspace_bytes(dt, T, d, f)


def moe_gated_ffn_bwd_workspace_bytes(dt, T, d, f) -> int:
    return lib().moe_gated_ffn_bwd_workspace_bytes(dt, T, d, f)


def moe_gated_ffn_fwd(act, x, w1, w3, w2, y, ws, add=None, h_save=None):
    """y = add + w2 (act(w1 x) * (w3 x)) for every row of x [T, d]; x, y and add may be rows of
    wider tensors."""
    (f, d), T, dtype = w1.shape, x.shape[0], x.dtype
    dt = _dt(x)
    ldx, ldy = _rows(x, "x", T, d, dtype), _rows(y, "y", T, d, dtype)
    ldadd = _rows(add, "add", T, d, dtype, optional=True)
    for name, w in (("w1", w1), ("w3", w3), ("w2", w2)):
        _need(w, f * d, name, dtype)
    if h_save is not None:
        _need(h_save, 3 * T * f, "h_save", dtype)
    with _Here(_device_of(x, w1, w3, w2, y, ws, add, h_save)) as stream:
        _check(lib().moe_gated_ffn_fwd(stream, dt, act, T, d, f, _at(x), ldx, _ptr(w1),
                                       _ptr(w3), _ptr(w2), _at(add), ldadd, _ptr(h_save), _at(y),
                                       ldy, _ptr(ws), _nbytes(ws)), "moe_gated_ffn_fwd")


def moe_gated_ffn_bwd(act, x, h_save, w1, w3, w2, dy, dx, dw1, dw3, dw2, ws, add=None):
    """Gradients of moe_gated_ffn_fwd; dw1, dw3, dw2 all float32 or all of the layer's type."""
    (f, d), T, dtype = w1.shape, x.shape[0], x.dtype
    dt = _dt(x)
    ldx, lddy, lddx = (_rows(t, n, T, d, dtype) for t, n in ((x, "x"), (dy, "dy"), (dx, "dx")))
    ldadd = _rows(add, "add", T, d, dtype, optional=True)
    _need(h_save, 3 * T * f, "h_save", dtype)
    for name, w in (("w1", w1), ("w3", w3), ("w2", w2)):
        _need(w, f * d, name, dtype)
    if dw1 is None or dw1.dtype not in (dtype, _F32):
        raise MoEError(f"dw1: a tensor of {dtype} or float32 is needed")
    for name, w in (("dw1", dw1), ("dw3", dw3), ("dw2", dw2)):
        _need(w, f * d, name, dw1.dtype)
    with _Here(_device_of(x, h_save, w1, w3, w2, dy, dx, dw1, dw3, dw2, ws, add)) as stream:
        _check(lib().moe_gated_ffn_bwd(stream, dt, act, T, d, f, _at(x), ldx, _ptr(h_save),
                                       _ptr(w1), _ptr(w3), _ptr(w2), _at(dy), lddy, _at(add),
                                       ldadd, _at(dx), lddx, _dt(dw1), _ptr(dw1), _ptr(dw3),
                                       _ptr(dw2), _ptr(ws), _nbytes(ws)), "moe_gated_ffn_bwd")


def moe_gate_bwd_workspace_bytes(T, d, E) -> int:
    return lib().moe_gate_bwd_workspace_bytes(T, d, E)


@_on_its_device
def moe_gate_bwd(x, logits, ids, dweights, renorm, dlogits, dw_g, ws, dprob_coef=None):
    T, d = x.shape
    E = logits.shape[1]
    k = ids.shape[1]
    _need(logits, T * E, "logits", _F32)
    _need(ids, T * k, "ids", _I32)
    _need(dweights, T * k, "dweights", _F32)
    _need(dprob_coef, E, "dprob_coef", _F32, optional=True)
    _need(dlogits, T * E, "dlogits", _F32)
    _need(dw_g, E * d, "dw_g", _F32)
    _check(lib().moe_gate_bwd(_stream(), _dt(x), T, d, E, k, int(renorm), _ptr(x), _ptr(logits),
                              _ptr(ids), _ptr(dweights), _ptr(dprob_coef), _ptr(dlogits),
                              _ptr(dw_g), _ptr(ws), _nbytes(ws)), "moe_gate_bwd")


@_on_its_device
def moe_dispatch_bwd(dx_disp, dest_row, E, dlogits, w_g, dx):
    T, k = dest_row.shape
    d = dx.shape[1]
    _need(dx_disp, dx_disp.shape[0] * d, "dx_disp", dx.dtype)
    _need(dest_row, T * k, "dest_row", _I32)
    _need(dlogits, T * E, "dlogits", _F32, optional=True)
    _need(w_g, E * d, "w_g", dx.dtype, optional=True)
    _need(dx, T * d, "dx")
    _check(lib().moe_dispatch_bwd(_stream(), _dt(dx), T, d, E, k, dx_disp.shape[0],
                                  _ptr(dx_disp), _ptr(dest_row), _ptr(dlogits), _ptr(w_g),
                                  _ptr(dx)), "moe_dispatch_bwd")


# ---- loss-side operators ------------------------------------------------------
def moe_balance_workspace_bytes(T, E) -> int:
    return lib().moe_balance_workspace_bytes(T, E)


@_on_its_device
def moe_balance_fwd(logits, counts, k, lam, loss, dprob_coef, ws):
    T, E = logits.shape
    _need(logits, T * E, "logits", _F32)
    _need(counts, E, "counts", _I32)
    _need(loss, 1, "loss", _F32)
    _need(dprob_coef, E, "dprob_coef", _F32)
    _check(lib().moe_balance_fwd(_stream(), T, E, k, float(lam), _ptr(logits), _ptr(counts),
                                 _ptr(loss), _ptr(dprob_coef), _ptr(ws), _nbytes(ws)),
           "moe_balance_fwd")


@_on_its_device
def moe_aggregate_spec(y_disp, dest_row, out):
    T, k = dest_row.shape
    d = out.shape[1]
    _need(y_disp, y_disp.shape[0] * d, "y_disp", out.dtype)
    _need(dest_row, T * k, "dest_row", _I32)
    _need(out, T * k * d, "out")
    _check(lib().moe_aggregate_spec(_stream(), _dt(out), T, d, k, _ptr(y_disp), _ptr(dest_row),
                                    y_disp.shape[0], _ptr(out)), "moe_aggregate_spec")


def moe_spec_loss_workspace_bytes(T) -> int:
    return lib().moe_spec_loss_workspace_bytes(T)


@_on_its_device
def moe_spec_loss(y_disp, dest_row, weights, target, dy_disp, dweights, loss, ws):
    T, k = dest_row.shape
    d = target.shape[1]
    R = y_disp.shape[0]
    _need(y_disp, R * d, "y_disp", target.dtype)
    _need(dest_row, T * k, "dest_row", _I32)
    _need(weights, T * k, "weights", _F32)
    _need(target, T * d, "target")
    _need(dy_disp, R * d, "dy_disp", target.dtype)
    _need(dweights, T * k, "dweights", _F32)
    _need(loss, 1, "loss", _F32)
    _check(lib().moe_spec_loss(_stream(), _dt(target), T, d, k, _ptr(y_disp), _ptr(dest_row),
                               _ptr(weights), _ptr(target), y_disp.shape[0], _ptr(dy_disp),
                               _ptr(dweights), _ptr(loss), _ptr(ws), _nbytes(ws)),
           "moe_spec_loss")


def moe_vocab_loss_workspace_bytes(dt, T, d, V, dw_dt=None) -> int:
    """dw_dt: the type of dw, or None without gradients."""
    return lib().moe_vocab_loss_workspace_bytes(dt, T, d, V, int(dw_dt is not None), dt if dw_dt is None else dw_dt)


def moe_vocab_loss(x, w, targets, loss, lse, status, ws, scale=1.0, weights=None, dx=None, dw=None):
    """Cross entropy of x w^T against targets [T] (negative: ignored) -> loss [T], lse [T] (or None);
    with dx and dw (float32 or the layer's type) the gradients of sum_t scale weights_t loss_t.  x [T, d] and
    dx may be rows of wider tensors; w [V, d]."""
    (T, d), V, dtype = x.shape, w.shape[0], x.dtype
    dt = _dt(x)
    ldx, lddx = _rows(x, "x", T, d, dtype), _rows(dx, "dx", T, d, dtype, optional=True)
    if tuple(w.shape) != (V, d):
        raise MoEError(f"w has shape {tuple(w.shape)}, expected {(V, d)}")
    _need(w, V * d, "w", dtype)
    _need(targets, T, "targets", _I32)
    _need(weights, T, "weights", _F32, optional=True)
    _need(loss, T, "loss", _F32)
    _need(lse, T, "lse", _F32, optional=True)
    _need(status, 1, "status", _I32)
    if (dx is None) != (dw is None):
        raise MoEError("dx and dw: both or neither")
    if dw is not None and dw.dtype not in (dtype, _F32):
        raise MoEError(f"dw: a tensor of {dtype} or float32 is needed")
    _need(dw, V * d, "dw", optional=True)
    with _Here(_device_of(x, w, targets, loss, lse, status, ws, weights, dx, dw)) as stream:
        _check(lib().moe_vocab_loss(stream, dt, T, d, V, _at(x), ldx, _ptr(w), _ptr(targets), scale,
                                    _ptr(weights), _ptr(loss), _ptr(lse), _at(dx), lddx,
                                    dt if dw is None else _dt(dw), _ptr(dw), _ptr(status), _ptr(ws),
                                    _nbytes(ws)), "moe_vocab_loss")


# ---- sample assignment caching ------------------------------------------------
@_on_its_device
def moe_cache_update(fresh_ids, cached, cache_out, unchanged):
    T, k = fresh_ids.shape
    for t, name in ((fresh_ids, "fresh_ids"), (cached, "cached"), (cache_out, "cache_out")):
        _need(t, T * k, name, _I32)
    _need(unchanged, 1, "unchanged", _I32)
    _check(lib().moe_cache_update(_stream(), T, k, _ptr(fresh_ids), _ptr(cached), _ptr(cache_out),
                                  _ptr(unchanged)), "moe_cache_update")


@_on_its_device
def moe_cached_weights(logits, ids, renorm, weights):
    T, E = logits.shape
    k = ids.shape[1]
    _need(logits, T * E, "logits", _F32)
    _need(ids, T * k, "ids", _I32)
    _need(weights, T * k, "weights", _F32)
    _check(lib().moe_cached_weights(_stream(), T, E, k, int(renorm), _ptr(logits), _ptr(ids),
                                    _ptr(weights)), "moe_cached_weights")


def moe_caching_decision(enabled, unchanged, samples, epoch, on=(96, 100), off=(90, 100),
                         min_epoch=10) -> bool:
    r = lib().moe_caching_decision(int(bool(enabled)), int(unchanged), int(samples), int(epoch),
                                   on[0], on[1], off[0], off[1], int(min_epoch))
    if r < 0:
        raise MoEError("moe_caching_decision: invalid arguments")
    return bool(r)


# ---- capacity policy at the launch frontier --------------------------------------
def moe_capacity_trigger(T, counts, cap, grow, shrink, cap_min=0):
    """Host trigger: returns (new capacities, recompiled)."""
    E = len(counts)
    c = (ctypes.c_int32 * E)(*[int(v) for v in counts])
    C = (ctypes.c_int32 * E)(*[int(v) for v in cap])
    r = lib().moe_capacity_trigger(T, E, c, C, grow[0], grow[1], shrink[0], shrink[1], cap_min)
    if r < 0:
        raise MoEError("moe_capacity_trigger: invalid arguments")
    return list(C), bool(r)


class CapacityPolicy:
    """Owner of one moe_capacity_policy object (see include/moe.h), for tensors of one device
    (device: its index; None: the current one)."""

    def __init__(self, T, k, E, delta_launch, grow, shrink, init_cap, cap_min=0, row_align=1,
                 device: Optional[int] = None):
        init = (ctypes.c_int32 * E)(*[int(c) for c in init_cap])
        self._h = h = ctypes.c_void_p()
        self.E = E
        self.device = torch.cuda.current_device() if device is None else device
        with _Here(self.device):
            _check(lib().moe_policy_create(T, k, E, delta_launch, grow[0], grow[1], shrink[0],
                                           shrink[1], cap_min, row_align, init, ctypes.byref(h)),
                   "moe_policy_create")

    def _here(self, *tensors):
        if _device_of(*tensors) != self.device:
            raise MoEError(f"tensors on device {_device_of(*tensors)}, the policy was made for {self.device}")
        return _Here(self.device)

    def begin(self, capacity, offsets):
        """Enqueue the capacities for the next launch; returns (rows needed,
        whether the trigger recompiled)."""
        _need(capacity, self.E, "capacity", _I32)
        _need(offsets, self.E + 1, "offsets", _I32)
        rows = ctypes.c_int64()
        rec = ctypes.c_int()
        with self._here(capacity, offsets) as stream:
            _check(lib().moe_policy_begin(self._h, stream, _ptr(capacity), _ptr(offsets),
                                          ctypes.byref(rows), ctypes.byref(rec)), "moe_policy_begin")
        return rows.value, bool(rec.value)

    def end(self, counts):
        _need(counts, self.E, "counts", _I32)
        with self._here(counts) as stream:
            _check(lib().moe_policy_end(self._h, stream, _ptr(counts)), "moe_policy_end")

    def state(self):
        cap = (ctypes.c_int32 * self.E)()
        n, c, r = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int64()
        _check(lib().moe_policy_state(self._h, cap, ctypes.byref(n), ctypes.byref(c),
                                      ctypes.byref(r)), "moe_policy_state")
        return dict(cap=list(cap), launched=n.value, consumed=c.value, recompiles=r.value)

    def close(self):
        if self._h is not None and self._h.value:
            lib().moe_policy_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# ---- the weights' step ------------------------------------------------------------
ADAMW_BLOCK = 128       # values of an 8-bit state that share an exponent


def adamw_blocks(n: int) -> int:
    """Exponents of n values in 8 bits."""
    return -(-n // ADAMW_BLOCK)


class AdamWTensor:
    """One tensor of the step: weights p, gradients g (float32 or bf16), moments m and v (float32,
    or uint8 with the exponents m_exp and v_exp, uint8 [adamw_blocks(n)]), and the float32 originals
    of bf16 weights (master), all of n values."""

    __slots__ = ("p", "g", "m", "v", "master", "m_exp", "v_exp", "weight_decay")

    def __init__(self, p, g, m, v, master=None, m_exp=None, v_exp=None, weight_decay=0.0):
        n, state = p.numel(), _F32 if m_exp is None else torch.uint8
        if master is not None and p.dtype != torch.bfloat16:
            raise MoEError("master: only bf16 weights have float32 originals")
        if (m_exp is None) != (v_exp is None):
            raise MoEError("m_exp and v_exp: both or neither")
        _dt(p), _dt(g)
        for t, count, name, dtype in ((g, n, "g", g.dtype), (m, n, "m", state), (v, n, "v", state),
                                      (master, n, "master", _F32), (m_exp, adamw_blocks(n), "m_exp", state),
                                      (v_exp, adamw_blocks(n), "v_exp", state)):
            _need(t, count, name, dtype, optional=name in ("master", "m_exp", "v_exp"))
            if t is not None and t.numel() != count:
                raise MoEError(f"{name} holds {t.numel()} elements, expected {count}")
        self.p, self.g, self.m, self.v, self.master = p, g, m, v, master
        self.m_exp, self.v_exp, self.weight_decay = m_exp, v_exp, float(weight_decay)

    def arrays(self):
        """(array, whether the step writes it) of every array: all but the gradient's."""
        every = (self.p, self.m, self.v, self.master, self.m_exp, self.v_exp)
        return [(self.g, False)] + [(a, True) for a in every if a is not None]


class AdamWList:
    """Tensors of one device, checked and laid out once for moe_adamw; their memory has to stay where
    it is (the list keeps the tensors)."""

    def __init__(self, tensors):
        self.tensors = list(tensors)
        every = [a for t in self.tensors for a, _ in t.arrays()]
        self.device = _device_of(*every)
        ends = {True: 0, False: 0}   # of the arrays so far, written ones and gradients
        spans = [(a.data_ptr(), a.data_ptr() + _nbytes(a), written)
                 for t in self.tensors for a, written in t.arrays() if a.numel()]
        for at, end, written in sorted(spans):
            if at < ends[True] or (written and at < ends[False]):
                raise MoEError("weights, moments or gradients overlap: a tensor is listed twice")
            ends[written] = max(ends[written], end)
        self.args = (AdamWTensorArgs * len(self.tensors))(*[
            AdamWTensorArgs(*[_ptr(a) for a in (t.p, t.g, t.master, t.m, t.v, t.m_exp, t.v_exp)], t.p.numel(),
                            t.weight_decay, _dt(t.p), _dt(t.g)) for t in self.tensors])


def adamw_schedule(lr, beta1, beta2, step, seed=0) -> torch.Tensor:
    """float32 [4] on the host with the bits of moe_adamw_schedule, to copy to the device tensor that a
    captured step reads."""
    t = torch.tensor([lr, 1 / (1 - beta1 ** step), (1 - beta2 ** step) ** -0.5, 0.0], dtype=_F32)
    t.view(torch.int32)[3] = (int(seed) & 0xFFFFFFFF) - ((int(seed) & 0x80000000) << 1)
    return t


def moe_adamw(tensors: AdamWList, lr, beta1, beta2, eps, step, seed=0, grad_scale=None, schedule=None):
    """One AdamW step over the list; grad_scale [1] and schedule [4] (adamw_schedule) on the device."""
    _need(grad_scale, 1, "grad_scale", _F32, optional=True)
    _need(schedule, 4, "schedule", _F32, optional=True)
    if not tensors.tensors:
        return
    if _device_of(tensors.tensors[0].p, grad_scale, schedule) != tensors.device:
        raise MoEError(f"grad_scale or schedule lies elsewhere than the tensors' device {tensors.device}")
    with _Here(tensors.device) as stream:
        _check(lib().moe_adamw(stream, len(tensors.args), tensors.args, lr, beta1, beta2, eps, step,
                               int(seed) & 0xFFFFFFFF, _ptr(grad_scale), _ptr(schedule)), "moe_adamw")


def moe_adamw_unpack(tensors: AdamWList, values):
    """values: for every tensor of the list, float32 tensors [n] that take what its m and v stand for."""
    if len(values) != len(tensors.tensors):
        raise MoEError(f"{len(values)} pairs of values for {len(tensors.tensors)} tensors")
    for t, pair in zip(tensors.tensors, values):
        for a in pair:
            _need(a, t.p.numel(), "values", _F32)
        if t.m_exp is None:
            raise MoEError("a tensor of the list has its moments in 32 bits")
        if _device_of(*pair) != tensors.device:
            raise MoEError(f"values lie elsewhere than the tensors' device {tensors.device}")
    if not values:
        return
    m, v = ((_p * len(values))(*[_ptr(pair[k]) for pair in values]) for k in (0, 1))
    with _Here(tensors.device) as stream:
        _check(lib().moe_adamw_unpack(stream, len(values), tensors.args, m, v), "moe_adamw_unpack")


# ---- kernel timing (instrumentation) ----------------------------------------
def moe_timing_enable(on: bool):
    _check(lib().moe_timing_enable(1 if on else 0), "moe_timing_enable")


def moe_set_gemm_tiles(mode: int):
    """0: automatic kernel and tile choice; 1: 256x256 tiles only; 2: 128-column tiles only (bf16
    and int8; fp32 runs on 128-column tiles in both)."""
    _check(lib().moe_set_gemm_tiles(int(mode)), "moe_set_gemm_tiles")


def moe_set_dx_weight_copy(mode: int):
    """0: automatic; 1: dX reads W1/W3 K-major; 2: dX reads a transposed copy (bf16)."""
    _check(lib().moe_set_dx_weight_copy(int(mode)), "moe_set_dx_weight_copy")


def moe_timing_report() -> dict:
    """{kernel name: (launches, total ms)} since the last report."""
    buf = ctypes.create_string_buffer(1 << 16)
    lib().moe_timing_report(buf, len(buf))
    out = {}
    for line in buf.value.decode().splitlines():
        name, n, ms = line.split()
        out[name] = (int(n), float(ms))
    return out
