"""ctypes binding of libmodse.so: same names as the C ABI (include/modse.h), argument marshalling only.

PyTorch is used for device memory and streams.  Tensors are passed as raw device pointers together with
the current HIP stream; nothing is computed on this side."""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional, Sequence

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None

MODSE_F32, MODSE_BF16 = 0, 1
MODSE_ERR_INVALID_ARG = 1
STAGES = ("route", "permute", "up", "down", "combine", "bwd_prep", "bwd_dgrad", "bwd_wgrad", "bwd_router")


class ModseError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: modse status {code} ({modse_status_string(code)})")
        self.code = code


class _Desc(C.Structure):
    _fields_ = [("d_model", C.c_int32), ("n_experts", C.c_int32), ("top_k", C.c_int32),
                ("d_ff", C.POINTER(C.c_int32)), ("dtype", C.c_int)]


class _Routing(C.Structure):
    _fields_ = [("topk_idx", C.c_void_p), ("topk_w", C.c_void_p), ("counts", C.c_void_p), ("offsets", C.c_void_p),
                ("row_of", C.c_void_p), ("src_of", C.c_void_p), ("near_tie_count", C.c_void_p)]


class _MatrixSet(C.Structure):
    _fields_ = [("n_matrices", C.c_int32), ("rows", C.POINTER(C.c_int32)), ("cols", C.POINTER(C.c_int32)),
                ("G", C.POINTER(C.c_void_p)), ("U", C.POINTER(C.c_void_p)), ("dtype", C.c_int)]


class _GateExt(C.Structure):
    _fields_ = [("W_noise", C.c_void_p), ("gamma", C.c_void_p), ("eps", C.c_float), ("noise_pre", C.c_void_p),
                ("aux_alpha", C.c_float), ("probs", C.c_void_p), ("aux_f", C.c_void_p), ("aux_P", C.c_void_p),
                ("aux_loss", C.c_void_p)]


def lib_path() -> str:
    return os.path.join(_HERE, "libmodse.so")


def load_library():
    """Load libmodse.so built in-tree.  Raises if it has not been built."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        raise FileNotFoundError(f"{path} not found: build it with `python -m paper_2409_12210_amd.build`")
    lib = C.CDLL(path)
    vp, i64, sz = C.c_void_p, C.c_int64, C.c_size_t
    dp, rp = C.POINTER(_Desc), C.POINTER(_Routing)
    lib.modse_status_string.restype = C.c_char_p
    lib.modse_status_string.argtypes = [C.c_int]
    lib.modse_workspace_size.argtypes = [dp, i64, C.c_int, C.POINTER(sz)]
    lib.modse_saved_size.argtypes = [dp, i64, C.POINTER(sz)]
    lib.modse_route.argtypes = [dp, i64, vp, vp, vp, rp, vp, sz, vp]
    lib.modse_route_static.argtypes = [dp, i64, vp, vp, vp, rp, vp]
    lib.modse_layer_fwd.argtypes = [dp, i64, vp, vp, vp, vp, vp, vp, vp, rp, vp, vp, sz, vp]
    lib.modse_layer_bwd.argtypes = [dp, i64, vp, vp, vp, vp, vp, rp, vp, vp, vp, vp, vp, vp, vp, C.c_int, vp, sz, vp]
    ep = C.POINTER(_GateExt)
    lib.modse_route_ext.argtypes = [dp, i64, vp, vp, vp, ep, rp, vp, sz, vp]
    lib.modse_layer_fwd_ext.argtypes = [dp, i64, vp, vp, vp, ep, vp, vp, vp, vp, rp, vp, vp, sz, vp]
    lib.modse_layer_bwd_ext.argtypes = [dp, i64, vp, vp, ep, C.c_float, vp, vp, vp, rp, vp, vp, vp, vp, vp, vp, vp, vp,
                                        vp, C.c_int, vp, sz, vp]
    lib.modse_routing_stats.argtypes = [dp, i64, rp, vp, vp, vp]
    lib.modse_stage_timing_enable.argtypes = [C.c_int]
    lib.modse_stage_times.argtypes = [C.POINTER(C.c_float)]
    i32, f32, szp, mp = C.c_int32, C.c_float, C.POINTER(sz), C.POINTER(_MatrixSet)
    lib.modse_norm_fwd.argtypes = [i64, i32, C.c_int, vp, vp, vp, f32, vp, vp, vp, vp, vp, i32, vp]
    lib.modse_norm_bwd_workspace_size.argtypes = [i64, i32, C.c_int, szp]
    lib.modse_norm_bwd.argtypes = [i64, i32, C.c_int, vp, vp, vp, vp, vp, vp, vp, C.c_int, vp, sz, vp]
    lib.modse_logprobs_workspace_size.argtypes = [i64, i32, C.c_int, i32, szp]
    lib.modse_logprobs_fwd.argtypes = [i64, i32, C.c_int, vp, i64, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
    lib.modse_orthogonalize_workspace_size.argtypes = [mp, szp]
    lib.modse_orthogonalize.argtypes = [mp, C.POINTER(f32), i32, f32, vp, sz, vp]
    lib.modse_logprobs_bwd.argtypes = [i64, i32, C.c_int, vp, i64, vp, vp, vp, vp, vp, vp, i64, vp]
    lib.modse_embed_fwd.argtypes = [i64, i32, i32, C.c_int, vp, vp, f32, vp, vp]
    lib.modse_embed_bwd_workspace_size.argtypes = [i64, i32, i32, C.c_int, szp]
    lib.modse_embed_bwd.argtypes = [i64, i32, i32, C.c_int, vp, vp, f32, vp, C.c_int, vp, sz, vp]
    lib.modse_dropout_fwd.argtypes = [i64, i32, C.c_int, vp, vp, C.c_double, vp, C.c_uint32, vp, vp]
    lib.modse_dropout_bwd.argtypes = [i64, i32, C.c_int, vp, C.c_double, vp, C.c_uint32, vp, vp]
    lib.modse_head_workspace_size.argtypes = [i64, i32, i32, C.c_int, C.c_int, szp]
    lib.modse_head_fwd.argtypes = [i64, i32, i32, C.c_int, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.modse_head_bwd.argtypes = [i64, i32, i32, C.c_int, vp, vp, vp, vp, vp, vp, vp, C.c_int, vp, sz, vp]
    for name in ("modse_head_workspace_size", "modse_head_fwd", "modse_head_bwd", "modse_embed_fwd", "modse_embed_bwd_workspace_size",
                 "modse_embed_bwd", "modse_dropout_fwd", "modse_dropout_bwd",
                 "modse_norm_fwd", "modse_norm_bwd_workspace_size", "modse_norm_bwd", "modse_logprobs_workspace_size",
                 "modse_logprobs_fwd", "modse_logprobs_bwd", "modse_orthogonalize_workspace_size", "modse_orthogonalize",
                 "modse_workspace_size", "modse_saved_size", "modse_route", "modse_layer_fwd", "modse_layer_bwd",
                 "modse_route_ext", "modse_layer_fwd_ext", "modse_layer_bwd_ext", "modse_routing_stats",
                 "modse_route_static",
                 "modse_stage_timing_enable", "modse_stage_times"):
        getattr(lib, name).restype = C.c_int
    _LIB = lib
    return lib


def modse_status_string(code: int) -> str:
    return load_library().modse_status_string(int(code)).decode()


def _dtype_code(dtype) -> int:
    if isinstance(dtype, int):
        return dtype
    s = str(dtype)
    if s in ("f32", "torch.float32", "float32"):
        return MODSE_F32
    if s in ("bf16", "torch.bfloat16", "bfloat16"):
        return MODSE_BF16
    return 99   # let the library reject it


def _desc(d_model: int, d_ff: Sequence[int], top_k: int, dtype):
    arr = (C.c_int32 * max(len(d_ff), 1))(*[int(v) for v in d_ff])
    d = _Desc(int(d_model), len(d_ff), int(top_k), C.cast(arr, C.POINTER(C.c_int32)), _dtype_code(dtype))
    d._keepalive = arr
    return d


def _ptr(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


_RAW_STREAM = _DEVICE = None


def _stream(stream) -> Optional[int]:
    if stream is None:
        # (torch.cuda.current_stream() makes an object of it first: 3.0 us where this takes 0.2, of a call's 7.5)
        if _RAW_STREAM is None:
            _find_stream()
        return _RAW_STREAM(_DEVICE()) or None
    if isinstance(stream, int):
        return stream or None
    return stream.cuda_stream or None


def _find_stream():
    global _RAW_STREAM, _DEVICE
    import torch
    torch.cuda.init()
    _DEVICE, _RAW_STREAM = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _check(code: int, what: str, raise_on_error: bool) -> int:
    if code != 0 and raise_on_error:
        raise ModseError(code, what)
    return code


@dataclass
class Routing:
    """Device tensors that receive the routing artefacts (see modse_routing in include/modse.h)."""
    topk_idx: object
    topk_w: object
    counts: object
    offsets: object
    row_of: object
    src_of: object
    near_tie_count: object

    @staticmethod
    def empty(T: int, n_experts: int, top_k: int, device="cuda"):
        import torch
        i32 = dict(dtype=torch.int32, device=device)
        return Routing(torch.empty((T, top_k), **i32), torch.empty((T, top_k), dtype=torch.float32, device=device),
                       torch.empty(n_experts, **i32), torch.empty(n_experts + 1, **i32),
                       torch.empty((T, top_k), **i32), torch.empty(T * top_k, **i32), torch.zeros(1, **i32))

    def _c(self):
        return _Routing(*[_ptr(getattr(self, f)) for f in
                          ("topk_idx", "topk_w", "counts", "offsets", "row_of", "src_of", "near_tie_count")])


@dataclass
class GateExt:
    """Optional parts of the gate (see modse_gate_ext in include/modse.h): device tensors or None."""
    W_noise: object = None
    gamma: object = None
    eps: float = 0.0
    noise_pre: object = None
    aux_alpha: float = 0.0
    probs: object = None
    aux_f: object = None
    aux_P: object = None
    aux_loss: object = None

    def _c(self):
        return _GateExt(_ptr(self.W_noise), _ptr(self.gamma), float(self.eps), _ptr(self.noise_pre),
                        float(self.aux_alpha), _ptr(self.probs), _ptr(self.aux_f), _ptr(self.aux_P),
                        _ptr(self.aux_loss))


WS_FWD, WS_BWD, WS_FWD_SAVED = 0, 1, 2   # `which` of modse_workspace_size (MODSE_WS_* in include/modse.h)


def modse_workspace_size(d_model, d_ff, top_k, dtype, T, which=WS_FWD, raise_on_error=True):
    out = C.c_size_t(0)
    d = _desc(d_model, d_ff, top_k, dtype)
    code = load_library().modse_workspace_size(C.byref(d), int(T), int(which), C.byref(out))
    _check(code, "modse_workspace_size", raise_on_error)
    return out.value if code == 0 else code


def modse_saved_size(d_model, d_ff, top_k, dtype, T, raise_on_error=True):
    out = C.c_size_t(0)
    d = _desc(d_model, d_ff, top_k, dtype)
    code = load_library().modse_saved_size(C.byref(d), int(T), C.byref(out))
    _check(code, "modse_saved_size", raise_on_error)
    return out.value if code == 0 else code


def modse_route(d_model, d_ff, top_k, dtype, T, x, W_gate, logit_bias, routing: Routing, ws, ws_bytes=None,
                stream=None, raise_on_error=True) -> int:
    d = _desc(d_model, d_ff, top_k, dtype)
    r = routing._c() if routing is not None else None
    nbytes = ws_bytes if ws_bytes is not None else (ws.numel() * ws.element_size() if ws is not None else 0)
    code = load_library().modse_route(C.byref(d), int(T), _ptr(x), _ptr(W_gate), _ptr(logit_bias),
                                      C.byref(r) if r is not None else None, _ptr(ws), nbytes, _stream(stream))
    return _check(code, "modse_route", raise_on_error)


def modse_route_static(d_model, d_ff, top_k, dtype, T, x, W_gate, logit_bias, routing: Routing, stream=None,
                       raise_on_error=True) -> int:
    d = _desc(d_model, d_ff, top_k, dtype)
    r = routing._c() if routing is not None else None
    code = load_library().modse_route_static(C.byref(d), int(T), _ptr(x), _ptr(W_gate), _ptr(logit_bias),
                                             C.byref(r) if r is not None else None, _stream(stream))
    return _check(code, "modse_route_static", raise_on_error)


def modse_layer_fwd(d_model, d_ff, top_k, dtype, T, x, W_gate, logit_bias, W1, W3, W2, y,
                    routing: Optional[Routing], saved, ws, ws_bytes=None, stream=None, raise_on_error=True) -> int:
    d = _desc(d_model, d_ff, top_k, dtype)
    r = routing._c() if routing is not None else None
    nbytes = ws_bytes if ws_bytes is not None else (ws.numel() * ws.element_size() if ws is not None else 0)
    code = load_library().modse_layer_fwd(C.byref(d), int(T), _ptr(x), _ptr(W_gate), _ptr(logit_bias), _ptr(W1),
                                          _ptr(W3), _ptr(W2), _ptr(y), C.byref(r) if r is not None else None,
                                          _ptr(saved), _ptr(ws), nbytes, _stream(stream))
    return _check(code, "modse_layer_fwd", raise_on_error)


def modse_layer_bwd(d_model, d_ff, top_k, dtype, T, x, W_gate, W1, W3, W2, routing: Routing, saved, dY, dX, dW_gate,
                    dW1, dW3, dW2, accumulate, ws, ws_bytes=None, stream=None, raise_on_error=True) -> int:
    d = _desc(d_model, d_ff, top_k, dtype)
    r = routing._c() if routing is not None else None
    nbytes = ws_bytes if ws_bytes is not None else (ws.numel() * ws.element_size() if ws is not None else 0)
    code = load_library().modse_layer_bwd(C.byref(d), int(T), _ptr(x), _ptr(W_gate), _ptr(W1), _ptr(W3), _ptr(W2),
                                          C.byref(r) if r is not None else None, _ptr(saved), _ptr(dY), _ptr(dX),
                                          _ptr(dW_gate), _ptr(dW1), _ptr(dW3), _ptr(dW2), int(bool(accumulate)),
                                          _ptr(ws), nbytes, _stream(stream))
    return _check(code, "modse_layer_bwd", raise_on_error)


def _nbytes(ws, ws_bytes):
    return ws_bytes if ws_bytes is not None else (ws.numel() * ws.element_size() if ws is not None else 0)


def modse_route_ext(d_model, d_ff, top_k, dtype, T, x, W_gate, logit_bias, ext: Optional[GateExt], routing: Routing,
                    ws, ws_bytes=None, stream=None, raise_on_error=True) -> int:
    d = _desc(d_model, d_ff, top_k, dtype)
    r = routing._c() if routing is not None else None
    e = ext._c() if ext is not None else None
    code = load_library().modse_route_ext(C.byref(d), int(T), _ptr(x), _ptr(W_gate), _ptr(logit_bias),
                                          C.byref(e) if e is not None else None,
                                          C.byref(r) if r is not None else None, _ptr(ws), _nbytes(ws, ws_bytes),
                                          _stream(stream))
    return _check(code, "modse_route_ext", raise_on_error)


def modse_layer_fwd_ext(d_model, d_ff, top_k, dtype, T, x, W_gate, logit_bias, ext: Optional[GateExt], W1, W3, W2, y,
                        routing: Optional[Routing], saved, ws, ws_bytes=None, stream=None, raise_on_error=True) -> int:
    d = _desc(d_model, d_ff, top_k, dtype)
    r = routing._c() if routing is not None else None
    e = ext._c() if ext is not None else None
    code = load_library().modse_layer_fwd_ext(C.byref(d), int(T), _ptr(x), _ptr(W_gate), _ptr(logit_bias),
                                              C.byref(e) if e is not None else None, _ptr(W1), _ptr(W3), _ptr(W2),
                                              _ptr(y), C.byref(r) if r is not None else None, _ptr(saved), _ptr(ws),
                                              _nbytes(ws, ws_bytes), _stream(stream))
    return _check(code, "modse_layer_fwd_ext", raise_on_error)


def modse_layer_bwd_ext(d_model, d_ff, top_k, dtype, T, x, W_gate, ext: Optional[GateExt], aux_grad, W1, W3, W2,
                        routing: Routing, saved, dY, dX, dW_gate, dW_noise, dgamma, dW1, dW3, dW2, accumulate, ws,
                        ws_bytes=None, stream=None, raise_on_error=True) -> int:
    d = _desc(d_model, d_ff, top_k, dtype)
    r = routing._c() if routing is not None else None
    e = ext._c() if ext is not None else None
    code = load_library().modse_layer_bwd_ext(C.byref(d), int(T), _ptr(x), _ptr(W_gate),
                                              C.byref(e) if e is not None else None, float(aux_grad), _ptr(W1),
                                              _ptr(W3), _ptr(W2), C.byref(r) if r is not None else None, _ptr(saved),
                                              _ptr(dY), _ptr(dX), _ptr(dW_gate), _ptr(dW_noise), _ptr(dgamma),
                                              _ptr(dW1), _ptr(dW3), _ptr(dW2), int(bool(accumulate)), _ptr(ws),
                                              _nbytes(ws, ws_bytes), _stream(stream))
    return _check(code, "modse_layer_bwd_ext", raise_on_error)


def modse_routing_stats(d_model, d_ff, top_k, dtype, T, routing: Routing, slot_counts, summary, stream=None,
                        raise_on_error=True) -> int:
    d = _desc(d_model, d_ff, top_k, dtype)
    r = routing._c() if routing is not None else None
    code = load_library().modse_routing_stats(C.byref(d), int(T), C.byref(r) if r is not None else None,
                                              _ptr(slot_counts), _ptr(summary), _stream(stream))
    return _check(code, "modse_routing_stats", raise_on_error)


def modse_stage_timing_enable(on: bool) -> int:
    return _check(load_library().modse_stage_timing_enable(int(bool(on))), "modse_stage_timing_enable", True)


def modse_stage_times() -> dict:
    buf = (C.c_float * len(STAGES))()
    _check(load_library().modse_stage_times(buf), "modse_stage_times", True)
    return {name: float(buf[i]) for i, name in enumerate(STAGES)}


# ---------------------------------------------------------------- the operators around the layer (see include/modse.h)
# A tensor that is of another type than the library reads, or whose elements do not follow each other, is refused as an invalid
# argument: int64 targets, a slice of columns, an expanded scalar.  (Raw pointers are taken as they are.)

class _Unfit(Exception):
    pass


_KINDS = {}


def _kind(dtype):
    """The code of `dtype`, and the types of tensors: its own (None where the library refuses it), float32, int32."""
    import torch
    code = _dtype_code(dtype)
    kind = code, {MODSE_F32: torch.float32, MODSE_BF16: torch.bfloat16}.get(code), torch.float32, torch.int32
    _KINDS[dtype] = kind
    return kind


def _data(t, dtype) -> Optional[int]:
    """The pointer of a tensor of `dtype` (None: the library refuses the type that the call names) whose elements lie side by side."""
    if t is None:
        return None
    try:      # (raw pointers have no type; to ask for them first costs a decode call another 0.3 us of 5 to 8)
        if (t.dtype is dtype or dtype is None) and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        return t
    raise _Unfit(f"{t.dtype} of shape {tuple(t.shape)} and strides {t.stride()}, expected contiguous {dtype or 'elements'}")


def _bytes(t) -> Optional[int]:
    """The pointer of a contiguous tensor of one byte an element."""
    if t is None:
        return None
    try:
        if t.element_size() == 1 and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        return t
    raise _Unfit(f"{t.dtype} of shape {tuple(t.shape)} and strides {t.stride()}, expected contiguous bytes")


def _rows(t, dtype) -> Optional[int]:
    """The pointer of a tensor of `dtype` whose strides are looked at elsewhere."""
    if t is None or isinstance(t, int):
        return t
    if t.dtype is not dtype and dtype is not None:
        raise _Unfit(f"{t.dtype}, expected {dtype}")
    return t.data_ptr()


def _unfit(e: _Unfit, what: str, raise_on_error: bool) -> int:
    return _check(MODSE_ERR_INVALID_ARG, f"{what}: {e}", raise_on_error)


def modse_norm_fwd(T, d_model, dtype, x, residual, gamma, eps, y, h, rstd, q=None, scale=None, group=0, stream=None,
                   raise_on_error=True) -> int:
    kind, own, f32, _ = _KINDS.get(dtype) or _kind(dtype)
    try:
        code = (_LIB or load_library()).modse_norm_fwd(T, d_model, kind, _data(x, own), _data(residual, own), _data(gamma, own), eps, _data(y, own),
                                             _data(h, own), _data(rstd, f32), _bytes(q), _data(scale, f32), group, _stream(stream))
    except _Unfit as e:
        return _unfit(e, "modse_norm_fwd", raise_on_error)
    return code and _check(code, "modse_norm_fwd", raise_on_error)


def modse_norm_bwd_workspace_size(T, d_model, dtype, raise_on_error=True):
    out = C.c_size_t(0)
    code = load_library().modse_norm_bwd_workspace_size(T, d_model, _dtype_code(dtype), C.byref(out))
    _check(code, "modse_norm_bwd_workspace_size", raise_on_error)
    return out.value if code == 0 else code


def modse_norm_bwd(T, d_model, dtype, h, gamma, rstd, dY, dH, dX, dgamma, accumulate, ws, ws_bytes=None, stream=None,
                   raise_on_error=True) -> int:
    kind, own, f32, _ = _KINDS.get(dtype) or _kind(dtype)
    try:
        code = (_LIB or load_library()).modse_norm_bwd(T, d_model, kind, _data(h, own), _data(gamma, own), _data(rstd, f32), _data(dY, own),
                                             _data(dH, own), _data(dX, own), _data(dgamma, f32), int(bool(accumulate)), _ptr(ws),
                                             _nbytes(ws, ws_bytes), _stream(stream))
    except _Unfit as e:
        return _unfit(e, "modse_norm_bwd", raise_on_error)
    return code and _check(code, "modse_norm_bwd", raise_on_error)


def _row_distance(t, ld, vocab: int) -> int:
    """Elements from one row to the next: as told, else the tensor's own (vocab for a raw pointer or a tensor of one
    dimension).  -1, which the library refuses, for a tensor whose entries do not lie side by side, or whose rows do not
    follow each other at one distance: of more than two dimensions only those that could be flattened in front of the
    last are rows of a matrix."""
    if ld is not None:
        return ld
    if t is None or isinstance(t, int):
        return vocab
    stride = t.stride()
    if len(stride) == 2 and stride[1] == 1 and stride[0] >= vocab:
        return stride[0]
    shape = t.shape
    if not shape or (stride[-1] != 1 and vocab > 1):
        return -1
    distance = rows = None
    for n, step in zip(shape[-2::-1], stride[-2::-1]):       # from the innermost rows outwards
        if n == 1:
            continue
        if distance is None:
            distance, rows = step, n
        elif step != distance * rows:
            return -1
        else:
            rows *= n
    if distance is None:                                      # one row
        return vocab if len(shape) == 1 else max(stride[-2], vocab)
    return distance


def modse_logprobs_workspace_size(T, vocab, dtype, top=0, raise_on_error=True):
    out = C.c_size_t(0)
    code = load_library().modse_logprobs_workspace_size(T, vocab, _dtype_code(dtype), top, C.byref(out))
    _check(code, "modse_logprobs_workspace_size", raise_on_error)
    return out.value if code == 0 else code


def modse_logprobs_fwd(T, vocab, dtype, logits, targets, logp, stats, entropy, top, top_idx, top_logp, ws, ws_bytes=None,
                       ld_logits=None, stream=None, raise_on_error=True) -> int:
    kind, own, f32, i32 = _KINDS.get(dtype) or _kind(dtype)
    try:
        code = (_LIB or load_library()).modse_logprobs_fwd(T, vocab, kind, _rows(logits, own), _row_distance(logits, ld_logits, vocab),
                                                 _data(targets, i32), _data(logp, f32), _data(stats, f32), _data(entropy, f32), top,
                                                 _data(top_idx, i32), _data(top_logp, f32), _ptr(ws), _nbytes(ws, ws_bytes),
                                                 _stream(stream))
    except _Unfit as e:
        return _unfit(e, "modse_logprobs_fwd", raise_on_error)
    return code and _check(code, "modse_logprobs_fwd", raise_on_error)


def modse_logprobs_bwd(T, vocab, dtype, logits, targets, stats, entropy, d_logp, d_entropy, d_logits, ld_logits=None,
                       ld_d_logits=None, stream=None, raise_on_error=True) -> int:
    kind, own, f32, i32 = _KINDS.get(dtype) or _kind(dtype)
    try:
        code = (_LIB or load_library()).modse_logprobs_bwd(T, vocab, kind, _rows(logits, own), _row_distance(logits, ld_logits, vocab),
                                                 _data(targets, i32), _data(stats, f32), _data(entropy, f32), _data(d_logp, f32),
                                                 _data(d_entropy, f32), _rows(d_logits, own),
                                                 _row_distance(d_logits, ld_d_logits, vocab), _stream(stream))
    except _Unfit as e:
        return _unfit(e, "modse_logprobs_bwd", raise_on_error)
    return code and _check(code, "modse_logprobs_bwd", raise_on_error)


class MatrixSet:
    """The matrices of modse_orthogonalize (see modse_matrix_set in include/modse.h): G, contiguous float32 device
    tensors of two dimensions, and U, which receive the results, of the same shapes and all of one type (float32 or
    bfloat16).  Keeps the tensors alive."""

    def __init__(self, G, U, dtype=None):
        self.G, self.U = list(G), list(U)
        n = len(self.G)
        if len(self.U) != n:
            raise ValueError(f"{n} matrices, {len(self.U)} results")
        for i, (g, u) in enumerate(zip(self.G, self.U)):
            if g.dim() != 2 or g.shape != u.shape:
                raise ValueError(f"matrix {i}: shapes {tuple(g.shape)} and {tuple(u.shape)}")
            if not (g.is_contiguous() and u.is_contiguous()):
                raise ValueError(f"matrix {i} is not contiguous")
            if _dtype_code(g.dtype) != MODSE_F32 or u.dtype != self.U[0].dtype or u.device != g.device:
                raise ValueError(f"matrix {i}: {g.dtype} on {g.device}, its result {u.dtype} on {u.device}")
        code = _dtype_code(dtype if dtype is not None else self.U[0].dtype if n else "f32")
        if n and code != _dtype_code(self.U[0].dtype):       # (the kernels write as wide as they are told)
            raise ValueError(f"results are {self.U[0].dtype}, not {dtype}")
        self._arrays = ((C.c_int32 * n)(*[g.shape[0] for g in self.G]), (C.c_int32 * n)(*[g.shape[1] for g in self.G]),
                        (C.c_void_p * n)(*[g.data_ptr() for g in self.G]), (C.c_void_p * n)(*[u.data_ptr() for u in self.U]))
        self._struct = _MatrixSet(n, *self._arrays, code)


def modse_orthogonalize_workspace_size(matrices: MatrixSet, raise_on_error=True):
    out = C.c_size_t(0)
    code = load_library().modse_orthogonalize_workspace_size(C.byref(matrices._struct), C.byref(out))
    _check(code, "modse_orthogonalize_workspace_size", raise_on_error)
    return out.value if code == 0 else code


def modse_orthogonalize(matrices: MatrixSet, coeffs, eps, ws, ws_bytes=None, stream=None, raise_on_error=True) -> int:
    flat = [float(v) for abc in coeffs for v in abc]
    if any(len(abc) != 3 for abc in coeffs):
        raise ValueError("coeffs: (a, b, c) for every step")
    code = load_library().modse_orthogonalize(C.byref(matrices._struct), (C.c_float * len(flat))(*flat), len(coeffs), eps,
                                              _ptr(ws), _nbytes(ws, ws_bytes), _stream(stream))
    return _check(code, "modse_orthogonalize", raise_on_error)


# ---------------------------------------------------------------- both ends of a model (see include/modse.h)

def modse_embed_fwd(T, d_model, vocab, dtype, tokens, E, scale, x, stream=None, raise_on_error=True) -> int:
    kind, own, _, i32 = _KINDS.get(dtype) or _kind(dtype)
    try:
        code = (_LIB or load_library()).modse_embed_fwd(T, d_model, vocab, kind, _data(tokens, i32), _data(E, own), scale, _data(x, own),
                                                        _stream(stream))
    except _Unfit as e:
        return _unfit(e, "modse_embed_fwd", raise_on_error)
    return code and _check(code, "modse_embed_fwd", raise_on_error)


def modse_embed_bwd_workspace_size(T, d_model, vocab, dtype, raise_on_error=True):
    out = C.c_size_t(0)
    code = load_library().modse_embed_bwd_workspace_size(T, d_model, vocab, _dtype_code(dtype), C.byref(out))
    _check(code, "modse_embed_bwd_workspace_size", raise_on_error)
    return out.value if code == 0 else code


def modse_embed_bwd(T, d_model, vocab, dtype, tokens, dX, scale, dE, accumulate, ws, ws_bytes=None, stream=None,
                    raise_on_error=True) -> int:
    kind, own, f32, i32 = _KINDS.get(dtype) or _kind(dtype)
    try:
        code = (_LIB or load_library()).modse_embed_bwd(T, d_model, vocab, kind, _data(tokens, i32), _data(dX, own), scale, _data(dE, f32),
                                                        int(bool(accumulate)), _ptr(ws), _nbytes(ws, ws_bytes), _stream(stream))
    except _Unfit as e:
        return _unfit(e, "modse_embed_bwd", raise_on_error)
    return code and _check(code, "modse_embed_bwd", raise_on_error)


def modse_head_workspace_size(T, d_model, vocab, dtype, which=WS_FWD, raise_on_error=True):
    out = C.c_size_t(0)
    code = load_library().modse_head_workspace_size(T, d_model, vocab, _dtype_code(dtype), which, C.byref(out))
    _check(code, "modse_head_workspace_size", raise_on_error)
    return out.value if code == 0 else code


def modse_head_fwd(T, d_model, vocab, dtype, x, W, targets, logp, log_z, ws, ws_bytes=None, stream=None, raise_on_error=True) -> int:
    kind, own, f32, i32 = _KINDS.get(dtype) or _kind(dtype)
    try:
        code = (_LIB or load_library()).modse_head_fwd(T, d_model, vocab, kind, _data(x, own), _data(W, own), _data(targets, i32),
                                                       _data(logp, f32), _data(log_z, f32), _ptr(ws), _nbytes(ws, ws_bytes), _stream(stream))
    except _Unfit as e:
        return _unfit(e, "modse_head_fwd", raise_on_error)
    return code and _check(code, "modse_head_fwd", raise_on_error)


def modse_head_bwd(T, d_model, vocab, dtype, x, W, targets, d_logp, logp, dX, dW, accumulate, ws, ws_bytes=None, stream=None,
                   raise_on_error=True) -> int:
    kind, own, f32, i32 = _KINDS.get(dtype) or _kind(dtype)
    try:
        code = (_LIB or load_library()).modse_head_bwd(T, d_model, vocab, kind, _data(x, own), _data(W, own), _data(targets, i32),
                                                       _data(d_logp, f32), _data(logp, f32), _data(dX, own), _data(dW, f32),
                                                       int(bool(accumulate)), _ptr(ws), _nbytes(ws, ws_bytes), _stream(stream))
    except _Unfit as e:
        return _unfit(e, "modse_head_bwd", raise_on_error)
    return code and _check(code, "modse_head_bwd", raise_on_error)


def _generator(rng) -> Optional[int]:
    """The pointer of seed and offset: two integers of 64 bits on the device.  (On the host they would be easy to make.)"""
    if rng is None or isinstance(rng, int):
        return rng
    if rng.dtype in (_WIDE or _find_wide()) and rng.is_cuda and rng.numel() == 2 and rng.is_contiguous():
        return rng.data_ptr()
    raise _Unfit(f"{rng.dtype} of shape {tuple(rng.shape)} on {rng.device}, expected two int64 on the GPU: seed and offset")


_WIDE = ()


def _find_wide():
    global _WIDE
    import torch
    _WIDE = (torch.int64, torch.uint64)
    return _WIDE


def modse_dropout_fwd(T, d_model, dtype, x, residual, p, rng, call, y, stream=None, raise_on_error=True) -> int:
    kind, own, _, _ = _KINDS.get(dtype) or _kind(dtype)
    try:
        code = (_LIB or load_library()).modse_dropout_fwd(T, d_model, kind, _data(x, own), _data(residual, own), p, _generator(rng), call,
                                                          _data(y, own), _stream(stream))
    except _Unfit as e:
        return _unfit(e, "modse_dropout_fwd", raise_on_error)
    return code and _check(code, "modse_dropout_fwd", raise_on_error)


def modse_dropout_bwd(T, d_model, dtype, dY, p, rng, call, dX, stream=None, raise_on_error=True) -> int:
    kind, own, _, _ = _KINDS.get(dtype) or _kind(dtype)
    try:
        code = (_LIB or load_library()).modse_dropout_bwd(T, d_model, kind, _data(dY, own), p, _generator(rng), call, _data(dX, own),
                                                          _stream(stream))
    except _Unfit as e:
        return _unfit(e, "modse_dropout_bwd", raise_on_error)
    return code and _check(code, "modse_dropout_bwd", raise_on_error)
