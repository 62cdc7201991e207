"""Binding of the edge operators of libjdob.so (include/jdob_edge.h).

What the edge GPU computes for the users that a policy offloads: `norm` (RMS norm of rows with the residual's
addition, in the rows' type or in 8 bits with scales), `project` (the projection that all users share beside each
row's low-rank adapter) and `attend` (causal attention of packed sequences of different lengths).

Argument marshalling only, like paper_2504_14611_amd.jdob: the work runs in the HIP kernels of the library, and
there is no fallback.  Tensors are device tensors (others are refused); outputs and workspaces that the caller does
not pass are allocated by torch on the stream that the call runs on.  `stream` is a raw HIP stream handle (default:
torch's current stream of the tensors' device).  The operators are forward only: outputs carry no gradient graph,
also where an input requires gradients.  Refused arguments raise jdob.JdobError with the library's status code.
"""

from __future__ import annotations

import ctypes as C
from typing import Dict, Optional

import torch

from . import jdob

try:  # a call's overhead on the host counts with few rows: these take a tenth of the public calls' time
    from torch._C import _cuda_getCurrentRawStream as _raw_stream, _cuda_getDevice as _current_device
except ImportError:
    def _raw_stream(index):
        return torch.cuda.current_stream(index).cuda_stream

    def _current_device():
        return torch.cuda.current_device()

EDGE_BF16, EDGE_F16, EDGE_F32 = 0, 1, 2
MAX_ROWS, MAX_NORM_DIM, MAX_RANK, MAX_HEAD_DIM, MAX_SEQUENCES = 1 << 30, 16384, 256, 128, 65535
_MAX_I32 = 0x7fffffff

EXPORTS = ("jdob_edge_norm", "jdob_edge_project", "jdob_edge_project_workspace", "jdob_edge_attend",
           "jdob_edge_attend_workspace")

_P, _I32, _I64, _F32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float


class NormArgs(C.Structure):
    _fields_ = [("rows", _I32), ("dim", _I32), ("dtype", _I32), ("eps", _F32), ("x", _P), ("x_stride", _I64),
                ("residual", _P), ("residual_stride", _I64), ("weight", _P), ("sum", _P), ("sum_stride", _I64),
                ("out", _P), ("out_stride", _I64), ("q", _P), ("q_stride", _I64), ("scale", _P)]


class ProjectArgs(C.Structure):
    _fields_ = [("rows", _I32), ("in_dim", _I32), ("out_dim", _I32), ("dtype", _I32), ("bits8", _I32),
                ("x", _P), ("x_stride", _I64), ("x_scale", _P), ("weight", _P), ("weight_stride", _I64),
                ("weight_scale", _P), ("num_adapters", _I32), ("max_rank", _I32), ("down", _P), ("up", _P),
                ("gain", _P), ("rank", _P), ("row_adapter", _P), ("out", _P), ("out_stride", _I64),
                ("workspace", _P), ("workspace_bytes", _I64)]


class AttendArgs(C.Structure):
    _fields_ = [("num_sequences", _I32), ("num_heads", _I32), ("num_kv_heads", _I32), ("head_dim", _I32),
                ("dtype", _I32), ("max_queries", _I32), ("max_keys", _I32), ("scale", _F32),
                ("query_rows", _I64), ("key_rows", _I64), ("q", _P), ("q_stride", _I64), ("q_head_stride", _I64),
                ("k", _P), ("k_stride", _I64), ("k_head_stride", _I64), ("v", _P), ("v_stride", _I64),
                ("v_head_stride", _I64), ("query_start", _P), ("key_start", _P), ("key_count", _P), ("out", _P),
                ("out_stride", _I64), ("out_head_stride", _I64), ("workspace", _P), ("workspace_bytes", _I64)]


_lib = None


def load():
    """libjdob.so with the edge operators' prototypes; raises OSError if it has not been built."""
    global _lib
    if _lib is None:
        lib = jdob.load()
        for name, args in (("norm", NormArgs), ("project", ProjectArgs), ("attend", AttendArgs)):
            call = getattr(lib, "jdob_edge_" + name)
            call.argtypes, call.restype = [C.POINTER(args), C.c_void_p], C.c_int
            if args is not NormArgs:
                size = getattr(lib, f"jdob_edge_{name}_workspace")
                size.argtypes, size.restype = [C.POINTER(args)], C.c_int64
        _lib = lib
    return _lib


_CODES16 = {torch.bfloat16: EDGE_BF16, torch.float16: EDGE_F16}
_CODES = {**_CODES16, torch.float32: EDGE_F32}


def _refuse(where: str, why: str, code: int = jdob.JDOB_ERR_INVALID_ARG):
    raise jdob.JdobError(code, f"{where}: {why}")


def _dtype(t, where: str, codes=_CODES16) -> int:
    code = codes.get(t)
    if code is None:
        _refuse(where, f"type {t}", jdob.JDOB_ERR_UNSUPPORTED)
    return code


def _array(t, where: str, name: str, shape, dtype, device):
    """A tensor whose shape, type and device the kernels take as given, with its innermost dimension contiguous."""
    if t.dtype is not dtype or t.shape != shape or t.device != device:
        _refuse(where, f"{name} is {tuple(t.shape)} {t.dtype} on {t.device}, "
                       f"expected {tuple(shape)} {dtype} on {device}")
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        _refuse(where, f"{name}'s last dimension is not contiguous")
    return t.data_ptr()


def _dense(t, where: str, name: str, shape, dtype, device):
    if t.dtype is not dtype or t.shape != shape or t.device != device or not t.is_contiguous():
        _array(t, where, name, shape, dtype, device)
        _refuse(where, f"{name} is not contiguous")
    return t.data_ptr()


def _row_stride(t, width: int) -> int:
    # a single row's stride is never used, whatever torch says it is
    stride = t.stride(0)
    return stride if stride > width or t.shape[0] > 1 else width


def _enter(device, stream, where: str):
    """The raw stream of a call on `device`, and the context (or None) in which its outputs are allocated and its
    kernels launched: `stream`'s, or the device's where it is not torch's current one.  Kernels that are given
    memory of the host would fault."""
    if device.type != "cuda":
        _refuse(where, f"tensors on {device}, expected a GPU's")
    if stream is not None:
        return stream, torch.cuda.stream(torch.cuda.ExternalStream(stream, device=device))
    index = device.index
    return _raw_stream(index), None if index == _current_device() else torch.cuda.device(index)


def norm(x, weight, eps: float = 1e-6, residual=None, bits8: bool = False, out16: Optional[bool] = None,
         into: Optional[dict] = None, stream=None) -> Dict[str, object]:
    """jdob_edge_norm of x [rows, dim]: a dict with `sum` (x + residual, None without a residual), `out` (the
    normalised rows in x's type; with bits8 only where out16 is true) and, with bits8, `q` and `scale`.
    `into` holds the caller's own buffers for any of them; `sum` may be x or residual itself."""
    where = "jdob_edge_norm"
    if x.dim() != 2:
        _refuse(where, "x has rows and columns")
    shape, dtype, dev = x.shape, x.dtype, x.device
    rows, dim = shape
    if rows > MAX_ROWS or dim > MAX_NORM_DIM:
        _refuse(where, f"{rows} rows of {dim}", jdob.JDOB_ERR_UNSUPPORTED)
    if out16 is None:
        out16 = not bits8
    if not (bits8 or out16):
        _refuse(where, "neither output is asked for")
    a = NormArgs(rows, dim, _dtype(dtype, where, _CODES), eps, _array(x, where, "x", shape, dtype, dev),
                 _row_stride(x, dim))
    a.weight = _dense(weight, where, "weight", (dim,), dtype, dev)
    if residual is not None:
        a.residual = _array(residual, where, "residual", shape, dtype, dev)
        a.residual_stride = _row_stride(residual, dim)
    handle, context = _enter(dev, stream, where)
    if context is not None:
        with context:
            return _norm(a, where, x, bits8, out16, into, handle)
    return _norm(a, where, x, bits8, out16, into, handle)


def _norm(a, where, x, bits8, out16, into, handle):
    shape, dtype, dev, dim = x.shape, x.dtype, x.device, a.dim
    total = out = q = scale = None
    if a.residual_stride:
        total = into.get("sum") if into else None
        if total is None:
            total = torch.empty_like(x, memory_format=torch.contiguous_format)
            a.sum, a.sum_stride = total.data_ptr(), dim
        else:
            a.sum, a.sum_stride = _array(total, where, "sum", shape, dtype, dev), _row_stride(total, dim)
    if out16:
        out = into.get("out") if into else None
        if out is None:
            out = torch.empty_like(x, memory_format=torch.contiguous_format)
            a.out, a.out_stride = out.data_ptr(), dim
        else:
            a.out, a.out_stride = _array(out, where, "out", shape, dtype, dev), _row_stride(out, dim)
    if bits8:
        q, scale = (into.get("q"), into.get("scale")) if into else (None, None)
        if q is None:
            q = torch.empty_like(x, dtype=torch.int8, memory_format=torch.contiguous_format)
            a.q, a.q_stride = q.data_ptr(), dim
        else:
            a.q, a.q_stride = _array(q, where, "q", shape, torch.int8, dev), _row_stride(q, dim)
        if scale is None:
            scale = torch.empty(shape[:1], dtype=torch.float32, device=dev)
            a.scale = scale.data_ptr()
        else:
            a.scale = _dense(scale, where, "scale", shape[:1], torch.float32, dev)
    code = (_lib or load()).jdob_edge_norm(C.byref(a), handle)
    if code:
        jdob._check(code, where)
    return {"sum": total, "out": out, "q": q, "scale": scale}


def project(x, weight, x_scale=None, weight_scale=None, adapters: Optional[dict] = None, row_adapter=None,
            dtype=None, out=None, workspace=None, stream=None):
    """jdob_edge_project: x [rows, in] W^T for weight [out, in], beside each row's adapter.

    x and weight are of the output's type, or int8 with x_scale [rows] and weight_scale [out] (dtype then names
    the output's type, default bfloat16).  adapters: {"down" [n, r, in], "up" [n, out, r], "gain" [n], optionally
    "rank" [n] int32} with row_adapter [rows] int32 (outside [0, n): none).  Returns out [rows, out]."""
    where = "jdob_edge_project"
    if x.dim() != 2 or weight.dim() != 2:
        _refuse(where, "x and weight have rows and columns")
    rows, i = x.shape
    o, dev = weight.shape[0], x.device
    if rows > MAX_ROWS or i > _MAX_I32 or o > _MAX_I32:  # (the library knows the smaller limits)
        _refuse(where, f"{rows} rows of {i} and {o}", jdob.JDOB_ERR_UNSUPPORTED)
    kind = x.dtype
    bits8 = kind is torch.int8
    if dtype is None:
        dtype = torch.bfloat16 if bits8 else kind
    elif not bits8 and kind is not dtype:
        _refuse(where, f"x is {kind}, expected {dtype} or int8")
    a = ProjectArgs(rows, i, o, _dtype(dtype, where), bits8, _array(x, where, "x", x.shape, kind, dev),
                    _row_stride(x, i), None, _array(weight, where, "weight", (o, i), kind, dev), _row_stride(weight, i))
    if bits8:
        if x_scale is None or weight_scale is None:
            _refuse(where, "8-bit x and weight have scales")
        a.x_scale = _dense(x_scale, where, "x_scale", (rows,), torch.float32, dev)
        a.weight_scale = _dense(weight_scale, where, "weight_scale", (o,), torch.float32, dev)
    elif x_scale is not None or weight_scale is not None:
        _refuse(where, "scales belong to 8-bit x and weight")
    if (adapters is None) != (row_adapter is None):
        _refuse(where, "adapters and row_adapter go together")
    if adapters is not None:
        down, rank = adapters["down"], adapters.get("rank")
        if down.dim() != 3:
            _refuse(where, "down is [adapters, rank, in]")
        n, most = down.shape[:2]
        if n > _MAX_I32 or most > MAX_RANK:
            _refuse(where, f"{n} adapters of rank {most}", jdob.JDOB_ERR_UNSUPPORTED)
        a.num_adapters, a.max_rank = n, most
        a.down = _dense(down, where, "down", (n, most, i), dtype, dev)
        a.up = _dense(adapters["up"], where, "up", (n, o, most), dtype, dev)
        a.gain = _dense(adapters["gain"], where, "gain", (n,), torch.float32, dev)
        a.row_adapter = _dense(row_adapter, where, "row_adapter", (rows,), torch.int32, dev)
        if rank is not None:
            a.rank = _dense(rank, where, "rank", (n,), torch.int32, dev)
    handle, context = _enter(dev, stream, where)
    if context is not None:
        with context:
            return _project(a, where, dtype, dev, out, workspace, handle)
    return _project(a, where, dtype, dev, out, workspace, handle)


def _project(a, where, dtype, dev, out, workspace, handle):
    shape = (a.rows, a.out_dim)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=dev)
        a.out, a.out_stride = out.data_ptr(), a.out_dim
    else:
        a.out, a.out_stride = _array(out, where, "out", shape, dtype, dev), _row_stride(out, a.out_dim)
    lib = _lib or load()
    if a.num_adapters:
        workspace = _workspace(a, workspace, lib.jdob_edge_project_workspace, dev, where)
    code = lib.jdob_edge_project(C.byref(a), handle)
    if code:
        jdob._check(code, where)
    return out


def _workspace(a, given, size, device, where: str):
    """Sets the caller's workspace, or a new one; none where none is needed (or the call will refuse)."""
    if given is None:
        given = size(C.byref(a))
        if given <= 0:
            return None
        given = torch.empty(given, dtype=torch.uint8, device=device)
    elif not given.is_contiguous() or given.device != device:
        _refuse(where, "workspace is contiguous, on the tensors' device")
    a.workspace, a.workspace_bytes = given.data_ptr(), given.numel() * given.element_size()
    return given


def attend(q, k, v, query_start, key_start, key_count, scale: Optional[float] = None,
           max_queries: Optional[int] = None, max_keys: Optional[int] = None, out=None, workspace=None, stream=None):
    """jdob_edge_attend: causal attention of packed sequences, q [rows, heads, dim], k and v [key rows, key heads,
    dim] (any row and head strides), query_start [n + 1] int32, key_start [n] int64, key_count [n] int32.
    Sequence u's rows query_start[u] .. query_start[u+1] stand at the end of its key_count[u] keys, which start at
    row key_start[u].  scale defaults to dim ** -0.5; max_queries and max_keys are at least the largest sequence's
    (default: all rows).  They choose the kernel for the whole call and are worth giving: without max_queries many
    single tokens look like one long prompt (32 after up to 8191 keys, 32 heads on 8: 376 us, with it 131).
    Returns out [rows, heads, dim]."""
    where = "jdob_edge_attend"
    if q.dim() != 3 or k.dim() != 3:
        _refuse(where, "q, k and v have rows, heads and columns")
    shape, dtype, dev = q.shape, q.dtype, q.device
    rows, h, d = shape
    if rows > MAX_ROWS:
        _refuse(where, f"{rows} rows", jdob.JDOB_ERR_UNSUPPORTED)
    if d % 8 or d > MAX_HEAD_DIM:
        _refuse(where, f"heads of {d}", jdob.JDOB_ERR_UNSUPPORTED)
    key_rows, g = k.shape[:2]
    n = key_count.shape[0]
    if n > MAX_SEQUENCES:
        _refuse(where, f"{n} sequences", jdob.JDOB_ERR_UNSUPPORTED)
    most = rows if max_queries is None else max_queries
    longest = key_rows if max_keys is None else max_keys
    if most < 0 or longest < 0:
        _refuse(where, f"max_queries {most}, max_keys {longest}")
    a = AttendArgs(n, h, g, d, _dtype(dtype, where), min(most, _MAX_I32), min(longest, _MAX_I32),
                   d ** -0.5 if scale is None else scale, rows, key_rows,
                   _array(q, where, "q", shape, dtype, dev), q.stride(0), q.stride(1),
                   _array(k, where, "k", (key_rows, g, d), dtype, dev), k.stride(0), k.stride(1),
                   _array(v, where, "v", (key_rows, g, d), dtype, dev), v.stride(0), v.stride(1),
                   _dense(query_start, where, "query_start", (n + 1,), torch.int32, dev),
                   _dense(key_start, where, "key_start", (n,), torch.int64, dev),
                   _dense(key_count, where, "key_count", (n,), torch.int32, dev))
    handle, context = _enter(dev, stream, where)
    if context is not None:
        with context:
            return _attend(a, where, shape, dtype, dev, out, workspace, handle)
    return _attend(a, where, shape, dtype, dev, out, workspace, handle)


def _attend(a, where, shape, dtype, dev, out, workspace, handle):
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=dev)
        a.out = out.data_ptr()
    else:
        a.out = _array(out, where, "out", shape, dtype, dev)
    a.out_stride, a.out_head_stride = out.stride(0), out.stride(1)
    lib = _lib or load()
    workspace = _workspace(a, workspace, lib.jdob_edge_attend_workspace, dev, where)
    code = lib.jdob_edge_attend(C.byref(a), handle)
    if code:
        jdob._check(code, where)
    return out
