"""Binding of the edge operators of libjdob.so (include/jdob_edge.h).

What the edge GPU computes for the users that a policy offloads: `norm` (RMS norm of rows with the residual's
addition, in the rows' type or in 8 bits with scales), `project` (the projection that all users share beside each
row's low-rank adapter) and `attend` (causal attention of packed sequences of different lengths).

Argument marshalling only, like paper_2504_14611_amd.jdob: the work runs in the HIP kernels of the library, and
there is no fallback.  Tensors are device tensors; outputs and workspaces that the caller does not pass are
allocated by torch on the stream that the call runs on.  `stream` is a raw HIP stream handle (default: torch's
current stream of the tensors' device).  Refused arguments raise jdob.JdobError with the library's status code.
"""

from __future__ import annotations

import contextlib
import ctypes as C
from typing import Dict, Optional

from . import jdob

EDGE_BF16, EDGE_F16, EDGE_F32 = 0, 1, 2
MAX_NORM_DIM, MAX_RANK, MAX_HEAD_DIM, MAX_SEQUENCES = 16384, 256, 128, 65535

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


def _refuse(where: str, why: str, code: int = jdob.JDOB_ERR_INVALID_ARG):
    raise jdob.JdobError(code, f"{where}: {why}")


def _dtype(t, where: str) -> int:
    import torch
    code = {torch.bfloat16: EDGE_BF16, torch.float16: EDGE_F16, torch.float32: EDGE_F32}.get(t)
    if code is None:
        _refuse(where, f"type {t}", jdob.JDOB_ERR_UNSUPPORTED)
    return code


def _need(ok: bool, where: str, why: str):
    if not ok:
        _refuse(where, why)


def _array(t, where: str, name: str, shape, dtype, device):
    """A tensor whose shape, type and device the kernels take as given, with its innermost dimension contiguous."""
    if t.dtype != dtype or t.device != device or tuple(t.shape) != tuple(shape):
        _refuse(where, f"{name} is {tuple(t.shape)} {t.dtype} on {t.device}, "
                       f"expected {tuple(shape)} {dtype} on {device}")
    if t.dim() and t.shape[-1] > 1 and t.stride(-1) != 1:
        _refuse(where, f"{name}'s last dimension is not contiguous")


def _dense(t, where: str, name: str, shape, dtype, device):
    _array(t, where, name, shape, dtype, device)
    _need(t.is_contiguous(), where, f"{name} is not contiguous")


def _on(device, stream):
    """The device's allocations and launches go to `stream` (a raw handle), or to torch's current stream."""
    import torch
    if device.type != "cuda":
        return contextlib.nullcontext()
    if stream is not None:
        return torch.cuda.stream(torch.cuda.ExternalStream(stream, device=device))
    if device.index is not None and device.index != torch.cuda.current_device():
        return torch.cuda.device(device)
    return contextlib.nullcontext()


def _handle(device, stream) -> Optional[int]:
    import torch
    if stream is not None or device.type != "cuda":
        return stream
    return torch.cuda.current_stream(device).cuda_stream


def _row_stride(t, width: int) -> int:
    # a single row's stride is never used, whatever torch says it is
    return t.stride(0) if t.shape[0] > 1 else max(width, t.stride(0))


def norm(x, weight, eps: float = 1e-6, residual=None, bits8: bool = False, out16: Optional[bool] = None,
         into: Optional[dict] = None, stream=None) -> Dict[str, object]:
    """jdob_edge_norm of x [rows, dim]: a dict with `sum` (x + residual, None without a residual), `out` (the
    normalised rows in x's type; with bits8 only where out16 is true) and, with bits8, `q` and `scale`.
    `into` holds the caller's own buffers for any of them; `sum` may be x or residual itself."""
    import torch
    where = "jdob_edge_norm"
    _need(x.dim() == 2, where, "x has rows and columns")
    rows, dim = x.shape
    code, dev = _dtype(x.dtype, where), x.device
    _array(x, where, "x", (rows, dim), x.dtype, dev)
    _dense(weight, where, "weight", (dim,), x.dtype, dev)
    if residual is not None:
        _array(residual, where, "residual", (rows, dim), x.dtype, dev)
    want16 = (not bits8) if out16 is None else out16
    _need(bits8 or want16, where, "neither output is asked for")
    r = dict.fromkeys(("sum", "out", "q", "scale"))
    into = into or {}
    with _on(dev, stream):
        for key, wanted, shape, dtype in (("sum", residual is not None, (rows, dim), x.dtype),
                                          ("out", want16, (rows, dim), x.dtype), ("q", bits8, (rows, dim), torch.int8),
                                          ("scale", bits8, (rows,), torch.float32)):
            if not wanted:
                continue
            t = into.get(key)
            if t is None:
                t = torch.empty(shape, dtype=dtype, device=dev)
            else:
                (_dense if key == "scale" else _array)(t, where, key, shape, dtype, dev)
            r[key] = t
        a = NormArgs(rows, dim, code, eps, x.data_ptr(), _row_stride(x, dim) if rows else dim,
                     *((residual.data_ptr(), _row_stride(residual, dim)) if residual is not None and rows else (None, 0)),
                     weight.data_ptr(), *[y for key in ("sum", "out", "q") for y in
                                          ((r[key].data_ptr(), _row_stride(r[key], dim))
                                           if r[key] is not None and rows else (None, 0))],
                     r["scale"].data_ptr() if bits8 else None)
        jdob._check(load().jdob_edge_norm(C.byref(a), _handle(dev, stream)), where)
    return r


def project(x, weight, x_scale=None, weight_scale=None, adapters: Optional[dict] = None, row_adapter=None,
            dtype=None, out=None, workspace=None, stream=None):
    """jdob_edge_project: x [rows, in] W^T for weight [out, in], beside each row's adapter.

    x and weight are of the output's type, or int8 with x_scale [rows] and weight_scale [out] (dtype then names
    the output's type, default bfloat16).  adapters: {"down" [n, r, in], "up" [n, out, r], "gain" [n], optionally
    "rank" [n] int32} with row_adapter [rows] int32 (outside [0, n): none).  Returns out [rows, out]."""
    import torch
    where = "jdob_edge_project"
    _need(x.dim() == 2 and weight.dim() == 2, where, "x and weight have rows and columns")
    (rows, i), o, dev = x.shape, weight.shape[0], x.device
    bits8 = x.dtype == torch.int8
    if dtype is None:
        dtype = torch.bfloat16 if bits8 else x.dtype
    code = _dtype(dtype, where)
    _array(x, where, "x", (rows, i), torch.int8 if bits8 else dtype, dev)
    _array(weight, where, "weight", (o, i), x.dtype, dev)
    _need((x_scale is not None and weight_scale is not None) == bits8 and
          (x_scale is None) == (weight_scale is None), where, "scales belong to 8-bit x and weight")
    if bits8:
        _dense(x_scale, where, "x_scale", (rows,), torch.float32, dev)
        _dense(weight_scale, where, "weight_scale", (o,), torch.float32, dev)
    _need((adapters is None) == (row_adapter is None), where, "adapters and row_adapter go together")
    a = ProjectArgs(rows=rows, in_dim=i, out_dim=o, dtype=code, bits8=bits8, x=x.data_ptr(), weight=weight.data_ptr(),
                    x_stride=_row_stride(x, i) if rows else i, weight_stride=_row_stride(weight, i) if o else i)
    if bits8:
        a.x_scale, a.weight_scale = x_scale.data_ptr(), weight_scale.data_ptr()
    if adapters is not None:
        down, up, gain, rank = adapters["down"], adapters["up"], adapters["gain"], adapters.get("rank")
        _need(down.dim() == 3, where, "down is [adapters, rank, in]")
        n, most = down.shape[:2]
        _dense(down, where, "down", (n, most, i), dtype, dev)
        _dense(up, where, "up", (n, o, most), dtype, dev)
        _dense(gain, where, "gain", (n,), torch.float32, dev)
        _dense(row_adapter, where, "row_adapter", (rows,), torch.int32, dev)
        a.num_adapters, a.max_rank, a.row_adapter = n, most, row_adapter.data_ptr()
        a.down, a.up, a.gain = down.data_ptr(), up.data_ptr(), gain.data_ptr()
        if rank is not None:
            _dense(rank, where, "rank", (n,), torch.int32, dev)
            a.rank = rank.data_ptr()
    lib = load()
    with _on(dev, stream):
        if out is None:
            out = torch.empty((rows, o), dtype=dtype, device=dev)
        else:
            _array(out, where, "out", (rows, o), dtype, dev)
        a.out, a.out_stride = out.data_ptr(), _row_stride(out, o) if rows else o
        if adapters is not None:
            workspace = _workspace(workspace, lib.jdob_edge_project_workspace(C.byref(a)), dev, where)
            if workspace is not None:
                a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        jdob._check(lib.jdob_edge_project(C.byref(a), _handle(dev, stream)), where)
    return out


def _workspace(given, size: int, device, where: str):
    """The caller's workspace, or one of `size` bytes; None where none is needed (or the call will refuse)."""
    import torch
    if given is not None:
        _need(given.is_contiguous() and given.device == device, where, "workspace is contiguous, on the tensors' device")
        return given
    return torch.empty(size, dtype=torch.uint8, device=device) if size > 0 else None


def attend(q, k, v, query_start, key_start, key_count, scale: Optional[float] = None,
           max_queries: Optional[int] = None, max_keys: Optional[int] = None, out=None, workspace=None, stream=None):
    """jdob_edge_attend: causal attention of packed sequences, q [rows, heads, dim], k and v [key rows, key heads,
    dim] (any row and head strides), query_start [n + 1] int32, key_start [n] int64, key_count [n] int32.
    Sequence u's rows query_start[u] .. query_start[u+1] stand at the end of its key_count[u] keys, which start at
    row key_start[u].  scale defaults to dim ** -0.5; max_queries and max_keys are at least the largest sequence's
    (default: all rows).  Returns out [rows, heads, dim]."""
    import torch
    where = "jdob_edge_attend"
    _need(q.dim() == 3 and k.dim() == 3, where, "q, k and v have rows, heads and columns")
    (rows, h, d), (key_rows, g), dev = q.shape, k.shape[:2], q.device
    code, n = _dtype(q.dtype, where), key_count.shape[0]
    _array(q, where, "q", (rows, h, d), q.dtype, dev)
    _array(k, where, "k", (key_rows, g, d), q.dtype, dev)
    _array(v, where, "v", (key_rows, g, d), q.dtype, dev)
    _dense(query_start, where, "query_start", (n + 1,), torch.int32, dev)
    _dense(key_start, where, "key_start", (n,), torch.int64, dev)
    _dense(key_count, where, "key_count", (n,), torch.int32, dev)
    a = AttendArgs(n, h, g, d, code, rows if max_queries is None else max_queries,
                   key_rows if max_keys is None else max_keys, d ** -0.5 if scale is None else scale, rows, key_rows,
                   q.data_ptr(), q.stride(0), q.stride(1), k.data_ptr(), k.stride(0), k.stride(1),
                   v.data_ptr(), v.stride(0), v.stride(1), query_start.data_ptr(), key_start.data_ptr(),
                   key_count.data_ptr())
    lib = load()
    with _on(dev, stream):
        if out is None:
            out = torch.empty((rows, h, d), dtype=q.dtype, device=dev)
        else:
            _array(out, where, "out", (rows, h, d), q.dtype, dev)
        a.out, a.out_stride, a.out_head_stride = out.data_ptr(), out.stride(0), out.stride(1)
        workspace = _workspace(workspace, lib.jdob_edge_attend_workspace(C.byref(a)), dev, where)
        if workspace is not None:
            a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
        jdob._check(lib.jdob_edge_attend(C.byref(a), _handle(dev, stream)), where)
    return out
