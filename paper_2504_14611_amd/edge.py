"""Binding of the edge operators of libjdob.so (include/jdob_edge.h).

What the edge GPU computes for the users that a policy offloads: `norm` (RMS norm of rows with the residual's
addition, in the rows' type or in 8 bits with scales), `project` (the projection that all users share beside each
row's low-rank adapter), `attend` (causal attention of packed sequences of different lengths), and what works on a paged
cache of keys and values (`make_cache`): `cache_write` and `cache_read` (rows into it, quantised to 8 bits where it is of
8 bits, and back) and `attend_paged` (attention of sequences' newest rows over it).

Argument marshalling only, like paper_2504_14611_amd.jdob: the work runs in the HIP kernels of the library, and
there is no fallback.  Tensors are device tensors (others are refused); outputs and workspaces that the caller does
not pass are allocated by torch on the stream that the call runs on.  `stream` is a raw HIP stream handle (default:
torch's current stream of the tensors' device).  The operators are forward only: outputs carry no gradient graph,
also where an input requires gradients.  Refused arguments raise jdob.JdobError with the library's status code.
"""

from __future__ import annotations

import ctypes as C
import struct
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
MAX_PAGE_SIZE = 65536
_MAX_I32 = 0x7fffffff

EXPORTS = ("jdob_edge_norm", "jdob_edge_project", "jdob_edge_project_workspace", "jdob_edge_attend",
           "jdob_edge_attend_workspace", "jdob_edge_cache_write", "jdob_edge_cache_read", "jdob_edge_attend_paged",
           "jdob_edge_attend_paged_workspace")

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


class Cache(C.Structure):
    _fields_ = [("num_pages", _I32), ("page_size", _I32), ("num_kv_heads", _I32), ("head_dim", _I32), ("dtype", _I32),
                ("bits8", _I32), ("k", _P), ("k_page_stride", _I64), ("k_head_stride", _I64), ("k_slot_stride", _I64),
                ("v", _P), ("v_page_stride", _I64), ("v_head_stride", _I64), ("v_slot_stride", _I64), ("k_scale", _P),
                ("k_scale_page_stride", _I64), ("k_scale_head_stride", _I64), ("k_scale_slot_stride", _I64),
                ("v_scale", _P), ("v_scale_page_stride", _I64), ("v_scale_head_stride", _I64),
                ("v_scale_slot_stride", _I64)]


class CacheRowsArgs(C.Structure):
    _fields_ = [("cache", Cache), ("num_sequences", _I32), ("table_width", _I32), ("table", _P), ("table_stride", _I64),
                ("row_start", _P), ("key_count", _P), ("rows", _I32), ("k", _P), ("k_stride", _I64),
                ("k_head_stride", _I64), ("v", _P), ("v_stride", _I64), ("v_head_stride", _I64)]


class AttendPagedArgs(C.Structure):
    _fields_ = [("cache", Cache), ("num_sequences", _I32), ("table_width", _I32), ("table", _P), ("table_stride", _I64),
                ("query_start", _P), ("key_count", _P), ("num_heads", _I32), ("max_queries", _I32), ("max_keys", _I32),
                ("scale", _F32), ("query_rows", _I64), ("q", _P), ("q_stride", _I64), ("q_head_stride", _I64),
                ("out", _P), ("out_stride", _I64), ("out_head_stride", _I64), ("workspace", _P),
                ("workspace_bytes", _I64)]


# The last two as their bytes: packed at once they take a fifth of the time that setting a structure's fields takes, and
# with single tokens a call's time is the host's.
_ROWS, _PAGED = struct.Struct("@6i16q2i4qi6q"), struct.Struct("@6i16q2i4q3if9q")
_NO_SCALES = (0,) * 8

_lib = None


def load():
    """libjdob.so with the edge operators' prototypes; raises OSError if it has not been built."""
    global _lib
    if _lib is None:
        lib = jdob.load()
        for name, args in (("norm", NormArgs), ("project", ProjectArgs), ("attend", AttendArgs),
                           ("cache_write", CacheRowsArgs), ("cache_read", CacheRowsArgs),
                           ("attend_paged", AttendPagedArgs)):
            call = getattr(lib, "jdob_edge_" + name)
            pointer = C.c_void_p if args in (CacheRowsArgs, AttendPagedArgs) else C.POINTER(args)  # (bytes, too)
            call.argtypes, call.restype = [pointer, C.c_void_p], C.c_int
            if args not in (NormArgs, CacheRowsArgs):
                size = getattr(lib, f"jdob_edge_{name}_workspace")
                size.argtypes, size.restype = [pointer], C.c_int64
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


def make_cache(pages: int, page_size: int, kv_heads: int, dim: int, dtype=torch.bfloat16, bits8: bool = False,
               device="cuda") -> Dict[str, object]:
    """A paged cache as the calls below take it: `k` and `v` [pages, kv_heads, page_size, dim] of `dtype`, or with bits8
    of int8 beside `k_scale` and `v_scale` [pages, kv_heads, page_size] (float32).  Nothing is set: keys that were not
    written are never seen.  Any tensors of these shapes will do, views of others among them (only the last dimension of
    k and v has to be contiguous); this order of dimensions reads fastest, and page sizes that are multiples of 16."""
    where = "make_cache"
    if min(pages, page_size, kv_heads, dim) < 0 or not (page_size and kv_heads and dim):
        _refuse(where, f"{pages} pages of {page_size} keys, {kv_heads} heads of {dim}")
    _dtype(dtype, where)
    if page_size > MAX_PAGE_SIZE or pages > _MAX_I32 or kv_heads > 1024 or dim > MAX_HEAD_DIM or dim % 8:
        _refuse(where, f"{pages} pages of {page_size} keys, {kv_heads} heads of {dim}", jdob.JDOB_ERR_UNSUPPORTED)
    shape = (pages, kv_heads, page_size, dim)
    kind = torch.int8 if bits8 else dtype
    cache = {name: torch.empty(shape, dtype=kind, device=device) for name in ("k", "v")}
    for name in ("k_scale", "v_scale"):
        cache[name] = torch.empty(shape[:3], dtype=torch.float32, device=device) if bits8 else None
    return cache


def _differs(t, where: str, name: str, shape, dtype, device):
    if t is None:
        _refuse(where, f"the cache has no {name}")
    _refuse(where, f"the cache's {name} is {tuple(t.shape)} {t.dtype} on {t.device}, "
                   f"expected {tuple(shape)} {dtype} on {device}")


def _cache(cache: dict, where: str, dtype, device, table, row_start, key_count):
    """The cache and the sequences as the first fields of CacheRowsArgs and AttendPagedArgs.  (Of a dimension with one
    entry the library never uses the stride.)"""
    k, v = cache.get("k"), cache.get("v")
    if k is None or v is None:
        _refuse(where, "the cache has no " + ("k" if k is None else "v"))
    shape, kind = k.shape, k.dtype
    if len(shape) != 4:
        _refuse(where, "the cache's k and v are [pages, heads, page size, columns]")
    pages, g, size, d = shape
    bits8 = kind is torch.int8
    if not bits8 and kind is not dtype:
        _refuse(where, f"the cache is {kind}, expected {dtype} or int8")
    if k.device != device:
        _refuse(where, f"the cache is on {k.device}, expected {device}")
    if v.shape != shape or v.dtype is not kind or v.device != device:
        _differs(v, where, "v", shape, kind, device)
    if pages > _MAX_I32 or g > 1024 or size > MAX_PAGE_SIZE or d > MAX_HEAD_DIM or d % 8:
        _refuse(where, f"{pages} pages of {size} keys, {g} heads of {d}", jdob.JDOB_ERR_UNSUPPORTED)
    k_page, k_head, k_slot, k_one = k.stride()
    v_page, v_head, v_slot, v_one = v.stride()
    if k_one != 1 or v_one != 1:
        _refuse(where, "the cache's last dimension is not contiguous")
    ks, vs = cache.get("k_scale"), cache.get("v_scale")
    if bits8:
        some = shape[:3]
        if ks is None or ks.shape != some or ks.dtype is not torch.float32 or ks.device != device:
            _differs(ks, where, "k_scale", some, torch.float32, device)
        if vs is None or vs.shape != some or vs.dtype is not torch.float32 or vs.device != device:
            _differs(vs, where, "v_scale", some, torch.float32, device)
        scales = (ks.data_ptr(), *ks.stride(), vs.data_ptr(), *vs.stride())
    elif ks is None and vs is None:
        scales = _NO_SCALES
    else:
        _refuse(where, "scales belong to an 8-bit cache")
    shape = table.shape
    if len(shape) != 2:
        _refuse(where, "table is [sequences, pages]")
    n, width = shape
    if n > MAX_SEQUENCES or width > _MAX_I32:
        _refuse(where, f"{n} sequences of {width} pages", jdob.JDOB_ERR_UNSUPPORTED)
    pitch, one = table.stride()
    if table.dtype is not torch.int32 or table.device != device or (one != 1 and width > 1):
        _array(table, where, "table", shape, torch.int32, device)
    return (pages, size, g, d, _dtype(dtype, where), bits8, k.data_ptr(), k_page, k_head, k_slot, v.data_ptr(), v_page, v_head,
            v_slot, *scales, n, width, table.data_ptr(), pitch if n > 1 or pitch > width else width,
            _dense(row_start, where, "row_start", (n + 1,), torch.int32, device),
            _dense(key_count, where, "key_count", (n,), torch.int32, device))


def cache_write(k, v, cache: dict, table, row_start, key_count, stream=None) -> None:
    """jdob_edge_cache_write: rows k and v [rows, kv_heads, dim] (any row and head strides) into the cache's pages.
    Sequence u's rows row_start[u] .. row_start[u+1] are the last of its key_count[u] keys; key j stands on page
    table[u][j // page_size], and rows whose entry is no page are left out.  table [n, width] int32, row_start [n + 1]
    int32, key_count [n] int32.  No two rows may go to one slot."""
    where = "jdob_edge_cache_write"
    if k.dim() != 3:
        _refuse(where, "k and v have rows, heads and columns")
    dev = k.device
    a = _rows(cache, where, k.dtype, dev, k, v, table, row_start, key_count)
    handle, context = _enter(dev, stream, where)
    lib = _lib or load()
    if context is not None:
        with context:
            code = lib.jdob_edge_cache_write(a, handle)
    else:
        code = lib.jdob_edge_cache_write(a, handle)
    if code:
        jdob._check(code, where)


def cache_read(cache: dict, table, row_start, key_count, rows: Optional[int] = None, dtype=None,
               into: Optional[dict] = None, stream=None):
    """jdob_edge_cache_read: the reverse of cache_write with the same arguments.  Returns k and v [rows, kv_heads, dim]:
    8-bit rows as the values that they stand for, rounded to `dtype` (default: a 16-bit cache's own, else bfloat16);
    rows whose key is absent are zeros.  `into` holds the caller's own `k` and `v` (rows of no sequence stay as they
    were); else `rows` is how many to allocate, which row_start on the GPU says, too, but not without waiting for it:
    row_start's last entry (further ones stay unset)."""
    where = "jdob_edge_cache_read"
    held = cache.get("k")
    if held is None:
        _refuse(where, "the cache has no k")
    k, v = (into.get("k"), into.get("v")) if into else (None, None)
    if dtype is None:
        dtype = k.dtype if k is not None else torch.bfloat16 if held.dtype is torch.int8 else held.dtype
    dev = held.device
    handle, context = _enter(dev, stream, where)
    if context is not None:
        with context:
            return _cache_read(cache, where, held, dtype, dev, k, v, rows, table, row_start, key_count, handle)
    return _cache_read(cache, where, held, dtype, dev, k, v, rows, table, row_start, key_count, handle)


def _cache_read(cache, where, held, dtype, dev, k, v, rows, table, row_start, key_count, handle):
    if k is None or v is None:
        given = v if k is None else k
        shape = held.shape
        if len(shape) != 4:
            _refuse(where, "the cache's k and v are [pages, heads, page size, columns]")
        if given is not None:
            rows = given.shape[0]
        elif rows is None or rows < 0:
            _refuse(where, f"rows is {rows}, and no buffer is given")
        _dtype(dtype, where)
        shape = (rows, shape[1], shape[3])
        k = torch.empty(shape, dtype=dtype, device=dev) if k is None else k
        v = torch.empty_like(k) if v is None and given is None else torch.empty(shape, dtype=dtype, device=dev) if v is None else v
    if k.dim() != 3 or (rows is not None and k.shape[0] != rows):
        _refuse(where, f"k is {tuple(k.shape)}, expected {rows} rows, heads and columns")
    a = _rows(cache, where, dtype, dev, k, v, table, row_start, key_count)
    code = (_lib or load()).jdob_edge_cache_read(a, handle)
    if code:
        jdob._check(code, where)
    return k, v


def _rows(cache, where, dtype, dev, k, v, table, row_start, key_count):
    rows = k.shape[0]
    if rows > MAX_ROWS:
        _refuse(where, f"{rows} rows", jdob.JDOB_ERR_UNSUPPORTED)
    part = _cache(cache, where, dtype, dev, table, row_start, key_count)
    shape = (rows, part[2], part[3])
    k_row, k_head, _ = k.stride()
    v_at = _array(v, where, "v", shape, dtype, dev)
    v_row, v_head, _ = v.stride()
    return _ROWS.pack(*part, rows, _array(k, where, "k", shape, dtype, dev), k_row, k_head, v_at, v_row, v_head)


def attend_paged(q, cache: dict, table, query_start, key_count, scale: Optional[float] = None,
                 max_queries: Optional[int] = None, max_keys: Optional[int] = None, out=None, workspace=None, stream=None):
    """jdob_edge_attend_paged: causal attention of sequences' newest rows, q [rows, heads, dim] (any row and head
    strides), over a paged cache.  Sequence u's rows query_start[u] .. query_start[u+1] stand at the end of its
    key_count[u] keys; key j stands on page table[u][j // page_size] and is not seen where that is no page.  The rows'
    own keys have been written before (cache_write).  Made for few rows a sequence; many go through cache_read and
    attend.  scale defaults to dim ** -0.5; max_queries and max_keys are at least the largest sequence's (default: all
    rows, all that the table has room for) and worth giving.  Returns out [rows, heads, dim]."""
    where = "jdob_edge_attend_paged"
    if q.dim() != 3:
        _refuse(where, "q has rows, heads and columns")
    shape, dtype, dev = q.shape, q.dtype, q.device
    rows, h, d = shape
    if rows > MAX_ROWS:
        _refuse(where, f"{rows} rows", jdob.JDOB_ERR_UNSUPPORTED)
    part = _cache(cache, where, dtype, dev, table, query_start, key_count)
    if part[3] != d:
        _refuse(where, f"the cache has heads of {part[3]}, expected {d}")
    if h > 1024:
        _refuse(where, f"{h} heads", jdob.JDOB_ERR_UNSUPPORTED)
    most = rows if max_queries is None else max_queries
    longest = part[23] * part[1] if max_keys is None else max_keys
    scale = d ** -0.5 if scale is None else scale
    if most < 0 or longest < 0 or not 0 < scale < 3e38:
        _refuse(where, f"max_queries {most}, max_keys {longest}, scale {scale}")
    q_row, q_head, _ = q.stride()
    part += (h, min(most, _MAX_I32), min(longest, _MAX_I32), scale, rows, _array(q, where, "q", shape, dtype, dev), q_row, q_head)
    handle, context = _enter(dev, stream, where)
    if context is not None:
        with context:
            return _attend_paged(part, where, shape, dtype, dev, out, workspace, handle)
    return _attend_paged(part, where, shape, dtype, dev, out, workspace, handle)


def _attend_paged(part, where, shape, dtype, dev, out, workspace, handle):
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=dev)
        at = out.data_ptr()
    else:
        at = _array(out, where, "out", shape, dtype, dev)
    row, head, _ = out.stride()
    lib = _lib or load()
    a = _PAGED.pack(*part, at, row, head, 0, 0)
    need = lib.jdob_edge_attend_paged_workspace(a)
    if workspace is None and need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    elif workspace is not None and not (workspace.is_contiguous() and workspace.device == dev):
        _refuse(where, "workspace is contiguous, on the tensors' device")
    if workspace is not None:
        a = _PAGED.pack(*part, at, row, head, workspace.data_ptr(), workspace.numel() * workspace.element_size())
    code = lib.jdob_edge_attend_paged(a, handle)
    if code:
        jdob._check(code, where)
    return out
