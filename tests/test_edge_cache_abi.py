"""The entry points of the paged cache: what include/jdob_edge.h declares is what the binding passes, and arguments that
are refused are refused before any HIP call (so these run without a GPU)."""

import ctypes as C
import os
import re

import pytest
import torch

from paper_2504_14611_amd import edge, jdob

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000  # never dereferenced: every call below is refused, or has nothing to do
INVALID, UNSUPPORTED, OK = jdob.JDOB_ERR_INVALID_ARG, jdob.JDOB_ERR_UNSUPPORTED, jdob.JDOB_OK


def test_header_and_binding_agree():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "jdob_edge.h")).read(), flags=re.S)
    kinds = {C.c_void_p: "pointer", C.c_int32: "int32_t", C.c_int64: "int64_t", C.c_float: "float", edge.Cache: "jdob_edge_cache"}
    for struct, cls in (("cache", edge.Cache), ("cache_rows_args", edge.CacheRowsArgs), ("attend_paged_args", edge.AttendPagedArgs)):
        body = re.search(r"typedef struct \{([^}]*)\}\s*jdob_edge_" + struct + ";", src).group(1)
        fields = []
        for line in body.split(";"):
            if line.strip():
                stars = line.replace("const", "")
                kind = re.match(r"\s*(\w+)", stars).group(1)
                for name in stars.strip()[len(kind):].split(","):
                    fields.append((name.strip().lstrip("* "), "pointer" if "*" in name else kind))
        assert [(n, kinds[t]) for n, t in cls._fields_] == fields
    assert re.search(rf"#define JDOB_EDGE_MAX_PAGE_SIZE {edge.MAX_PAGE_SIZE}\b", src)


@pytest.mark.parametrize("cls,packed", [(edge.CacheRowsArgs, edge._ROWS), (edge.AttendPagedArgs, edge._PAGED)])
def test_what_is_packed_is_the_structure(cls, packed):
    def flat(x):
        for name, kind in x._fields_:
            value = getattr(x, name)
            yield from flat(value) if kind is edge.Cache else (value,)

    numbers = list(range(1, 1 + len(list(flat(cls())))))
    assert packed.size == C.sizeof(cls)
    assert list(flat(cls.from_buffer_copy(packed.pack(*numbers)))) == numbers


def cache(**kw):
    # [40 pages][2 heads][16 slots][64]
    c = edge.Cache(40, 16, 2, 64, edge.EDGE_BF16, 1, FAKE, 2048, 1024, 64, FAKE, 2048, 1024, 64, FAKE, 32, 16, 1, FAKE, 32, 16, 1)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def rows_args(cache_fields=(), **kw):
    a = edge.CacheRowsArgs(cache(**dict(cache_fields)), 3, 10, FAKE, 10, FAKE, FAKE, 20, FAKE, 128, 64, FAKE, 128, 64)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def paged_args(cache_fields=(), **kw):
    a = edge.AttendPagedArgs(cache(**dict(cache_fields)), 3, 1000, FAKE, 1000, FAKE, FAKE, 8, 1, 16000, 0.125, 3, FAKE, 512, 64,
                             FAKE, 512, 64, FAKE, 1 << 30)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def calls():
    lib = edge.load()
    return ((lib.jdob_edge_cache_write, rows_args), (lib.jdob_edge_cache_read, rows_args), (lib.jdob_edge_attend_paged, paged_args))


@pytest.mark.parametrize("fields,code", [
    ({"num_pages": -1}, INVALID), ({"page_size": 0}, INVALID), ({"page_size": 65537}, UNSUPPORTED), ({"num_kv_heads": 0}, INVALID),
    ({"num_kv_heads": 1025}, UNSUPPORTED), ({"head_dim": 0}, INVALID), ({"head_dim": 136}, UNSUPPORTED), ({"head_dim": 60}, UNSUPPORTED),
    ({"dtype": edge.EDGE_F32}, UNSUPPORTED), ({"bits8": 2}, INVALID), ({"k": None}, INVALID), ({"v": None}, INVALID),
    ({"k_scale": None}, INVALID), ({"v_scale": None}, INVALID), ({"k_slot_stride": 63}, INVALID), ({"k_slot_stride": -64}, INVALID),
    ({"k_head_stride": 0}, INVALID), ({"v_head_stride": 1023}, INVALID), ({"v_page_stride": 2047}, INVALID), ({"k_page_stride": 1 << 62}, INVALID),
    ({"k_scale_slot_stride": 0}, INVALID), ({"v_scale_head_stride": 15}, INVALID), ({"v_scale_page_stride": 31}, INVALID),
])
def test_a_cache_is_refused(fields, code):
    for call, args in calls():
        assert call(C.byref(args(fields)), None) == code, call


@pytest.mark.parametrize("fields,code", [
    ({"num_sequences": -1}, INVALID), ({"num_sequences": 65536}, UNSUPPORTED), ({"table_width": -1}, INVALID), ({"table": None}, INVALID),
    ({"table_stride": 9}, INVALID), ({"key_count": None}, INVALID),
])
def test_sequences_are_refused(fields, code):
    for call, args in calls():
        assert call(C.byref(args(**fields)), None) == code, call


@pytest.mark.parametrize("fields,code", [
    ({"rows": -1}, INVALID), ({"rows": (1 << 30) + 1}, UNSUPPORTED), ({"k": None}, INVALID), ({"v": None}, INVALID),
    ({"row_start": None}, INVALID), ({"k_stride": -1}, INVALID), ({"v_head_stride": -64}, INVALID),
])
def test_rows_are_refused(fields, code):
    for call, args in calls()[:2]:
        assert call(C.byref(rows_args(**fields)), None) == code, call


@pytest.mark.parametrize("fields", [{"k_stride": 63}, {"v_stride": 0}, {"k_head_stride": 0}, {"v_head_stride": 32}])
def test_rows_that_would_be_read_into_the_same_elements_are_refused(fields):
    assert edge.load().jdob_edge_cache_read(C.byref(rows_args(**fields)), None) == INVALID


@pytest.mark.parametrize("fields,code", [
    ({"num_heads": 0}, INVALID), ({"num_heads": 7}, INVALID), ({"num_heads": 1026}, UNSUPPORTED), ({"max_queries": -1}, INVALID),
    ({"max_keys": -1}, INVALID), ({"scale": 0.0}, INVALID), ({"scale": float("nan")}, INVALID), ({"scale": float("inf")}, INVALID),
    ({"query_rows": -1}, INVALID), ({"query_rows": (1 << 30) + 1}, UNSUPPORTED), ({"q": None}, INVALID), ({"out": None}, INVALID),
    ({"query_start": None}, INVALID), ({"q_stride": -8}, INVALID), ({"q_head_stride": -8}, INVALID), ({"out_stride": 63}, INVALID),
    ({"out_head_stride": 0}, INVALID), ({"workspace": None}, INVALID), ({"workspace": FAKE + 4}, INVALID), ({"workspace_bytes": 16}, INVALID),
])
def test_attend_paged_is_refused(fields, code):
    assert edge.load().jdob_edge_attend_paged(C.byref(paged_args(**fields)), None) == code


def test_more_workgroups_than_a_grid_takes_are_refused():
    lib = edge.load()
    a = paged_args({"num_kv_heads": 1024, "k_page_stride": 1 << 21, "v_page_stride": 1 << 21, "k_scale_page_stride": 1 << 15,
                    "v_scale_page_stride": 1 << 15}, num_heads=1024, num_sequences=65535, max_queries=1 << 30, query_rows=1 << 30,
                   out_stride=1 << 16, workspace_bytes=(1 << 63) - 1)
    assert lib.jdob_edge_attend_paged(C.byref(a), None) == UNSUPPORTED
    b = rows_args({"num_kv_heads": 1024, "k_page_stride": 1 << 21, "v_page_stride": 1 << 21, "k_scale_page_stride": 1 << 15,
                   "v_scale_page_stride": 1 << 15}, rows=1 << 30, k_stride=1 << 16, v_stride=1 << 16)
    assert lib.jdob_edge_cache_read(C.byref(b), None) == UNSUPPORTED


def test_null_structs_are_refused_and_nothing_to_do_is_ok():
    lib = edge.load()
    for call, args in calls():
        assert call(None, None) == INVALID
        assert call(C.byref(args(num_sequences=0, table=None, key_count=None)), None) == OK
    for fields in ({"rows": 0, "k": None, "v": None, "table": None},):
        assert lib.jdob_edge_cache_write(C.byref(rows_args(**fields)), None) == OK
        assert lib.jdob_edge_cache_read(C.byref(rows_args(**fields)), None) == OK
    for fields in ({"query_rows": 0, "q": None}, {"max_queries": 0, "out": None}):
        assert lib.jdob_edge_attend_paged(C.byref(paged_args(**fields)), None) == OK
    assert lib.jdob_edge_attend_paged_workspace(None) == -1


def test_workspaces_follow_the_sizes():
    size = lambda c=(), **kw: edge.load().jdob_edge_attend_paged_workspace(C.byref(paged_args(c, **kw)))  # noqa: E731
    assert size(num_heads=0) == -1 and size({"dtype": 2}) == -1
    assert size(max_keys=100) == 0 and size(num_sequences=0) == 0 and size(max_queries=0) == 0
    some = size()
    assert some > 0 and some % 16 == 0
    # no more than the table has room for, and no sequence has more rows than there are
    assert size(max_keys=0x7fffffff) == some and size(max_queries=0x7fffffff) == size(max_queries=3)


@pytest.mark.parametrize("bits8", [False, True])
def test_the_binding_refuses(bits8):
    bf, i32 = torch.bfloat16, torch.int32
    c = edge.make_cache(4, 16, 2, 64, bits8=bits8, device="cpu")
    k = torch.zeros(3, 2, 64, dtype=bf)
    where = dict(table=torch.zeros(1, 4, dtype=i32), row_start=torch.zeros(2, dtype=i32), key_count=torch.zeros(1, dtype=i32))
    for bad in ({}, {"k": k[:, :, ::2]}, {"table": where["table"].long()}, {"table": where["table"].t()}, {"key_count": where["row_start"]}):
        with pytest.raises(jdob.JdobError):  # ({}: tensors of the host)
            edge.cache_write(**{"k": k, "v": k, "cache": c, **where, **bad})
    scales = {"k_scale": None} if bits8 else {"k_scale": torch.zeros(4, 2, 16)}
    for bad in (scales, {"k": c["k"].transpose(2, 3)}, {"k": c["k"][0]}, {"v": c["v"].half()}):
        with pytest.raises(jdob.JdobError):
            edge.cache_write(k, k, {**c, **bad}, **where)
        with pytest.raises(jdob.JdobError):
            edge.cache_read({**c, **bad}, rows=3, **where)
        with pytest.raises(jdob.JdobError):
            edge.attend_paged(k, {**c, **bad}, where["table"], where["row_start"], where["key_count"])
    for kw in ({"scale": 0.0}, {"scale": float("nan")}, {"scale": 1e39}, {"max_queries": -1}, {"max_keys": -2}):
        with pytest.raises(jdob.JdobError):
            edge.attend_paged(k, c, where["table"], where["row_start"], where["key_count"], **kw)
    for kw in ({"pages": -1}, {"page_size": 0}, {"page_size": 65537}, {"kv_heads": 0}, {"dim": 12}, {"dim": 136}, {"dtype": torch.float32}):
        with pytest.raises(jdob.JdobError):
            edge.make_cache(**{"pages": 4, "page_size": 16, "kv_heads": 2, "dim": 64, "device": "cpu", **kw})
