"""The edge operators' entry points: what include/jdob_edge.h declares is what the library exports and the binding
passes, and arguments that it refuses are refused before any HIP call (so these run without a GPU)."""

import ctypes as C
import os
import re

import pytest
import torch

from paper_2504_14611_amd import edge, jdob

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x1000  # never dereferenced: every call below is refused, or has nothing to do
INVALID, UNSUPPORTED, OK = jdob.JDOB_ERR_INVALID_ARG, jdob.JDOB_ERR_UNSUPPORTED, jdob.JDOB_OK


def header():
    src = open(os.path.join(ROOT, "include", "jdob_edge.h")).read()
    return re.sub(r"/\*.*?\*/", "", src, flags=re.S)


def test_header_binding_and_library_agree():
    src, lib = header(), edge.load()
    assert sorted(set(re.findall(r"\b(jdob_edge_[a-z_]+)\s*\(", src))) == sorted(edge.EXPORTS)
    for name in edge.EXPORTS:
        assert hasattr(lib, name)
    for struct, cls in (("norm", edge.NormArgs), ("project", edge.ProjectArgs), ("attend", edge.AttendArgs)):
        body = re.search(r"typedef struct \{([^}]*)\}\s*jdob_edge_" + struct + "_args;", src).group(1)
        fields = []
        for line in body.split(";"):
            if line.strip():
                stars = line.replace("const", "")
                kind = re.match(r"\s*(\w+)", stars).group(1)
                for name in stars.strip()[len(kind):].split(","):
                    fields.append((name.strip().lstrip("* "), "pointer" if "*" in name else kind))
        kinds = {C.c_void_p: "pointer", C.c_int32: "int32_t", C.c_int64: "int64_t", C.c_float: "float"}
        assert [(n, kinds[t]) for n, t in cls._fields_] == fields
    for name, value in (("MAX_ROWS", edge.MAX_ROWS), ("MAX_NORM_DIM", edge.MAX_NORM_DIM), ("MAX_RANK", edge.MAX_RANK),
                        ("MAX_HEAD_DIM", edge.MAX_HEAD_DIM), ("MAX_SEQUENCES", edge.MAX_SEQUENCES)):
        assert re.search(rf"#define JDOB_EDGE_{name} {value}\b", src), name


def norm_args(**kw):
    a = edge.NormArgs(4, 64, edge.EDGE_BF16, 1e-6, FAKE, 64, FAKE, 64, FAKE, FAKE, 64, FAKE, 64, FAKE, 64, FAKE)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("fields,code", [
    ({"rows": -1}, INVALID), ({"dim": 0}, INVALID), ({"eps": -1e-6}, INVALID), ({"eps": float("nan")}, INVALID),
    ({"eps": float("inf")}, INVALID), ({"dtype": 3}, UNSUPPORTED), ({"dtype": -1}, UNSUPPORTED), ({"rows": (1 << 30) + 1}, UNSUPPORTED),
    ({"dim": 16385, **{k: 20000 for k in ("x_stride", "residual_stride", "sum_stride", "out_stride", "q_stride")}}, UNSUPPORTED),
    ({"x": None}, INVALID), ({"weight": None}, INVALID), ({"out": None, "q": None}, INVALID), ({"scale": None}, INVALID),
    ({"residual": None}, INVALID), ({"x_stride": 63}, INVALID), ({"residual_stride": 1}, INVALID),
    ({"sum_stride": 0}, INVALID), ({"out_stride": -64}, INVALID), ({"q_stride": 63}, INVALID),
])
def test_norm_refuses(fields, code):
    assert edge.load().jdob_edge_norm(C.byref(norm_args(**fields)), None) == code


def project_args(**kw):
    a = edge.ProjectArgs(4, 64, 32, edge.EDGE_F16, 1, FAKE, 64, FAKE, FAKE, 64, FAKE, 2, 8, FAKE, FAKE, FAKE, None,
                         FAKE, FAKE, 32, FAKE, 1 << 20)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("fields,code", [
    ({"rows": -1}, INVALID), ({"in_dim": 0}, INVALID), ({"out_dim": 0}, INVALID), ({"num_adapters": -1}, INVALID),
    ({"max_rank": 0}, INVALID), ({"bits8": 2}, INVALID), ({"dtype": edge.EDGE_F32}, UNSUPPORTED),
    ({"max_rank": 257}, UNSUPPORTED), ({"rows": (1 << 30) + 1}, UNSUPPORTED), ({"out_dim": (1 << 20) + 1}, UNSUPPORTED), ({"in_dim": 131073, "x_stride": 1 << 20, "weight_stride": 1 << 20}, UNSUPPORTED),
    ({"x": None}, INVALID), ({"weight": None}, INVALID), ({"out": None}, INVALID), ({"x_scale": None}, INVALID),
    ({"weight_scale": None}, INVALID), ({"down": None}, INVALID), ({"up": None}, INVALID), ({"gain": None}, INVALID),
    ({"row_adapter": None}, INVALID), ({"workspace": None}, INVALID), ({"workspace": FAKE + 4}, INVALID),
    ({"workspace_bytes": 64}, INVALID), ({"x_stride": 63}, INVALID), ({"weight_stride": 63}, INVALID),
    ({"out_stride": 31}, INVALID),
])
def test_project_refuses(fields, code):
    assert edge.load().jdob_edge_project(C.byref(project_args(**fields)), None) == code


def attend_args(**kw):
    a = edge.AttendArgs(2, 8, 2, 64, edge.EDGE_BF16, 1, 5000, 0.125, 2, 6000, FAKE, 512, 64, FAKE, 128, 64, FAKE, 128,
                        64, FAKE, FAKE, FAKE, FAKE, 512, 64, FAKE, 1 << 30)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("fields,code", [
    ({"num_sequences": -1}, INVALID), ({"num_heads": 0}, INVALID), ({"num_kv_heads": 0}, INVALID),
    ({"num_kv_heads": 3}, INVALID), ({"head_dim": 0}, INVALID), ({"max_queries": -1}, INVALID),
    ({"max_keys": -1}, INVALID), ({"query_rows": -1}, INVALID), ({"key_rows": -1}, INVALID),
    ({"scale": 0.0}, INVALID), ({"scale": -0.1}, INVALID), ({"scale": float("nan")}, INVALID),
    ({"scale": float("inf")}, INVALID), ({"dtype": edge.EDGE_F32}, UNSUPPORTED), ({"head_dim": 136}, UNSUPPORTED),
    ({"head_dim": 60}, UNSUPPORTED), ({"num_sequences": 65536}, UNSUPPORTED), ({"num_heads": 1026}, UNSUPPORTED),
    ({"query_rows": 1 << 31}, UNSUPPORTED), ({"q": None}, INVALID), ({"k": None}, INVALID), ({"v": None}, INVALID),
    ({"out": None}, INVALID), ({"query_start": None}, INVALID), ({"key_start": None}, INVALID),
    ({"key_count": None}, INVALID), ({"workspace": None}, INVALID), ({"workspace_bytes": 16}, INVALID),
    ({"q_stride": -1}, INVALID), ({"k_head_stride": -64}, INVALID), ({"v_stride": -2}, INVALID),
    ({"out_stride": -8}, INVALID),
])
def test_attend_refuses(fields, code):
    assert edge.load().jdob_edge_attend(C.byref(attend_args(**fields)), None) == code


def test_null_structs_are_refused():
    lib = edge.load()
    for name in ("norm", "project", "attend"):
        assert getattr(lib, "jdob_edge_" + name)(None, None) == INVALID
    assert lib.jdob_edge_project_workspace(None) == -1 and lib.jdob_edge_attend_workspace(None) == -1


def test_workspaces_follow_the_sizes():
    lib = edge.load()
    assert lib.jdob_edge_project_workspace(C.byref(project_args(num_adapters=0, max_rank=0))) == 0
    assert lib.jdob_edge_project_workspace(C.byref(project_args(rows=0))) == 0
    assert lib.jdob_edge_project_workspace(C.byref(project_args())) > 0
    assert lib.jdob_edge_project_workspace(C.byref(project_args(in_dim=-1))) == -1
    assert lib.jdob_edge_attend_workspace(C.byref(attend_args())) > 0
    assert lib.jdob_edge_attend_workspace(C.byref(attend_args(max_keys=10))) == 0
    assert lib.jdob_edge_attend_workspace(C.byref(attend_args(dtype=9))) == -1


def test_nothing_to_do_launches_nothing():
    """No rows, no sequences: every array pointer may be NULL; the rest is still checked."""
    lib = edge.load()
    assert lib.jdob_edge_norm(C.byref(edge.NormArgs(rows=0, dim=8, eps=0.1)), None) == OK
    assert lib.jdob_edge_norm(C.byref(edge.NormArgs(rows=0, dim=0)), None) == INVALID
    assert lib.jdob_edge_project(C.byref(edge.ProjectArgs(rows=0, in_dim=8, out_dim=8)), None) == OK
    assert lib.jdob_edge_project(C.byref(edge.ProjectArgs(rows=0, in_dim=8, out_dim=8, dtype=2)), None) == UNSUPPORTED
    for kw in ({"num_sequences": 0}, {"query_rows": 0}, {"max_queries": 0}):
        a = edge.AttendArgs(2, 8, 2, 64, 0, 1, 10, 0.1, 2, 10)
        for k, v in kw.items():
            setattr(a, k, v)
        assert lib.jdob_edge_attend(C.byref(a), None) == OK


def refused(code, call, *args, **kw):
    with pytest.raises(jdob.JdobError) as e:
        call(*args, **kw)
    assert e.value.code == code, e.value
    return str(e.value)


def test_binding_refuses_tensors_that_do_not_fit():
    x, w = torch.zeros(3, 8, dtype=torch.bfloat16), torch.zeros(8, dtype=torch.bfloat16)
    assert "weight" in refused(INVALID, edge.norm, x, w[:7])
    refused(INVALID, edge.norm, x, w.float())
    refused(INVALID, edge.norm, x[0], w)
    refused(INVALID, edge.norm, x, w, residual=x[:2])
    refused(INVALID, edge.norm, x.T.contiguous().T, w)
    refused(INVALID, edge.norm, x, w, into={"out": x.float()})
    refused(INVALID, edge.norm, x, w, out16=False)
    refused(UNSUPPORTED, edge.norm, x.double(), w.double())
    refused(INVALID, edge.norm, x, w, eps=-1.0)
    m = torch.zeros(5, 8, dtype=torch.bfloat16)
    ones = torch.ones(5)
    refused(INVALID, edge.project, x, m[:, :7])
    refused(INVALID, edge.project, x, m.half())
    refused(INVALID, edge.project, x, m, x_scale=ones[:3])
    refused(INVALID, edge.project, x, m, x_scale=ones[:3], weight_scale=ones)
    refused(INVALID, edge.project, x.to(torch.int8), m.to(torch.int8))
    refused(INVALID, edge.project, x.to(torch.int8), m.to(torch.int8), x_scale=ones, weight_scale=ones)
    refused(UNSUPPORTED, edge.project, x.float(), m.float())
    a = {"down": torch.zeros(2, 4, 8, dtype=torch.bfloat16), "up": torch.zeros(2, 5, 4, dtype=torch.bfloat16),
         "gain": torch.ones(2)}
    ids = torch.zeros(3, dtype=torch.int32)
    refused(INVALID, edge.project, x, m, adapters=a)
    refused(INVALID, edge.project, x, m, adapters=a, row_adapter=ids.long())
    refused(INVALID, edge.project, x, m, adapters={**a, "up": a["up"][:, :4]}, row_adapter=ids)
    refused(INVALID, edge.project, x, m, adapters={**a, "down": a["down"].half()}, row_adapter=ids)
    refused(INVALID, edge.project, x, m, adapters={**a, "rank": ids}, row_adapter=ids)
    refused(INVALID, edge.project, x, m, out=torch.zeros(3, 4, dtype=torch.bfloat16))
    q, k = torch.zeros(3, 4, 16, dtype=torch.float16), torch.zeros(9, 2, 16, dtype=torch.float16)
    at, first, count = (torch.tensor(v, dtype=t) for v, t in (([0, 3], torch.int32), ([0], torch.int64), ([9], torch.int32)))
    refused(INVALID, edge.attend, q, k, k[:8], at, first, count)
    refused(INVALID, edge.attend, q, k.bfloat16(), k, at, first, count)
    refused(INVALID, edge.attend, q, k, k, at.long(), first, count)
    refused(INVALID, edge.attend, q, k, k, at[:1], first, count)
    refused(INVALID, edge.attend, q, k, k, at, first.int(), count)
    refused(INVALID, edge.attend, q[:, :3], k, k, at, first, count)
    refused(INVALID, edge.attend, q, k, k, at, first, count, scale=-1.0)
    refused(UNSUPPORTED, edge.attend, q.float(), k.float(), k.float(), at, first, count)
    refused(UNSUPPORTED, edge.attend, q[:, :, :12], k[:, :, :12], k[:, :, :12], at, first, count)


def test_binding_refuses_tensors_on_the_host():
    """Tensors that fit but for where they are: a kernel would be given the host's memory."""
    x, w, m = (torch.zeros(s, dtype=torch.bfloat16) for s in ((3, 8), (8,), (5, 8)))
    assert "cpu" in refused(INVALID, edge.norm, x, w)
    refused(INVALID, edge.norm, x, w, residual=x, bits8=True, into={"sum": x}, stream=0)
    refused(INVALID, edge.norm, x[:0], w)
    a = {"down": torch.zeros(2, 4, 8, dtype=torch.bfloat16), "up": torch.zeros(2, 5, 4, dtype=torch.bfloat16),
         "gain": torch.ones(2)}
    assert "cpu" in refused(INVALID, edge.project, x, m)
    refused(INVALID, edge.project, x, m, adapters=a, row_adapter=torch.zeros(3, dtype=torch.int32), stream=0)
    q, k = torch.zeros(3, 4, 16, dtype=torch.float16), torch.zeros(9, 2, 16, dtype=torch.float16)
    at, first, count = (torch.tensor(v, dtype=t) for v, t in (([0, 3], torch.int32), ([0], torch.int64), ([9], torch.int32)))
    assert "cpu" in refused(INVALID, edge.attend, q, k, k, at, first, count)
    refused(INVALID, edge.attend, *(t.to("meta") for t in (q, k, k, at, first, count)))


def test_binding_refuses_sizes_that_32_bits_would_cut():
    """Shapes and hints whose low 32 bits are small numbers are not taken for those."""
    def t(*shape, dtype=torch.bfloat16):
        return torch.empty(*shape, dtype=dtype, device="meta")
    big = 1 << 32
    refused(UNSUPPORTED, edge.norm, t(1, big + 8), t(8))
    refused(UNSUPPORTED, edge.norm, t(big + 1, 8), t(8))
    refused(UNSUPPORTED, edge.project, t(1, big + 8), t(5, big + 8))
    refused(UNSUPPORTED, edge.project, t(1, 8), t(big + 5, 8))
    for down, up, gain in ((t(2, big + 4, 8), t(2, 5, big + 4), t(2, dtype=torch.float32)),
                           (t(big + 2, 4, 8), t(big + 2, 5, 4), t(big + 2, dtype=torch.float32))):
        refused(UNSUPPORTED, edge.project, t(1, 8), t(5, 8), adapters={"down": down, "up": up, "gain": gain},
                row_adapter=t(1, dtype=torch.int32))
    q, k, at = t(3, 4, 16), t(9, 2, 16), t(2, dtype=torch.int32)
    first, count = t(1, dtype=torch.int64), t(1, dtype=torch.int32)
    refused(UNSUPPORTED, edge.attend, q, k, k, t(big + 2, dtype=torch.int32), t(big + 1, dtype=torch.int64), t(big + 1, dtype=torch.int32))
    assert "max_" in refused(INVALID, edge.attend, q, k, k, at, first, count, max_queries=1 - big)
    assert "max_" in refused(INVALID, edge.attend, q, k, k, at, first, count, max_keys=1 - big)


@pytest.mark.parametrize("fields,code", [
    ({"out_stride": 0}, INVALID), ({"out_stride": 63}, INVALID), ({"out_head_stride": 0}, INVALID),
    ({"out_head_stride": 56}, INVALID),
])
def test_attend_refuses_outputs_whose_rows_or_heads_overlap(fields, code):
    assert edge.load().jdob_edge_attend(C.byref(attend_args(**fields)), None) == code


def test_the_longest_key_hints_split_the_keys():
    """Hints up to the largest a call can give: the workspace grows with the splits, to as many as there are at most."""
    lib = edge.load()
    sizes = [lib.jdob_edge_attend_workspace(C.byref(attend_args(num_sequences=1, max_keys=n)))
             for n in (100000, 1 << 28, (1 << 31) - 257, (1 << 31) - 255, (1 << 31) - 1)]
    assert 0 < sizes[0] <= sizes[1] and len(set(sizes[1:])) == 1


def test_grids_that_no_launch_takes_are_refused_before_anything_is_launched():
    lib = edge.load()
    a = project_args(rows=1 << 30, out_dim=1 << 20, out_stride=1 << 20, workspace_bytes=1 << 40)
    assert lib.jdob_edge_project(C.byref(a), None) == UNSUPPORTED and lib.jdob_edge_project_workspace(C.byref(a)) == -1
    a = attend_args(num_heads=1024, num_kv_heads=1024, query_rows=1 << 30, max_queries=1 << 30)
    assert lib.jdob_edge_attend(C.byref(a), None) == UNSUPPORTED
