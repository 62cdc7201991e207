"""The attentions' sources compiled for the CPU as the library compiles them for the GPU, multiply and add fused, and run on
inputs that show what their softmax loses (edge_precision_model)."""

import json
import os
import subprocess
import sys

import pytest

from tests.test_edge_kernels_on_cpu import CHILD as OTHERS, CLANG, CSRC, ROOT, for_the_cpu

CHILD = r"""
import ctypes as C, json, sys
sys.path.insert(0, __ROOT__)
import torch
from paper_2504_14611_amd import edge
from tests import edge_precision_model as model
lib, libc = C.CDLL(__SO__), C.CDLL(None, use_errno=True)
libc.mmap.restype, libc.mmap.argtypes = C.c_void_p, [C.c_void_p, C.c_size_t, C.c_int, C.c_int, C.c_int, C.c_long]
libc.mprotect.argtypes = [C.c_void_p, C.c_size_t, C.c_int]
for name in ("attend", "attend_paged"):
    getattr(lib, f"jdob_edge_{name}_workspace").restype = C.c_int64
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
CODES = {torch.bfloat16: edge.EDGE_BF16, torch.float16: edge.EDGE_F16}
__GUARDED__
def ptr(t):
    return None if t is None else t.data_ptr()

def paged(c, scores, v, v_scale=None):
    dt, new = TYPES[c["dtype"]], c["new"]
    s = model.paged(scores, v, c["base"], new, c["page"], c["kv_heads"], c["group"], dt, c["bits8"], v_scale)
    cache = {n: None if t is None else guarded(t) for n, t in s["cache"].items()}
    pages, g, page, d = cache["k"].shape
    a = edge.Cache(pages, page, g, d, CODES[dt], c["bits8"], ptr(cache["k"]), *cache["k"].stride()[:3], ptr(cache["v"]),
                   *cache["v"].stride()[:3])
    if c["bits8"]:
        a.k_scale, a.k_scale_page_stride, a.k_scale_head_stride, a.k_scale_slot_stride = ptr(cache["k_scale"]), *cache["k_scale"].stride()
        a.v_scale, a.v_scale_page_stride, a.v_scale_head_stride, a.v_scale_slot_stride = ptr(cache["v_scale"]), *cache["v_scale"].stride()
    q, table, start, count = (guarded(s[n]) for n in ("q", "table", "row_start", "key_count"))
    h, m, width = q.shape[1], len(scores), table.shape[1]
    out = guarded(torch.full((new, h, d), 7.0, dtype=dt))
    a = edge.AttendPagedArgs(a, 1, width, ptr(table), width, ptr(start), ptr(count), h, new, m, 1.0, new, ptr(q), h * d, d, ptr(out),
                             h * d, d)
    need = lib.jdob_edge_attend_paged_workspace(C.byref(a))
    space = guarded(torch.full((max(need, 1),), 255, dtype=torch.uint8))
    a.workspace, a.workspace_bytes = ptr(space), need
    assert lib.jdob_edge_attend_paged(C.byref(a), None) == 0
    return out

def packed(c, scores, v):
    dt, new, m = TYPES[c["dtype"]], c["new"], len(scores)
    q, k, v, start, first, count = (guarded(x) for x in model.packed(scores, v, c["base"], new, c["kv_heads"], c["group"], dt))
    (h, d), g = q.shape[1:], k.shape[1]
    out = guarded(torch.full_like(q, 7.0))
    a = edge.AttendArgs(1, h, g, d, CODES[dt], new, m, 1.0, new, m, ptr(q), h * d, d, ptr(k), g * d, d, ptr(v), g * d, d, ptr(start),
                        ptr(first), ptr(count), ptr(out), h * d, d)
    need = lib.jdob_edge_attend_workspace(C.byref(a))
    space = guarded(torch.full((max(need, 1),), 255, dtype=torch.uint8))
    a.workspace, a.workspace_bytes = ptr(space), need
    assert lib.jdob_edge_attend(C.byref(a), None) == 0
    return out

def far(c):
    scores, v = model.far_scores(c["keys"], c["seed"], "cpu")
    return scores, v, None

def rising(c):
    scores, v = model.rising_scores(c["keys"], c["seed"], "cpu")
    return scores, v, None

def small(c):
    scores, v, v_scale = model.small_weights(c["keys"], c["above"], "cpu")
    return (scores, v, v_scale) if c["bits8"] else (scores, v * v_scale[:, None], None)

def huge(c):
    scores, v, v_scale = model.huge_values(c["keys"], c["seed"], "cpu")
    return (scores, v, v_scale) if c["bits8"] else (scores, v * v_scale[:, None], None)

def cancelling(c):
    scores, v, v_scale = model.cancelling_values(c["keys"], c["seed"], TYPES[c["dtype"]], c["bits8"], "cpu")
    return scores, v, v_scale if c["bits8"] else None

for c in json.loads(sys.stdin.read()):
    print(c, flush=True)
    dt = TYPES[c["dtype"]]
    scores, v, v_scale = globals()[c["what"]](c)
    values = v if v_scale is None else v.double() * v_scale.double()[:, None]
    got = packed(c, scores, v) if c["op"] == "attend" else paged(c, scores, v, v_scale)
    over = model.over(got, scores, values, c["new"], dt, c["part"], c.get("reach", 128))
    assert over <= 0, (c, over)
print("RUN COMPLETE", flush=True)
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    """Builds the library once; returns a function that runs a list of cases."""
    if "fma" not in open("/proc/cpuinfo").read():
        pytest.skip("the CPU does not fuse multiply and add")
    tmp = tmp_path_factory.mktemp("precision_cpu")
    for f in ("edge_common.h", "pages.h", "attend.hip", "paged.hip"):
        (tmp / f.replace(".hip", ".cpp")).write_text(for_the_cpu(f, open(os.path.join(CSRC, f)).read()))
    objs = [str(f) for f in sorted(tmp.glob("*.cpp"))]
    flags = ["-O1", "-std=c++17", "-fPIC", "-ffp-contract=fast", "-mfma", "-w", "-I", os.path.join(ROOT, "tests", "group_cpu"),
             "-I", os.path.join(ROOT, "include")]
    procs = [subprocess.Popen([CLANG, *flags, "-c", f, "-o", f + ".o"]) for f in objs]
    assert all([p.wait() == 0 for p in procs])
    so = str(tmp / "libjdob_precision_cpu.so")
    subprocess.run([CLANG, "-shared", "-o", so, *[f + ".o" for f in objs]], check=True)
    guarded = "def guarded" + OTHERS.split("def guarded")[1].split("\ndef ptr")[0]
    code = CHILD.replace("__ROOT__", repr(ROOT)).replace("__SO__", repr(so)).replace("__GUARDED__", guarded)

    def go(cases):
        r = subprocess.run([sys.executable, "-c", code], input=json.dumps(cases), capture_output=True, text=True,
                           timeout=600)
        assert r.returncode == 0 and "RUN COMPLETE" in r.stdout, \
            f"exit {r.returncode}\n{r.stdout[-600:]}\n{r.stderr[-3000:]}"
    return go


BASES = [0, 1 << 12, 1 << 20, 1 << 23, -(1 << 23)]


@pytest.mark.parametrize("base", BASES)
@pytest.mark.parametrize("bits8", [0, 1])
def test_scores_far_from_zero_over_pages(run, base, bits8):
    """Waves whose maxima differ, scores far from zero: weights are those of the differences."""
    run([dict(op="paged", what="far", keys=keys, seed=seed, new=new, page=page, kv_heads=1, group=2, dtype=dtype, bits8=bits8,
              base=base, part=2.0 ** -16)
         for keys, new, page in ((64, 1, 16), (64, 3, 20), (700, 1, 16)) for seed in (0, 1) for dtype in ("bf16", "f16")])


@pytest.mark.parametrize("base", BASES)
def test_scores_far_from_zero(run, base):
    """Packed keys: few rows by two waves that take other keys, many rows whose maximum rises from tile to tile."""
    run([dict(op="attend", what=what, keys=keys, seed=seed, new=new, kv_heads=1, group=2, dtype=dtype, base=base,
              part=2.0 ** -8 if dtype == "bf16" else 2.0 ** -11)
         for what, keys, new, seed in (("far", 64, 1, 0), ("far", 300, 3, 1), ("rising", 200, 2, 0), ("rising", 200, 70, 0),
                                       ("far", 150, 70, 1))
         for dtype in ("bf16", "f16")])


@pytest.mark.parametrize("bits8", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_small_weights(run, dtype, bits8):
    """Weights of e^-5 to e^-60 beside one of 1 whose value is zero."""
    run([dict(op="paged", what="small", keys=keys, above=above, new=new, page=page, kv_heads=1, group=2, dtype=dtype, bits8=bits8,
              base=0, part=2.0 ** -16)
         for keys, new, page in ((500, 1, 16), (90, 3, 20), (700, 1, 16)) for above in (5, 10, 15, 17, 18, 22, 25, 60)])


@pytest.mark.parametrize("bits8", [0, 1])
def test_huge_values(run, bits8):
    """Sums that pass binary32 before they are divided."""
    run([dict(op="paged", what="huge", keys=keys, seed=seed, new=new, page=page, kv_heads=1, group=2, dtype="bf16", bits8=bits8,
              base=0, part=2.0 ** -16)
         for keys, new, page in ((1, 1, 16), (200, 1, 16), (90, 3, 20), (1500, 1, 16)) for seed in (0, 1)])


@pytest.mark.parametrize("bits8", [0, 1])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_weights_keep_16_bits(run, dtype, bits8):
    """Sums of terms that cancel: a weight of one part, 8 or 11 bits, would show."""
    run([dict(op="paged", what="cancelling", keys=keys, seed=seed, new=1, page=page, kv_heads=1, group=2, dtype=dtype, bits8=bits8,
              base=0, part=2.0 ** -16, reach=9)
         for keys, page in ((2, 16), (5, 16), (20, 16), (60, 20), (300, 16)) for seed in range(3)])
