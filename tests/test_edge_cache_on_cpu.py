"""The sources of the operators on a paged cache compiled for the CPU (tests/group_cpu) and run against the definitions
in 64 bits at small sizes, as test_edge_kernels_on_cpu does with the others: every array ends before a page that may not
be touched, lanes and waves run in both orders, workspaces and outputs hold rubbish before."""

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
from tests import edge_cache_model as model
lib, libc = C.CDLL(__SO__), C.CDLL(None, use_errno=True)
libc.mmap.restype, libc.mmap.argtypes = C.c_void_p, [C.c_void_p, C.c_size_t, C.c_int, C.c_int, C.c_int, C.c_long]
libc.mprotect.argtypes = [C.c_void_p, C.c_size_t, C.c_int]
lib.jdob_edge_attend_paged_workspace.restype = C.c_int64
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
CODES = {torch.bfloat16: edge.EDGE_BF16, torch.float16: edge.EDGE_F16}
__GUARDED__
def ptr(t):
    return None if t is None else t.data_ptr()

def cache_of(s, c, shift):
    # k and v at the end of their pages; `order`: slots before heads
    kind = {}
    for n, t in s["cache"].items():
        if t is not None:
            t = t.transpose(1, 2).contiguous() if c.get("order") else t
            t = guarded(t, shift if n in ("k", "v") else 0)
            kind[n] = t.transpose(1, 2) if c.get("order") else t
    pages, g, page, d = kind["k"].shape
    a = edge.Cache(pages, page, g, d, CODES[TYPES[c["dtype"]]], c["bits8"], ptr(kind["k"]), *kind["k"].stride()[:3],
                   ptr(kind["v"]), *kind["v"].stride()[:3])
    if c["bits8"]:
        a.k_scale, a.k_scale_page_stride, a.k_scale_head_stride, a.k_scale_slot_stride = ptr(kind["k_scale"]), *kind["k_scale"].stride()
        a.v_scale, a.v_scale_page_stride, a.v_scale_head_stride, a.v_scale_slot_stride = ptr(kind["v_scale"]), *kind["v_scale"].stride()
    return kind, a

def run(c):
    dt, new, keys, g, d, page, shift = TYPES[c["dtype"]], c["new"], c["keys"], c["kv_heads"], c["dim"], c["page"], c.get("shift", 0)
    gone = [tuple(x) for x in c.get("gone", ())]
    s = model.inputs(new, keys, page, g, d, dt, c["bits8"], c.get("group", 1), device="cpu", gone=gone, spare=c.get("spare", 1))
    kind, cache = cache_of(s, c, shift)
    longest = max(keys)
    if c.get("wide"):  # a table and a hint of many keys: 32 columns at once, keys split
        more = torch.full((len(keys), 140000 // page), -1, dtype=torch.int32)
        more[:, :s["table"].shape[1]] = s["table"]
        s["table"], longest = more, 140000
    table, start, count = (guarded(s[n]) for n in ("table", "row_start", "key_count"))
    n, width, rows = len(keys), table.shape[1], sum(new)
    if c["op"] == "attend":
        h = g * c["group"]
        if c.get("unseen"):  # the last sequence's last value, which its last row alone sees
            u, j = n - 1, keys[-1] - 1
            spot = (int(table[u, j // page]), slice(None), j % page)
            if c["bits8"]:
                kind["v_scale"][spot] = float("inf")
            else:
                kind["v"][spot] = float("inf")
        q, out = guarded(s["q"], shift), guarded(torch.full((rows, h, d), 7.0, dtype=dt))
        a = edge.AttendPagedArgs(cache, n, width, ptr(table), width, ptr(start), ptr(count), h, max(new), longest, d ** -0.5, rows,
                                 ptr(q), h * d, d, ptr(out), h * d, d)
        need = lib.jdob_edge_attend_paged_workspace(C.byref(a))
        space = guarded(torch.full((max(need, 1),), 255, dtype=torch.uint8))
        a.workspace, a.workspace_bytes = ptr(space), need
        assert lib.jdob_edge_attend_paged(C.byref(a), None) == 0
        if c.get("unseen"):
            assert not out[-1].isfinite().all(dim=-1).any(), c
            clean = run({**c, "unseen": False})[0]
            assert torch.equal(out[:-1], clean[:-1]), c
            return [out[:-1].clone()]
        want, mass, spread, most = model.attend(q, kind, table.tolist(), start.tolist(), keys, d ** -0.5)
        off = (out.double() - want).abs() - model.attend_bound(want, mass, spread, most, d, max(keys), dt, c["bits8"])
        assert not out.isnan().any() and (off.numel() == 0 or off.max() <= 0), (c, off.max())
        return [out]
    gen = torch.Generator().manual_seed(9)
    k, v = (guarded(torch.randn(rows, g, d, generator=gen).to(dt), shift) for _ in range(2))
    want = {name: t.clone() for name, t in kind.items()}
    stands, belong = model.rows_of(table.tolist(), start.tolist(), keys, page, kind["k"].shape[0])
    if stands:
        row, at, slot = (torch.tensor(x) for x in zip(*stands))
        for name, x in (("k", k), ("v", v)):
            if c["bits8"]:
                want[name][at, :, slot], want[name + "_scale"][at, :, slot] = model.quantised(x[row])
            else:
                want[name][at, :, slot] = x[row]
    a = edge.CacheRowsArgs(cache, n, width, ptr(table), width, ptr(start), ptr(count), rows, ptr(k), g * d, d, ptr(v), g * d, d)
    assert lib.jdob_edge_cache_write(C.byref(a), None) == 0
    for name, t in want.items():
        assert torch.equal(kind[name].contiguous().view(torch.uint8), t.contiguous().view(torch.uint8)), (c, name)
    back = [guarded(torch.full((rows, g, d), 7.0, dtype=dt), shift) for _ in range(2)]
    a.k, a.v = ptr(back[0]), ptr(back[1])
    assert lib.jdob_edge_cache_read(C.byref(a), None) == 0
    for name, got in zip("kv", back):
        x = torch.full((rows, g, d), 7.0, dtype=dt)
        if belong:
            x[torch.tensor([b[0] for b in belong])] = 0
        if stands:
            x[row] = model.values(want, name)[at, :, slot].float().to(dt)
        assert torch.equal(got, x), (c, name)
    return back

for c in json.loads(sys.stdin.read()):
    print(c, flush=True)
    first = None
    for descending in (0, 1):
        lib.group_cpu_mode(descending, 0, 0)
        got = run(c)
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first)), (c, descending)
print("RUN COMPLETE", flush=True)
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    """Builds the library once; returns a function that runs a list of cases."""
    tmp = tmp_path_factory.mktemp("cache_cpu")
    for f in ("edge_common.h", "pages.h", "cache.hip", "paged.hip"):
        (tmp / f.replace(".hip", ".cpp")).write_text(for_the_cpu(f, open(os.path.join(CSRC, f)).read()))
    objs = [str(f) for f in sorted(tmp.glob("*.cpp"))]
    flags = ["-O1", "-std=c++17", "-fPIC", "-ffp-contract=off", "-w", "-I", os.path.join(ROOT, "tests", "group_cpu"),
             "-I", os.path.join(ROOT, "include")]
    procs = [subprocess.Popen([CLANG, *flags, "-c", f, "-o", f + ".o"]) for f in objs]
    assert all([p.wait() == 0 for p in procs])
    so = str(tmp / "libjdob_cache_cpu.so")
    subprocess.run([CLANG, "-shared", "-o", so, *[f + ".o" for f in objs]], check=True)
    guarded = "def guarded" + OTHERS.split("def guarded")[1].split("\ndef ptr")[0]
    code = CHILD.replace("__ROOT__", repr(ROOT)).replace("__SO__", repr(so)).replace("__GUARDED__", guarded)

    def go(cases):
        r = subprocess.run([sys.executable, "-c", code], input=json.dumps(cases), capture_output=True, text=True,
                           timeout=600)
        assert r.returncode == 0 and "RUN COMPLETE" in r.stdout, \
            f"exit {r.returncode}\n{r.stdout[-600:]}\n{r.stderr[-3000:]}"
    return go


KINDS = [("bf16", 0, 0), ("f16", 0, 1), ("bf16", 1, 0), ("f16", 1, 1)]


@pytest.mark.parametrize("kv_heads,dim", [(2, 128), (3, 80), (1, 8)])
def test_rows(run, kv_heads, dim):
    """Rows into pages and back, rows that stand nowhere and that belong to no sequence."""
    run([dict(op="rows", new=new, keys=keys, kv_heads=kv_heads, dim=dim, page=page, dtype=dtype, bits8=bits8, shift=shift,
              order=page == 5, gone=gone)
         for new, keys, gone in (([1], [1], ()), ([3, 0, 5], [3, 9, 40], [(2, 0)]), ([20, 4], [9, 33], [(1, 1)]),
                                 ([0] * 20 + [2] * 3, list(range(23)), ()))
         for page in (16, 5) for dtype, bits8, shift in KINDS])


@pytest.mark.parametrize("dim", [8, 64, 80, 128])
@pytest.mark.parametrize("page", [16, 32, 20, 3])
def test_attend(run, dim, page):
    """Few keys and many, split and not, one tile of columns and more, rows that see none, pages that are not there; a
    value that one row alone may see."""
    cases = [dict(op="attend", new=new, keys=keys, kv_heads=g, group=group, dim=dim, page=page, dtype=dtype, bits8=bits8,
                  shift=shift, order=shift == 0 and group == 3, gone=gone)
             for new, keys, g, group, gone in (([1], [1], 1, 2, ()), ([1, 0, 3], [70, 5, 2], 2, 3, [(0, 0)]),
                                               ([1, 1], [600, 33], 1, 4, [(0, 1), (0, 2)]), ([9, 3], [50, 0], 1, 4, ()))
             for dtype, bits8, shift in KINDS]
    cases += [dict(c, new=[9, 2], keys=[700, 3], kv_heads=1, group=4, gone=[(0, 2)], wide=True) for c in cases[:4]]
    run(cases + [dict(c, unseen=True) for c in cases[:4]] +
        [dict(c, new=[3], keys=[60], kv_heads=2, group=4, gone=(), unseen=True) for c in cases[:4]])
