"""The edge operators' sources compiled for the CPU (tests/group_cpu: workgroups of several waves) and run against
the definitions in 64 bits at small sizes, every array ending before a page that may not be touched.  Lanes, and waves
between two barriers, run one after the other, lowest first and highest first, and what is loaded straight to LDS
arrives at once or only when it is waited for: LDS that is read before another lane has written it or its load has been
waited for, or that is written before all have read it, changes a result; a read or write past an array ends the run.
Every run is a process of its own."""

import json
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2504_14611_amd", "edge_csrc")
CLANG = "/opt/rocm/llvm/bin/clang++"

CHILD = r"""
import ctypes as C, json, sys
sys.path.insert(0, __ROOT__)
import torch
from paper_2504_14611_amd import edge
from tests import test_gpu_edge_attend as A, test_gpu_edge_norm as N, test_gpu_edge_project as P
lib, libc = C.CDLL(__SO__), C.CDLL(None, use_errno=True)
libc.mmap.restype, libc.mmap.argtypes = C.c_void_p, [C.c_void_p, C.c_size_t, C.c_int, C.c_int, C.c_int, C.c_long]
libc.mprotect.argtypes = [C.c_void_p, C.c_size_t, C.c_int]
for name in ("project", "attend"):
    getattr(lib, f"jdob_edge_{name}_workspace").restype = C.c_int64
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODES = {torch.bfloat16: edge.EDGE_BF16, torch.float16: edge.EDGE_F16, torch.float32: edge.EDGE_F32}

def guarded(t, shift=0):
    # the tensor's values in pages of their own, `shift` elements from a multiple of 16 bytes, with a page behind
    # the last 16 bytes and one before the first page that may not be touched
    n = t.numel() * t.element_size()
    at = shift * t.element_size()
    room = (n + at + 15) // 16 * 16
    pages = (room + 4095) // 4096 * 4096
    base = libc.mmap(None, pages + 8192, 3, 0x22, -1, 0)
    assert base not in (None, C.c_void_p(-1).value)
    libc.mprotect(base, 4096, 0), libc.mprotect(base + 4096 + pages, 4096, 0)
    if not n:
        return t.clone()
    raw = (C.c_char * n).from_address(base + 4096 + pages - room + at)
    return torch.frombuffer(raw, dtype=t.dtype).view(t.shape).copy_(t)

def ptr(t):
    return None if t is None else t.data_ptr()

def ok(code):
    assert code == 0, code

def norm(c, gen):
    dt, rows, dim = TYPES[c["dtype"]], c["rows"], c["dim"]
    x = torch.randn(rows, dim, generator=gen).to(dt)
    if c.get("size"):
        x[::2] *= c["size"]
    x = guarded(x, c.get("shift", 0))
    r = guarded(torch.randn(rows, dim, generator=gen).mul_(3).to(dt)) if c["residual"] else None
    w = guarded(torch.randn(dim, generator=gen).add_(1).to(dt), c.get("shift", 0))
    got = {"sum": None if r is None else guarded(torch.zeros_like(x)), "out": guarded(torch.zeros_like(x)),
           "q": guarded(torch.zeros_like(x, dtype=torch.int8)), "scale": guarded(torch.zeros(rows))}
    a = edge.NormArgs(rows, dim, CODES[dt], 1e-5, ptr(x), dim, ptr(r), dim, ptr(w), ptr(got["sum"]), dim,
                      ptr(got["out"]), dim, ptr(got["q"]), dim, ptr(got["scale"]))
    ok(lib.jdob_edge_norm(C.byref(a), None))
    N.check(got, x, w, 1e-5, r, c)
    return [t for t in got.values() if t is not None]

def project(c, gen):
    dt, rows, i, o, n, rank, bits8 = TYPES[c["dtype"]], c["rows"], c["i"], c["o"], c["n"], c["rank"], c["bits8"]
    shift = c.get("shift", 0)
    s = {"dtype": dt}
    if bits8:
        s["x"], s["weight"] = (guarded(torch.randn(r, i, generator=gen).mul_(50).round_().clamp_(-127, 127).to(torch.int8), shift)
                               for r in (rows, o))
        s["x_scale"], s["weight_scale"] = (guarded(torch.rand(r, generator=gen) * 0.02) for r in (rows, o))
    else:
        s["x"] = guarded(torch.randn(rows, i, generator=gen).to(dt), shift)
        s["weight"] = guarded((torch.randn(o, i, generator=gen) / i ** 0.5).to(dt), shift)
    a = edge.ProjectArgs(rows, i, o, CODES[dt], bits8, ptr(s["x"]), i, ptr(s.get("x_scale")), ptr(s["weight"]), i,
                         ptr(s.get("weight_scale")))
    if n:
        s["adapters"] = {"down": guarded((torch.randn(n, rank, i, generator=gen) / i ** 0.5).to(dt), shift),
                         "up": guarded(torch.randn(n, o, rank, generator=gen).to(dt), shift),
                         "gain": guarded(torch.rand(n, generator=gen) * 2 - 0.5),
                         "rank": guarded(torch.randint(0, rank + 1, (n,), generator=gen).int())}
        s["adapters"]["rank"][0] = rank
        s["row_adapter"] = guarded(torch.randint(-1, n + 1, (rows,), generator=gen).int())
        d = s["adapters"]
        a.num_adapters, a.max_rank, a.down, a.up, a.gain = n, rank, ptr(d["down"]), ptr(d["up"]), ptr(d["gain"])
        a.rank, a.row_adapter = ptr(d["rank"]), ptr(s["row_adapter"])
        space = guarded(torch.full((lib.jdob_edge_project_workspace(C.byref(a)),), 255, dtype=torch.uint8))
        a.workspace, a.workspace_bytes = ptr(space), space.numel()
    out = guarded(torch.zeros(rows, o, dtype=dt))
    a.out, a.out_stride = ptr(out), o
    ok(lib.jdob_edge_project(C.byref(a), None))
    P.check(s, out, c)
    return [out]

def attend(c, gen):
    dt, new, keys, h, g, d = TYPES[c["dtype"]], c["new"], c["keys"], c["heads"], c["kv_heads"], c["dim"]
    shift = c.get("shift", 0)
    q = guarded(torch.randn(sum(new), h, d, generator=gen).to(dt), shift)
    k, v = (torch.randn(sum(keys) + 1, g, d, generator=gen).to(dt) for _ in range(2))
    starts = [sum(keys[:u]) for u in range(len(keys))]
    k[-1], v[-1] = float("nan"), float("nan")  # behind the last sequence's keys
    if c.get("unseen"):  # the last sequence's last value, which its last row alone sees
        v[-2] = float("inf")
    s = {"q": q, "k": guarded(k, shift), "v": guarded(v, shift),
         "query_start": guarded(torch.tensor([sum(new[:u]) for u in range(len(new) + 1)], dtype=torch.int32)),
         "key_start": guarded(torch.tensor(starts)), "key_count": guarded(torch.tensor(keys, dtype=torch.int32)),
         "max_queries": max(new), "max_keys": max(keys)}
    out = guarded(torch.zeros_like(q))
    a = edge.AttendArgs(len(new), h, g, d, CODES[dt], max(new), max(keys), d ** -0.5, q.shape[0], k.shape[0],
                        ptr(q), h * d, d, ptr(s["k"]), g * d, d, ptr(s["v"]), g * d, d, ptr(s["query_start"]),
                        ptr(s["key_start"]), ptr(s["key_count"]), ptr(out), h * d, d)
    need = lib.jdob_edge_attend_workspace(C.byref(a))
    space = guarded(torch.full((max(need, 1),), 255, dtype=torch.uint8))
    a.workspace, a.workspace_bytes = ptr(space), need
    ok(lib.jdob_edge_attend(C.byref(a), None))
    if c.get("unseen"):
        assert not out[-1].isfinite().any(), c
        out[-1] = 0
        s["v"][-2] = 0
        clean = out.clone()
        ref = attend({**c, "unseen": False}, torch.Generator().manual_seed(c["seed"]))[0]
        assert torch.equal(clean[:-1], ref[:-1]), c
    else:
        A.check(s, c, out)
    return [out]

for c in json.loads(sys.stdin.read()):
    print(c, flush=True)
    first = None
    for descending, late in ((0, 0), (1, 1), (0, 1), (1, 0)):
        lib.group_cpu_mode(descending, late, c.get("tile", 0))
        c["seed"] = c.get("seed", 0)
        got = {"norm": norm, "project": project, "attend": attend}[c["op"]](c, torch.Generator().manual_seed(c["seed"]))
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first)), (c, descending, late)
print("RUN COMPLETE", flush=True)
"""


def for_the_cpu(name, src):
    """The source with what a header cannot define away: address spaces, inline assembly, the launch, and the rule
    that gives small products small tiles (a test names its tiles)."""
    def rep(a, b):
        nonlocal src
        assert src.count(a) == 1, (name, a)
        src = src.replace(a, b)

    src = src.replace("__attribute__((address_space(3)))", "")
    src = re.sub(r'asm volatile\("" : "\+v"\([^;]*;', "(void)0;", src)
    src = src.replace('asm volatile("" ::: "memory");', "(void)0;")
    src = src.replace('asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");', '(void)group_cpu::meet("order", 0);')
    if name == "edge_common.h":
        rep("(unsigned)(uintptr_t)(const  char *)p", "group_cpu::lds_offset(p)")
        src = re.sub(r'asm volatile\("s_mov_b32 m0[^;]*?%1, %2"[^;]*;',
                     "group_cpu::load((const char *)same + offset, __builtin_amdgcn_readfirstlane(to));", src)
        src = re.sub(r'asm volatile\("s_mov_b32 m0[^;]*?%1, off"[^;]*;',
                     "group_cpu::load(from, __builtin_amdgcn_readfirstlane(to));", src)
        src = re.sub(r'asm volatile\("s_waitcnt vmcnt[^;]*;', "group_cpu::wait(N);", src)
        rep("hipLaunchKernel((const void *)kernel, grid, dim3(threads), args, 0, stream) == hipSuccess",
            "group_cpu::run([&] { kernel(params); }, grid, threads)")
    if name == "project.hip":
        rep("if (t64 <= t128 && t64 <= t256) return", "if (group_cpu::g().tile == 64) return")
        rep("if (t128 <= t256) return", "if (group_cpu::g().tile == 128) return")
    assert "asm" not in src, name
    return src


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    """Builds the library once; returns a function that runs a list of cases."""
    tmp = tmp_path_factory.mktemp("group_cpu")
    for f in os.listdir(CSRC):
        (tmp / f.replace(".hip", ".cpp")).write_text(for_the_cpu(f, open(os.path.join(CSRC, f)).read()))
    objs = [str(f) for f in sorted(tmp.glob("*.cpp"))]
    flags = ["-O1", "-std=c++17", "-fPIC", "-ffp-contract=off", "-w", "-I", os.path.join(ROOT, "tests", "group_cpu"),
             "-I", os.path.join(ROOT, "include")]
    procs = [subprocess.Popen([CLANG, *flags, "-c", f, "-o", f + ".o"]) for f in objs]
    assert all([p.wait() == 0 for p in procs])
    so = str(tmp / "libjdob_edge_cpu.so")
    subprocess.run([CLANG, "-shared", "-o", so, *[f + ".o" for f in objs]], check=True)
    code = CHILD.replace("__ROOT__", repr(ROOT)).replace("__SO__", repr(so))

    def go(cases):
        r = subprocess.run([sys.executable, "-c", code], input=json.dumps(cases), capture_output=True, text=True,
                           timeout=600)
        assert r.returncode == 0 and "RUN COMPLETE" in r.stdout, \
            f"exit {r.returncode}\n{r.stdout[-600:]}\n{r.stderr[-3000:]}"
    return go


def test_norm(run):
    run([dict(op="norm", rows=rows, dim=dim, dtype=dtype, residual=residual, shift=shift) for rows, dim in
         ((1, 1), (3, 7), (5, 64), (2, 513), (6, 1000), (2, 4096), (1, 8192), (1, 12345))
         for dtype, residual, shift in (("bf16", True, 0), ("f16", False, 1), ("f32", True, 1))] +
        [dict(op="norm", rows=1025, dim=600, dtype="bf16", residual=True)] +
        [dict(op="norm", rows=3, dim=dim, dtype="f32", residual=False, size=size)
         for dim in (100, 3000, 9000) for size in (1e30, 1e-30)])


def project(rows, i, o, n=0, rank=0, **kw):
    return [dict(op="project", rows=rows, i=i, o=o, n=n, rank=rank, dtype=dtype, bits8=bits8, **kw)
            for dtype, bits8 in (("bf16", 0), ("f16", 0), ("bf16", 1), ("f16", 1))]


@pytest.mark.parametrize("rows", [1, 16, 21, 50])
def test_few_rows(run, rows):
    """W streams past the rows: whole slices for all waves, for some, none; adapters dealt to workgroups."""
    run(sum([project(rows, i, o, n, rank, shift=shift) for i, o, n, rank, shift in
             ((1100, 20, 0, 0, 0), (130, 17, 3, 5, 1), (31, 16, 2, 40, 0), (1048, 33, 5, 16, 1), (640, 5, 4, 70, 0))], []))


@pytest.mark.parametrize("tile", [64, 128, 256])
def test_tiles(run, tile):
    """Fewer slices than buffers and more, low-rank slices behind them, edges in rows and columns."""
    run(sum([project(rows, i, o, n, rank, tile=tile) for rows, i, o, n, rank in
             ((70, 32, 70, 0, 0), (70, 32, 40, 3, 40), (tile + 5, 272, 24, 2, 8), (65, 656, tile + 9, 1, 70))], []))


@pytest.mark.parametrize("rows,sizes", [
    (65, ((31, 70, 0, 0, 0), (331, 30, 3, 40, 1), (129, 70, 25, 7, 1), (400, 40, 20, 40, 0))),
    (150, ((70, 20, 3, 7, 1), (64, 20, 30, 16, 0)))])
def test_tiles_of_rows_at_any_alignment(run, rows, sizes):
    """Slices that come through registers, and the low-rank part output by output (many adapters)."""
    run(sum([project(rows, i, o, n, rank, shift=shift) for i, o, n, rank, shift in sizes], []))


@pytest.mark.parametrize("dim", [8, 64, 80, 128])
def test_attend(run, dim):
    """Few rows and many, keys split and not, sequences without rows or keys, rows that see none; a value that one row
    alone may see."""
    cases = [dict(op="attend", new=new, keys=keys, heads=h, kv_heads=g, dim=dim, dtype=dtype, shift=shift)
             for new, keys, h, g in (([1], [1], 2, 1), ([1, 0, 3], [70, 5, 2], 4, 2), ([1, 1], [1100, 33], 2, 1),
                                     ([40, 3], [70, 0], 4, 1), ([129, 9], [140, 20], 2, 2))
             for dtype, shift in (("bf16", 0), ("f16", 1))]
    run(cases + [dict(c, unseen=True) for c in cases[2:4] + cases[-2:]])
