"""Every kernel that jdob_edge_project chooses from, against the definition in 64 bits: sizes that reach each tile, for
either type, in 16 and 8 bits, without adapters and with one or more slabs of 32 ranks."""

import pytest
import torch

from tests.test_gpu_edge_project import BF16, F16, check, inputs

# name, rows, columns, adapters (0: with and without)
SIZES = [("stream 16", 9, 100, 0), ("stream 32", 20, 100, 0), ("stream 64", 50, 100, 0), ("64", 300, 257, 0),
         ("128", 2000, 2050, 0), ("256", 2055, 4100, 0), ("64 row by row", 128, 200, 20)]
# inner dimensions: whole 16 bytes with a partial slice at the end, or one partial slice; rows at any alignment
DIRECT, ANY = (336, 32), (331, 31)
RANKS = (7, 24, 40, 70)


def variant(rows, in_dim, out_dim, adapters, bits8):
    """The rule of project.hip for contiguous x and W: the kernel's name, and whether memory goes to LDS directly."""
    if rows <= 64:
        return f"stream {16 if rows <= 16 else 32 if rows <= 32 else 64}", False
    direct = in_dim * (1 if bits8 else 2) % 16 == 0
    if rows <= 512 and adapters * 8 >= rows:
        return "64 row by row", direct
    if not direct:
        return "128", False

    def rounds(side, at_once):
        return -(-(-(-rows // side) * -(-out_dim // side)) // at_once)
    cost = {"64": 0.47 * rounds(64, 512), "128": (1.4 if bits8 else 1.1) * rounds(128, 512), "256": 1.86 * rounds(256, 256)}
    return min(cost, key=cost.get), True


def cases():
    for name, rows, out_dim, adapters in SIZES:
        for in_dim in (*DIRECT, *(ANY if name in ("128", "64 row by row") or rows <= 64 else ())):
            for n in ((0, 6) if adapters == 0 else (adapters,)):
                for rank in (RANKS if n else (0,)):
                    yield name, rows, in_dim, out_dim, n, rank


def test_the_sizes_reach_every_kernel():
    for bits8 in (False, True):
        reached = {variant(rows, in_dim, out_dim, n, bits8) for _, rows, in_dim, out_dim, n, _ in cases()}
        assert reached >= {("stream 16", False), ("stream 32", False), ("stream 64", False), ("64", True), ("128", True),
                           ("256", True), ("64 row by row", True), ("128", False), ("64 row by row", False)}
        for name, rows, in_dim, out_dim, n, _ in cases():
            if in_dim in DIRECT:
                assert variant(rows, in_dim, out_dim, n, bits8)[0] == name


@pytest.mark.gpu
@pytest.mark.parametrize("bits8", [False, True], ids=["16", "8"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("name,rows,in_dim,out_dim,n,rank", list(cases()))
def test_project_variants(name, rows, in_dim, out_dim, n, rank, dtype, bits8):
    s = inputs(rows, in_dim, out_dim, dtype, bits8, n, rank, seed=rows + in_dim + rank)
    check(s, label=name)
    if n:  # rows in any order, an adapter of every rank
        gen = torch.Generator(device="cuda").manual_seed(rank)
        s["row_adapter"] = torch.randint(-1, n + 1, (rows,), generator=gen, device="cuda").int()
        s["adapters"]["rank"] = torch.arange(n, device="cuda", dtype=torch.int32) * rank // (n - 1)
        for a, r in enumerate(s["adapters"]["rank"].tolist()):
            s["adapters"]["down"][a, r:] = float("nan")
            s["adapters"]["up"][a, :, r:] = float("nan")
        check(s, label=name)
