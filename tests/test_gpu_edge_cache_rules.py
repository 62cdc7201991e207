"""The paged cache's kernels on either side of the rules that choose them: rows by one block a workgroup and by four, keys
that are split over workgroups and not, more workgroups than stand in one row of a grid (2^21)."""

import random

import pytest
import torch

from paper_2504_14611_amd import edge
from tests import edge_cache_model as model, test_gpu_edge_cache as R, test_gpu_edge_paged as P

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("dim,kv_heads,dtype", [(128, 8, BF16), (72, 8, F16), (64, 16, F16), (8, 16, BF16)])
@pytest.mark.parametrize("more", [False, True])
def test_rows(more, dim, kv_heads, dtype, bits8):
    """2048 workgroups of four blocks of 16 (heads to 64: 32) rows, and one block fewer."""
    each = 64 if dim > 64 else 128
    rows = 2048 // kv_heads * each - (0 if more else each) - 5
    r = random.Random(rows)
    at = sorted(r.randrange(rows) for _ in range(6))
    new = [b - a for a, b in zip([0, *at], [*at, rows])]
    keys = [max(0, n + r.randint(-30, 100)) for n in new]
    s = model.inputs(new, keys, 24, kv_heads, dim, dtype, bits8, gone=[(1, 0), (3, 1)])
    R.check(s, *R.rows(rows, kv_heads, dim, dtype), (rows, new, keys))


@pytest.mark.parametrize("bits8", [False, True])
def test_more_workgroups_of_rows_than_stand_in_a_row_of_the_grid(bits8):
    """262,272 rows of 1024 heads, of which the first and the last 20 stand on pages."""
    rows, g, d, page = 262272, 1024, 8, 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, 2, 1, d, generator=gen, device="cuda").to(BF16)
    k, v = (x[:, i].expand(rows, g, d) for i in range(2))
    cache = edge.make_cache(4, page, g, d, bits8=bits8)
    for t in cache.values():
        if t is not None:
            t.zero_()
    table = torch.full((1, rows // page), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[0, 1], table[0, -2], table[0, -1] = 3, 1, 0, 2
    where = (table, torch.tensor([0, rows], dtype=torch.int32, device="cuda"), torch.tensor([rows], dtype=torch.int32, device="cuda"))
    edge.cache_write(k, v, cache, *where)
    ends = torch.cat([torch.arange(32, device="cuda"), torch.arange(rows - 32, rows, device="cuda")])
    held = cache["k"][[3, 1, 0, 2]].transpose(1, 2).reshape(64, g, d)
    want = k[ends]
    if bits8:
        want, scale = model.quantised(want)
        assert torch.equal(cache["k_scale"][[3, 1, 0, 2]].transpose(1, 2).reshape(64, g), scale)
    assert torch.equal(held, want)
    got = edge.cache_read(cache, *where, rows=rows)
    for y, name, x in zip(got, "kv", (k, v)):
        want = x[ends]
        if bits8:
            codes, scale = model.quantised(want)
            want = (codes.double() * scale.double()[..., None]).float().to(BF16)
        assert torch.equal(y[ends], want), name
        assert not y[32:rows - 32].any(), name


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("page", [16, 20])
@pytest.mark.parametrize("n,kv_heads,longest", [(1025, 2, 9000), (1024, 1, 9000), (256, 8, 8192), (255, 8, 8192), (256, 8, 8193),
                                                (20, 2, 512), (20, 2, 513), (128, 1, 3000), (129, 1, 3000)])
def test_one_long_history_among_many_short_ones(n, kv_heads, longest, page, bits8):
    """Either side of where keys are split and of how finely."""
    r = random.Random(n)
    new = [r.choice([0, 1, 1]) for _ in range(n)]
    keys = [r.randint(0, 40) for _ in range(n)]
    new[n // 3], keys[n // 3], new[-1], keys[-1] = 1, longest, 1, 30
    P.check(model.inputs(new, keys, page, kv_heads, 64, BF16, bits8, 2, seed=n), new, keys, (n, kv_heads, longest))


def test_more_workgroups_of_keys_than_stand_in_a_row_of_the_grid():
    """65,535 sequences of 40 key heads, of which a few at either end have a row."""
    n, g = 65535, 40
    new, keys = [0] * n, [0] * n
    for u, m in ((0, 5), (1, 33), (n - 3, 70), (n - 2, 0), (n - 1, 20)):
        new[u], keys[u] = 1, m
    s = model.inputs(new, keys, 16, g, 64, BF16, False, 1)
    P.check(s, new, keys, "many")


def test_more_columns_than_stand_in_a_row_of_the_joins_grid():
    """Hints of 128 rows of 72 heads for 1024 sequences, so that there are 9.4 million columns to join, nearly all unused."""
    n, g, group = 1024, 8, 9
    new, keys = [0] * n, [0] * n
    for u, m in ((0, 300), (500, 9000), (n - 1, 4000)):
        new[u], keys[u] = 2, m
    s = model.inputs(new, keys, 16, g, 8, BF16, False, group)
    P.check(s, new, keys, "join", got=P.call(s, new, keys, max_queries=128, max_keys=9000))
