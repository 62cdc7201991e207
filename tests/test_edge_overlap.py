"""Outputs whose rows or heads would share elements are refused before any HIP call (so these run without a GPU), whichever
strides do it together."""

import ctypes as C
import itertools

import pytest

from paper_2504_14611_amd import edge, jdob
from tests.test_edge_abi import attend_args
from tests.test_edge_cache_abi import paged_args, rows_args

INVALID = jdob.JDOB_ERR_INVALID_ARG
D = 64


def overlaps(rows, row, heads, head):
    spots = sorted(r * row + h * head for r, h in itertools.product(range(rows), range(heads)))
    return any(b - a < D for a, b in zip(spots, spots[1:]))


# three rows and two or four heads of 64
STRIDES = [(row, head) for row in (64, 100, 128, 192, 256, 1000) for head in (64, 96, 128, 150, 192, 384, 500)]


@pytest.mark.parametrize("heads", [2, 4])
def test_rows_and_heads_that_share_elements(heads):
    lib, some = edge.load(), 0
    for row, head in STRIDES:
        if not overlaps(3, row, heads, head):
            continue
        some += 1
        cache = {"num_kv_heads": heads, "k_head_stride": 1024, "v_head_stride": 1024, "k_page_stride": 4096, "v_page_stride": 4096,
                 "k_scale_page_stride": 64, "v_scale_page_stride": 64}
        for name in "kv":
            wide = {"k_stride": 1024, "k_head_stride": 64, "v_stride": 1024, "v_head_stride": 64}
            a = rows_args(cache, rows=3, **{**wide, name + "_stride": row, name + "_head_stride": head})
            assert lib.jdob_edge_cache_read(C.byref(a), None) == INVALID, (row, head)
        a = paged_args({**cache, "num_kv_heads": 2}, num_heads=heads, query_rows=3, out_stride=row, out_head_stride=head)
        assert lib.jdob_edge_attend_paged(C.byref(a), None) == INVALID, (row, head)
        a = attend_args(num_heads=heads, num_kv_heads=2, head_dim=D, query_rows=3, out_stride=row, out_head_stride=head)
        assert lib.jdob_edge_attend(C.byref(a), None) == INVALID, (row, head)
    assert some > 5


def test_strides_beyond_any_memory():
    lib, huge = edge.load(), 1 << 61
    a = paged_args(num_heads=4, query_rows=3, out_stride=huge, out_head_stride=huge)
    assert lib.jdob_edge_attend_paged(C.byref(a), None) == INVALID
