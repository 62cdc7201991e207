"""Outputs whose rows and heads lie in any order, as long as none share elements."""

import pytest
import torch

from paper_2504_14611_amd import edge, jdob
from tests import edge_cache_model as model

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


# rows, row stride, heads, head stride of pieces of 64
LAYOUTS = [(3, 128, 2, 64), (3, 64, 4, 192), (3, 128, 2, 192), (3, 256, 4, 64), (2, 320, 3, 128), (1, 0, 4, 64), (1, 64, 2, 70)]


@pytest.mark.parametrize("rows,row,heads,head", LAYOUTS)
def test_any_order(rows, row, heads, head):
    s = model.inputs([rows], [90], 16, heads, 64, BF16, False, 1)
    where = (s["table"], s["row_start"], s["key_count"])
    want = edge.attend_paged(s["q"], s["cache"], *where)
    k, v = edge.cache_read(s["cache"], *where, rows=rows)

    def out():
        return torch.zeros(2000, dtype=BF16, device="cuda").as_strided((rows, heads, 64), (row, head, 1))

    got = edge.attend_paged(s["q"], s["cache"], *where, out=out())
    assert torch.equal(got, want)
    back = edge.cache_read(s["cache"], *where, into={"k": out(), "v": out()})
    assert torch.equal(back[0], k) and torch.equal(back[1], v)
    m = torch.tensor([90], dtype=torch.int32, device="cuda")
    start, first = torch.tensor([0, 90], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    kk, vv = edge.cache_read(s["cache"], s["table"], start, m, rows=90)
    same = edge.attend(s["q"], kk, vv, s["row_start"], first, m)
    assert torch.equal(edge.attend(s["q"], kk, vv, s["row_start"], first, m, out=out()), same)


@pytest.mark.parametrize("rows,row,heads,head", [(3, 64, 2, 64), (3, 128, 2, 128), (3, 128, 2, 160)])
def test_pieces_that_share_elements(rows, row, heads, head):
    s = model.inputs([rows], [90], 16, heads, 64, BF16, False, 1)
    where = (s["table"], s["row_start"], s["key_count"])
    out = torch.zeros(2000, dtype=BF16, device="cuda").as_strided((rows, heads, 64), (row, head, 1))
    with pytest.raises(jdob.JdobError):
        edge.attend_paged(s["q"], s["cache"], *where, out=out)
    with pytest.raises(jdob.JdobError):
        edge.cache_read(s["cache"], *where, into={"k": out, "v": torch.zeros(rows, heads, 64, dtype=BF16, device="cuda")})
    assert (out == 0).all()
