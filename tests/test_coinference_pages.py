"""The paged cache of the co-inference example as far as it goes without a GPU: who takes which pages, and what is refused."""

import pytest

from paper_2504_14611_amd import coinference as co

SHAPE = co.Shape(blocks=2, width=64, heads=2, kv_heads=1, inner=64, rank=4)


@pytest.fixture(scope="module")
def chain():
    pytest.importorskip("torch")
    return co.make_chain(SHAPE, 2, device="cpu")


def test_users_take_pages_as_they_grow(chain):
    e = co.Edge(SHAPE, chain, [0, 1], 0, 40, device="cpu", page=16, bits8=True, pages=4)
    assert e.cache[0]["k"].shape == (4, 1, 16, 32) and e.cache[1]["k_scale"].shape == (4, 1, 16)
    table = e._take_pages([3, 17])
    assert table.shape == (2, 2) and (table >= 0).sum() == 3 and table[0, 1] == -1
    again = e._take_pages([16, 18])
    assert (again == table).all()
    assert (e._take_pages([17, 18]) >= 0).all()
    held = [list(h) for h in e.held]
    with pytest.raises(ValueError):
        e._take_pages([17, 33])
    assert e.held == held and not e.free


def test_refusals(chain):
    import torch
    with pytest.raises(ValueError):
        co.Edge(SHAPE, chain, [0], 0, 40, device="cpu", bits8=True)
    with pytest.raises(ValueError):
        co.Edge(SHAPE, chain, [0], 0, 40, device="cpu", pages=3)
    e = co.Edge(SHAPE, chain, [0], 0, 4, device="cpu", page=16)
    with pytest.raises(ValueError):
        e.run(torch.zeros(5, 64).bfloat16(), [5])
