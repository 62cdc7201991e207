"""Which users of a batch go over the pages as they are and whose rows are read back first, as far as it goes without a GPU."""

import pytest

from paper_2504_14611_amd import coinference as co

SHAPE = co.Shape(blocks=1, width=64, heads=2, kv_heads=1, inner=64, rank=4)


@pytest.fixture(scope="module")
def chain():
    pytest.importorskip("torch")
    return co.make_chain(SHAPE, 5, device="cpu")


def plan(chain, lengths, history, bits8=False):
    e = co.Edge(SHAPE, chain, list(range(len(lengths))), 0, 100, device="cpu", page=16, bits8=bits8)
    return e._plan(lengths, [a + b for a, b in zip(lengths, history)])


def test_each_user_for_itself(chain):
    p = plan(chain, [40, 1, 9, 0, 8], [0, 50, 20, 30, 0])
    assert p["query_start"].tolist() == [0, 40, 41, 50, 50, 58] and p["key_count"].tolist() == [40, 51, 29, 30, 8]
    few, many = p["groups"]
    assert few["few"] and few["rows"].tolist() == [40, *range(50, 58)] and few["query_start"].tolist() == [0, 1, 9]
    assert few["key_count"].tolist() == [51, 8] and (few["most"], few["longest"]) == (8, 51)
    assert (few["table"] == p["table"][[1, 4]]).all() and not few["read"]
    assert many["rows"].tolist() == [*range(40), *range(41, 50)] and many["query_start"].tolist() == [0, 40, 49]
    assert many["key_count"].tolist() == [40, 29] and many["key_start"].tolist() == [0, 40, 69] and many["keys"] == 69
    assert many["read"] and (many["most"], many["longest"]) == (40, 40) and (many["table"] == p["table"][[0, 2]]).all()


def test_a_batch_of_one_kind_goes_as_it_is(chain):
    for lengths, history, bits8, read in (([1, 8], [3, 0], True, False), ([9, 30], [0, 0], False, False),
                                          ([9, 30], [0, 0], True, True), ([9, 30], [1, 0], False, True)):
        p = plan(chain, lengths, history, bits8)
        g, = p["groups"]
        assert g["rows"] is None and g["table"] is p["table"] and g["read"] is read
        assert g["query_start"] is p["query_start"] and g["key_count"] is p["key_count"]
    g, = plan(chain, [0, 20], [30, 0])["groups"]  # an idle user's history is not read
    assert g["rows"] is None and g["key_count"].tolist() == [20] and not g["read"]
    assert plan(chain, [0, 0], [30, 0])["groups"] == []
