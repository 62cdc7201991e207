"""What a user's rows see on pages is the same alone and beside others: tokens, chunks, prompts and idle users in one batch.

The attention's outputs of one block are compared to the bit: with adapters that add nothing, the rows' queries, keys and
values are integer sums times scales, the same in any batch, and at these sizes neither attention's kernel nor its order of
sums depends on the others."""

import pytest
import torch

from paper_2504_14611_amd import coinference as co

pytestmark = pytest.mark.gpu
SHAPE = co.Shape(blocks=1, width=512, heads=8, kv_heads=2, inner=1024, rank=8)
HISTORY, NEW = (0, 100, 30, 20, 5), (40, 1, 50, 0, 8)


def attended(chain, users, runs, rows, page, bits8):
    """Each user's rows of the last run as they leave the attention."""
    e = co.Edge(SHAPE, chain, users, 0, 200, page=page, bits8=bits8)
    got, attend = [], e._attend_pages
    e._attend_pages = lambda *a: got.append(attend(*a)) or got[-1]
    at = [0] * len(users)
    for lengths in runs:
        e.run(torch.cat([rows[u][i:i + m] for u, i, m in zip(users, at, lengths)]), lengths)
        at = [i + m for i, m in zip(at, lengths)]
    return got[-1].split(list(runs[-1]))


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("page", [16, 24])
def test_alone_and_beside_others(page, bits8):
    chain = co.make_chain(SHAPE, 5)
    chain[0]["qkv"]["adapters"]["gain"].zero_()
    gen = torch.Generator(device="cuda").manual_seed(4)
    rows = [torch.randn(h + n, SHAPE.width, generator=gen, device="cuda").bfloat16() for h, n in zip(HISTORY, NEW)]
    together = attended(chain, list(range(5)), (HISTORY, NEW), rows, page, bits8)
    for u in range(5):
        runs = [(m,) for m in (HISTORY[u], NEW[u]) if m]
        if NEW[u]:
            alone = attended(chain, [u], runs, rows, page, bits8)
            assert torch.equal(together[u], alone[0]), u


@pytest.mark.parametrize("bits8", [False, True])
def test_a_batch_without_rows(bits8):
    chain = co.make_chain(SHAPE, 2)
    e = co.Edge(SHAPE, chain, [0, 1], 0, 40, page=16, bits8=bits8)
    none = torch.empty(0, SHAPE.width, dtype=torch.bfloat16, device="cuda")
    assert e.run(none, [0, 0]).shape == (0, SHAPE.width)
    e.run(torch.randn(21, SHAPE.width, device="cuda").bfloat16(), [20, 1])
    assert e.run(none, [0, 0]).shape == (0, SHAPE.width) and e.count == [20, 1]
