"""The co-inference example with the edge's keys and values on pages: what it computes is what it computes with slabs.

Of 16 bits the pages hold what slabs hold, and the attention differs in the order of its sums: the bound of
test_gpu_coinference (0.04) holds.  In 8 bits a key or value is off by up to half of 1/127 of its row's largest; with
128 or fewer nearly normal elements that is about 3 / 127 / sqrt(12) = 0.007 of its root mean square.  Scores are sums of
head_dim such products over sqrt(head_dim): off by 0.007, and p with them; values as much again: 0.01 a block at most,
over three blocks 0.01 * sqrt(3) * 2 = 0.035, the factor of two for what one block's differences become in the next, to be
added to the others."""

import pytest
import torch

from paper_2504_14611_amd import coinference as co

pytestmark = pytest.mark.gpu
SHAPE = co.Shape(blocks=3, width=512, heads=8, kv_heads=2, inner=1024, rank=8)
BOUND = {False: 0.04, True: 0.075}


def off(a, b):
    return ((a.double() - b.double()).norm() / b.double().norm()).item()


@pytest.fixture(scope="module")
def chain():
    return co.make_chain(SHAPE, 5)


@pytest.fixture(scope="module")
def rows():
    gen = torch.Generator(device="cuda").manual_seed(2)
    return {u: torch.randn(n, SHAPE.width, generator=gen, device="cuda").bfloat16()
            for u, n in enumerate((1, 40, 7, 130, 64))}


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("page", [16, 24])
def test_pages_are_slabs(chain, rows, page, bits8):
    """Prompts, chunks after a history, a few rows, single rows of some users, in one batch."""
    users = [3, 1, 4, 2]
    room = 140
    slabs = co.Edge(SHAPE, chain, users, 0, room)
    pages = co.Edge(SHAPE, chain, users, 0, room, page=page, bits8=bits8, pages=27 if page == 16 else 18)
    at = [0] * 4
    for lengths in ((100, 20, 0, 3), (20, 11, 50, 1), (1, 1, 1, 1), (5, 0, 8, 1), (1, 1, 1, 0), (3, 7, 2, 1)):
        x = torch.cat([rows[u][i:i + m] for u, i, m in zip(users, at, lengths)])
        at = [i + m for i, m in zip(at, lengths)]
        assert off(pages.run(x, lengths), slabs.run(x, lengths)) < BOUND[bits8], lengths
    taken = [p for held in pages.held for p in held]
    assert [len(h) for h in pages.held] == [-(-n // page) for n in at] and len(set(taken)) == len(taken)


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("cut", [0, 2])
def test_a_policy_on_pages(chain, rows, cut, bits8):
    users = [2, 0, 4]
    out = co.carry_out(SHAPE, chain, cut, users, rows, 2, page=16, bits8=bits8)
    for u in users:
        e = co.Edge(SHAPE, chain, [u], 0, 80)
        want = [e.run(rows[u], [rows[u].shape[0]])]
        for _ in range(2):
            want.append(e.run(want[-1][-1:], [1]))
        assert off(out[u][:-2], want[0]) < BOUND[bits8]
        for k in range(2):
            assert off(out[u][k - 2], want[k + 1][0]) < BOUND[bits8] * (k + 2), (u, k)


def test_the_command(capsys):
    r = co.main(["--users", "6", "--tokens", "48", "--more", "2", "--blocks", "3", "--width", "512", "--heads", "8",
                 "--kv-heads", "2", "--inner", "1024", "--rank", "8", "--page", "16", "--cache-bits", "8"])
    assert "policy" in capsys.readouterr().out
    for o in r.get("out", {}).values():
        assert torch.isfinite(o).all()
