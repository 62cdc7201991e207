"""The planning half of the co-inference example: the fit of a batch's latency and the problem made of it."""

import numpy as np
import pytest

import oracle
from paper_2504_14611_amd import coinference as co


def test_fit_recovers_a_line_and_stays_non_negative():
    b = [1, 4, 8, 12, 16]
    alpha, beta = co.fit(b, [3e-4 + 2e-5 * x for x in b])
    assert abs(alpha - 3e-4) < 1e-12 and abs(beta - 2e-5) < 1e-13
    assert co.fit([5], [2e-4]) == (2e-4, 0.0)
    alpha, beta = co.fit(b, [1e-3 - 1e-5 * x for x in b])   # falls with the batch: no slope
    assert beta == 0.0 and alpha > 0
    alpha, beta = co.fit([1, 2], [0.0, 1.0])                # a negative intercept
    assert alpha == 0.0 and beta == 1.0


@pytest.mark.parametrize("tokens", [1, 64])
def test_instance_is_a_feasible_problem(tokens):
    shape = co.Shape(blocks=5, width=256, heads=4, kv_heads=2, inner=512, rank=8)
    prob = co.instance(shape, 6, tokens, 1e-4, 1e-5)
    assert prob["cycles"].shape == (1, 5) and prob["bits"].shape == (1, 6) and prob["rate"].shape == (1, 6)
    # 4 multiplications a cycle
    per_row = 256 * ((4 + 2 * 2) * 64 + 256 + 2 * 512)
    assert np.isclose(prob["cycles"][0, 0] * 4, tokens * per_row + tokens * (tokens + 1) * 256)
    assert prob["bits"][0, 0] == tokens * 16 and (prob["bits"][0, 1:] == tokens * 256 * 16).all()
    got = oracle.solve(prob)
    assert got["status"][0] == 0 and np.isfinite(got["energy"][0])


def test_edge_refuses_rows_that_do_not_fit():
    torch = pytest.importorskip("torch")
    shape = co.Shape(blocks=1, width=64, heads=2, kv_heads=1, inner=64, rank=4)
    chain = co.make_chain(shape, 2, device="cpu")
    assert chain[0]["qkv"]["weight"].dtype == torch.int8 and chain[0]["o"]["weight"].dtype == torch.bfloat16
    e = co.Edge(shape, chain, [0, 1], 0, 4, device="cpu")
    with pytest.raises(ValueError):
        e.run(torch.zeros(3, 64).bfloat16(), [3])
    with pytest.raises(ValueError):
        e.run(torch.zeros(3, 64).bfloat16(), [1, 1])
    with pytest.raises(ValueError):
        e.run(torch.zeros(6, 64).bfloat16(), [1, 5])


def test_profile_charges_a_batch_once_for_what_it_does_once(monkeypatch):
    """A batch that takes 5 ms once and (2 + 0.1 b) ms a block: over 10 blocks that is 2.5 ms + 0.1 ms a user a block."""
    torch = pytest.importorskip("torch")
    now = [0.0]

    class Timed:
        def __init__(self, shape, chain, users, first, room, device="cuda"):
            self.blocks, self.users = len(chain[first:]), len(users)

        def run(self, rows, lengths):
            now[0] += 5e-3 + self.blocks * (2e-3 + 1e-4 * self.users)

    monkeypatch.setattr(co, "Edge", Timed)
    monkeypatch.setattr(co.time, "perf_counter", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: None)
    alpha, beta = co.profile(co.Shape(width=64), [{}] * 10, 8, 4, device="cpu")
    assert abs(alpha - 2.5e-3) < 1e-9 and abs(beta - 1e-4) < 1e-10
