"""The co-inference example on the GPU: what a batch computes is what its users compute alone, a prompt is its tokens
one by one, and a block is its definition.

Rows are bfloat16 (unit roundoff 2^-8, about 2^-9.5 root mean square) and pass through about eight roundings a
block that two ways of computing them may decide differently (the kernels sum in other orders), besides 8-bit codes
at the middle between two; over three blocks the root mean square of their sum is below 2^-9.5 * sqrt(24) * 2 = 0.014,
the factor of two for what one block's differences become in the next.  0.04 leaves a factor of three."""

import pytest
import torch

from paper_2504_14611_amd import coinference as co

pytestmark = pytest.mark.gpu
SHAPE = co.Shape(blocks=3, width=512, heads=8, kv_heads=2, inner=1024, rank=8)


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


@pytest.mark.parametrize("cut", [0, 1, 3])
def test_a_batch_is_its_users(chain, rows, cut):
    users = [3, 0, 4, 1, 2]
    out = co.carry_out(SHAPE, chain, cut, users, rows)
    for u in users:
        alone = co.Edge(SHAPE, chain, [u], 0, 200).run(rows[u], [rows[u].shape[0]])
        assert out[u].shape == rows[u].shape and off(out[u], alone) < 0.04, u


def test_a_prompt_is_its_tokens(chain, rows):
    users = [1, 4]
    e, f = (co.Edge(SHAPE, chain, users, 0, 64) for _ in range(2))
    whole = e.run(torch.cat([rows[1][:30], rows[4][:50]]), [30, 50])
    first = f.run(torch.cat([rows[1][:27], rows[4][:49]]), [27, 49])
    got = [first[:27], first[27:]]
    for at in range(3):  # single tokens, of one user in the end
        m = [1, 1 if at == 0 else 0]
        step = f.run(torch.cat([rows[1][27 + at:28 + at], rows[4][49:49 + m[1]]]), m)
        got[0] = torch.cat([got[0], step[:1]])
        got[1] = torch.cat([got[1], step[1:]])
    assert off(torch.cat(got), whole) < 0.04


def test_a_block_is_its_definition(chain, rows):
    s, block, u = SHAPE, chain[0], 3
    got = co.Edge(s, chain[:1], [u], 0, 130).run(rows[u], [130])

    def norm(h, w):
        y = h * w.double() / torch.sqrt((h * h).mean(dim=1, keepdim=True) + 1e-6)
        step = y.abs().amax(dim=1, keepdim=True) / 127
        return torch.round(y / step) * step

    def project(part, x):
        w = part["weight"].double() * (part["weight_scale"].double()[:, None] if "weight_scale" in part else 1)
        a = {k: v[u].double() for k, v in part["adapters"].items()}
        return x @ w.T + a["gain"] * ((x @ a["down"].T) @ a["up"].T)

    h = rows[u].double()
    qkv = project(block["qkv"], norm(h, block["first"])).view(130, -1, s.head_dim).transpose(0, 1)
    q, k, v = qkv[:8], qkv[8:10].repeat_interleave(4, dim=0), qkv[10:].repeat_interleave(4, dim=0)
    score = q @ k.transpose(1, 2).contiguous() * s.head_dim ** -0.5
    late = torch.ones(130, 130, dtype=torch.bool, device="cuda").triu(1)
    y = torch.softmax(score.masked_fill(late, float("-inf")), dim=2) @ v
    h = h + project(block["o"], y.transpose(0, 1).reshape(130, -1))
    want = h + project(block["down"], torch.nn.functional.gelu(project(block["up"], norm(h, block["second"]))))
    assert off(got, want) < 0.04


def test_the_command(capsys):
    r = co.main(["--users", "6", "--tokens", "48", "--more", "2", "--blocks", "3", "--width", "512", "--heads", "8",
                 "--kv-heads", "2", "--inner", "1024", "--rank", "8"])
    assert r["alpha"] >= 0 and r["beta"] >= 0 and "policy" in capsys.readouterr().out
    for o in r.get("out", {}).values():
        assert torch.isfinite(o).all()


@pytest.mark.parametrize("cut", [0, 1, 3])
def test_further_rows_pass_every_block(chain, rows, cut):
    """Where the chain is cut does not change what comes out of it.  (A further row is the output before it: what two
    ways of computing differ by enters the next pass, so each pass may add its own 0.04.)"""
    users = [2, 0, 4]
    out = co.carry_out(SHAPE, chain, cut, users, rows, 3)
    for u in users:
        e = co.Edge(SHAPE, chain, [u], 0, 80)
        n = rows[u].shape[0]
        want = [e.run(rows[u], [n])]
        for _ in range(3):
            want.append(e.run(want[-1][-1:], [1]))
        assert out[u].shape == (n + 3, SHAPE.width)
        assert off(out[u][:n], want[0]) < 0.04, u
        for k in range(3):
            assert off(out[u][n + k], want[k + 1][0]) < 0.04 * (k + 2), (u, k)
