"""jdob_edge_project against its definition in 64 bits."""

import math

import pytest
import torch

from paper_2504_14611_amd import edge
from tests import edge_model as model

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def inputs(rows, i, o, dtype, bits8, n=0, rank=0, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")
    s = {"dtype": dtype}
    if bits8:
        s["x"], s["weight"] = (normal(r, i).mul_(50).round_().clamp_(-127, 127).to(torch.int8) for r in (rows, o))
        s["x_scale"], s["weight_scale"] = (torch.rand(r, generator=gen, device="cuda") * 0.02 for r in (rows, o))
    else:
        s["x"], s["weight"] = normal(rows, i).to(dtype), (normal(o, i) / math.sqrt(i)).to(dtype)
    if n:
        s["adapters"] = {"down": (normal(n, rank, i) / math.sqrt(i)).to(dtype), "up": normal(n, o, rank).to(dtype),
                         "gain": torch.rand(n, generator=gen, device="cuda") * 2 - 0.5}
        # rows of one adapter stand together, -1 and n stand for none
        s["row_adapter"] = torch.sort(torch.randint(-1, n + 1, (rows,), generator=gen, device="cuda"))[0].int()
    return s


def check(s, got=None, label=None):
    got = edge.project(**s) if got is None else got
    ref = {k: v for k, v in s.items() if k in ("x", "weight", "x_scale", "weight_scale", "adapters", "row_adapter")}
    y, shared, low = model.project(**ref)
    rank = s["adapters"]["down"].shape[1] if s.get("adapters") else 0
    off = (got.double() - y).abs() - model.project_bound(y, shared, low, s["x"].shape[1], rank, s["dtype"])
    assert got.dtype == s["dtype"] and off.max() <= 0, (label, off.max(), (off > 0).sum())
    return got


SIZES = [(1, 1, 1), (1, 64, 64), (1, 4096, 1000), (2, 7, 3), (16, 128, 48), (17, 200, 130), (33, 1000, 257),
         (64, 513, 64), (65, 264, 300), (128, 2048, 512), (200, 96, 1111), (300, 1031, 129), (513, 320, 640)]


@pytest.mark.parametrize("bits8", [False, True], ids=["16", "8"])
@pytest.mark.parametrize("dtype", [BF16, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("rows,i,o", SIZES)
def test_project(rows, i, o, dtype, bits8):
    check(inputs(rows, i, o, dtype, bits8, seed=rows + i + o))


@pytest.mark.parametrize("n,rank", [(1, 1), (3, 8), (7, 16), (5, 20), (40, 33), (4, 64), (2, 100), (2, 256)])
@pytest.mark.parametrize("rows,i,o,dtype,bits8", [(1, 64, 70, BF16, False), (31, 500, 130, F16, False),
                                                  (64, 1024, 256, BF16, True), (100, 136, 257, BF16, False),
                                                  (333, 1000, 200, F16, True), (700, 512, 384, BF16, False)])
def test_project_with_adapters(rows, i, o, dtype, bits8, n, rank):
    check(inputs(rows, i, o, dtype, bits8, n, rank, seed=rows + n + rank))


def test_large_tiles():
    """Enough rows and columns for the largest tiles, with ragged edges in both."""
    for dtype, bits8 in ((BF16, False), (F16, True)):
        check(inputs(2055, 328, 4100, dtype, bits8, 6, 24))


@pytest.mark.parametrize("rows", [5, 90, 600])
def test_rows_in_any_order_and_ranks_of_their_own(rows):
    s = inputs(rows, 256, 192, BF16, False, 9, 40, seed=rows)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    s["row_adapter"] = torch.randint(-2, 11, (rows,), generator=gen, device="cuda").int()
    s["adapters"]["rank"] = torch.tensor([0, 1, 8, 15, 16, 17, 33, 40, 99], dtype=torch.int32, device="cuda")
    # what lies behind an adapter's rank is not used
    for a, r in enumerate(s["adapters"]["rank"].tolist()):
        s["adapters"]["down"][a, r:] = float("nan")
        s["adapters"]["up"][a, :, r:] = float("nan")
    check(s)


def test_adapters_do_not_touch_other_rows():
    """An adapter that holds NaN or infinities reaches its own rows only."""
    for rows in (6, 150):
        s = inputs(rows, 128, 96, F16, False, 3, 16)
        s["row_adapter"] = (torch.arange(rows, device="cuda") % 4).int()  # 3: none
        clean = check(s)
        s["adapters"]["down"][1, 3, 5], s["adapters"]["up"][2, 7, 0] = float("inf"), float("nan")
        got = edge.project(**s)
        keep = (s["row_adapter"] == 0) | (s["row_adapter"] == 3)
        assert torch.equal(got[keep], clean[keep])
        assert got[s["row_adapter"] == 2][:, 7].isnan().all() and not got[s["row_adapter"] == 2][:, 8].isnan().any()


@pytest.mark.parametrize("shift", [0, 1, 4])
def test_strides_and_offsets(shift):
    for rows, bits8 in ((20, False), (300, False), (20, True), (300, True)):
        s = inputs(rows, 512, 320, BF16, bits8, 4, 16)
        for key, width in (("x", 512), ("weight", 512)):
            wide = torch.ones(s[key].shape[0], width + 48, dtype=s[key].dtype, device="cuda")
            wide[:, shift:shift + width] = s[key]
            s[key] = wide[:, shift:shift + width]
        wide = torch.full((rows, 400), 7.0, dtype=BF16, device="cuda")
        got = edge.project(**s, out=wide[:, shift:shift + 320])
        check(s, got, (rows, bits8, shift))
        assert (wide[:, :shift] == 7).all() and (wide[:, shift + 320:] == 7).all()


def test_eight_bits_without_rounding():
    """8-bit products are summed exactly: with unit scales small results are exact integers."""
    s = inputs(70, 4096, 200, F16, True)
    s["x"], s["weight"] = s["x"].clamp(-1, 1), s["weight"].clamp(-1, 1)
    s["x_scale"].fill_(1), s["weight_scale"].fill_(1)
    want = s["x"].double() @ s["weight"].double().T
    assert torch.equal(edge.project(**s).double(), want)
    top = torch.full((1, 131072), 127, dtype=torch.int8, device="cuda")
    one = torch.ones(1, device="cuda")
    got = edge.project(top, top, x_scale=one * 2.0 ** -20, weight_scale=one, dtype=F16)
    assert got.item() == torch.tensor(127.0 * 127 * 131072 / 2 ** 20).half().item()


def test_equal_calls_give_equal_bits_also_on_another_stream():
    for rows in (32, 500):
        s = inputs(rows, 2048, 512, BF16, False, 8, 16)
        first = edge.project(**s)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        again = edge.project(**s, stream=side.cuda_stream)
        side.synchronize()
        assert torch.equal(first, again) and torch.equal(first, edge.project(**s))
    assert edge.project(s["x"][:0], s["weight"]).shape == (0, 512)


def test_in_a_graph():
    s = inputs(48, 1024, 512, BF16, False, 8, 16)
    out = torch.empty(48, 512, dtype=BF16, device="cuda")
    space = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        edge.project(**s, out=out, workspace=space)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        edge.project(**s, out=out, workspace=space)
    for seed in range(3):
        new = inputs(48, 1024, 512, BF16, False, 8, 16, seed=10 + seed)
        s["x"].copy_(new["x"])
        want = edge.project(**s)
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("rows,out", [(1, 1), (20, 40), (64, 17), (70, 70), (300, 300)])
@pytest.mark.parametrize("shift", [0, 1])
def test_the_largest_eight_bit_sum(rows, out, shift):
    """131072 products of -128 and -128 are 2^31, one more than 32-bit integers hold; the others are exact beside it."""
    x, w = (torch.full((n, 131072 + 16), -128, dtype=torch.int8, device="cuda")[:, shift:shift + 131072] for n in (rows, out))
    x[1::2] = 127
    x[2::3, 5] = 127
    one = torch.ones(max(rows, out), device="cuda")
    got = edge.project(x, w, x_scale=one[:rows] * 2.0 ** -16, weight_scale=one[:out], dtype=BF16)
    want = x.double() @ w.double().T * 2.0 ** -16
    assert torch.equal(got, want.float().to(BF16))


@pytest.mark.parametrize("x,down,up", [(100.0, 100.0, 2.0 ** -14), (1e4, 3e3, 2.0 ** -24), (2.0 ** -9, 2.0 ** -10, 2.0 ** 13),
                                       (2.0 ** -6, 2.0 ** -8, 2.0 ** 10), (2.0 ** -12, 2.0 ** -13, 2.0 ** 13)])
@pytest.mark.parametrize("rows,i,o,n", [(40, 128, 96, 3), (200, 128, 96, 3), (300, 1000, 1111, 5), (100, 128, 96, 40),
                                        (2055, 328, 4100, 6)])
def test_low_rank_rows_of_any_size(rows, i, o, n, x, down, up):
    """binary16 low-rank rows x A^T above 65504 and far below 1, of many rows as of few."""
    s = inputs(rows, i, o, F16, False, n, 40, seed=rows)
    s["adapters"]["rank"] = torch.tensor([40, 17, 33][:n] + [40] * (n - 3), dtype=torch.int32, device="cuda")
    s["x"].mul_(x)
    s["weight"].mul_(min(1.0, 1 / x))
    s["adapters"]["down"].mul_(down)
    s["adapters"]["up"].normal_().mul_(up)
    s["adapters"]["down"][:, 3] *= 2.0 ** -6   # ranks of different sizes beside each other
    got = check(s)
    assert got.isfinite().all()


@pytest.mark.parametrize("rows,n", [((1 << 28) + 37, 1), (1 << 30, 0)])
def test_more_rows_than_one_dimension_of_a_grid(rows, n):
    gen = torch.Generator(device="cuda").manual_seed(0)
    s = inputs(1, 8, 8, BF16, False, n, 4)
    s["x"] = torch.empty(rows, 8, dtype=BF16, device="cuda").normal_(generator=gen)
    if n:
        s["row_adapter"] = torch.zeros(rows, dtype=torch.int32, device="cuda")
    got = edge.project(**s)
    for at in (0, rows // 2, rows - 500):
        part = {**s, "x": s["x"][at:at + 500]}
        if n:
            part["row_adapter"] = s["row_adapter"][at:at + 500]
        check(part, got[at:at + 500], at)
