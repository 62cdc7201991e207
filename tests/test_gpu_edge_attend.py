"""jdob_edge_attend against its definition in 64 bits."""

import random

import pytest
import torch

from paper_2504_14611_amd import edge
from tests import edge_model as model

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def inputs(new, keys, heads, kv_heads, dim, dtype, seed=0, room=5, fill=float("nan")):
    """Packed rows and slabs with `room` rows between them that hold `fill`."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    starts, at = [], room
    for m in keys:
        starts.append(at)
        at += m + room
    q = torch.randn(sum(new), heads, dim, generator=gen, device="cuda").to(dtype)
    k, v = (torch.full((at, kv_heads, dim), fill, dtype=dtype, device="cuda") for _ in range(2))
    for s, m in zip(starts, keys):
        for t in (k, v):
            t[s:s + m] = torch.randn(m, kv_heads, dim, generator=gen, device="cuda").to(dtype)
    return {"q": q, "k": k, "v": v,
            "query_start": torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device="cuda"),
            "key_start": torch.tensor(starts, dtype=torch.int64, device="cuda"),
            "key_count": torch.tensor(keys, dtype=torch.int32, device="cuda"),
            "max_queries": max(new, default=0), "max_keys": max(keys, default=0)}


def check(s, label, got=None, scale=None):
    got = edge.attend(**s, scale=scale) if got is None else got
    ref = {k: s[k] for k in ("q", "k", "v", "query_start", "key_start", "key_count")}
    dim = s["q"].shape[2]
    out, size, spread = model.attend(**ref, scale=dim ** -0.5 if scale is None else scale)
    off = (got.double() - out).abs() - model.attend_bound(out, size, spread, dim, s["max_keys"], got.dtype)
    assert not got.isnan().any(), label
    assert got.numel() == 0 or off.max() <= 0, (label, off.max(), (off > 0).sum())
    return got


CASES = [
    # new rows, keys
    ([1], [1]), ([1], [2]), ([1], [31]), ([1], [127]), ([1], [128]), ([1], [129]), ([1, 1, 1], [5, 300, 64]),
    ([1] * 5, [0, 1, 700, 33, 257]), ([2, 3], [2, 130]), ([7, 0, 1], [300, 10, 0]), ([33], [33]), ([20, 5], [10, 3]),
    ([64], [64]), ([65, 63], [65, 200]), ([128], [128]), ([129, 1, 0, 50], [129, 300, 7, 50]), ([200], [150]),
    ([130, 140], [1, 0]), ([257], [400]),
]


@pytest.mark.parametrize("heads,kv_heads,dim,dtype", [(4, 4, 64, BF16), (8, 2, 128, BF16), (6, 2, 80, F16),
                                                      (2, 1, 8, F16), (16, 1, 96, BF16), (5, 5, 40, BF16)])
@pytest.mark.parametrize("new,keys", CASES)
def test_attend(new, keys, heads, kv_heads, dim, dtype):
    check(inputs(new, keys, heads, kv_heads, dim, dtype, seed=sum(new) + sum(keys)), (new, keys))


@pytest.mark.parametrize("new,keys", [([1], [20000]), ([3], [5000]), ([1, 1], [9000, 4]), ([40], [3000])])
def test_long_histories(new, keys):
    check(inputs(new, keys, 4, 2, 128, BF16, seed=3), (new, keys))


@pytest.mark.parametrize("seed", range(4))
def test_many_sequences(seed):
    r = random.Random(seed)
    n = r.choice([65, 130, 200])
    new = [r.choice([0, 0, 1, 2, 9]) for _ in range(n)]
    keys = [max(0, x + r.randint(-3, 12)) for x in new]
    new[n // 2], keys[n // 2] = (140, 150) if seed % 2 else (3, 90)
    check(inputs(new, keys, 2, 1, 64, F16, seed=seed), (new, keys))


@pytest.mark.parametrize("new", [1, 5, 100, 300])
def test_large_scores_and_growing_maxima(new):
    """Scores far apart, whose maximum grows along the keys; a scale of its own."""
    s = inputs([new], [600], 2, 1, 64, BF16)
    s["k"][s["key_start"][0]:s["key_start"][0] + 600] *= torch.linspace(0.1, 12, 600, device="cuda")[:, None, None].to(BF16)
    check(s, new)
    check(s, new, scale=0.01)
    s["q"] *= 0  # equal scores
    check(s, new)


@pytest.mark.parametrize("new,keys", [(1, 1), (3, 70), (40, 40), (100, 250), (300, 300), (200, 130)])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_unseen_keys_and_values_change_nothing(new, keys, dtype):
    """Infinities and NaN in keys and values reach the rows that see them, and no others."""
    s = inputs([new], [keys], 4, 2, 64, dtype)
    clean = check(s, "clean")
    at = int(s["key_start"][0])
    for j in {0, keys // 2, keys - 1}:
        for name, value in (("k", float("nan")), ("k", float("inf")), ("v", float("nan")), ("v", float("-inf"))):
            t = {**s, name: s[name].clone()}
            t[name][at + j, 0, 5] = value
            got = edge.attend(**t)
            first = max(0, j - (keys - new))  # the first row that sees key j
            assert torch.equal(got[:first], clean[:first]), (j, name, value)
            assert torch.equal(got[first:, 2:], clean[first:, 2:]), (j, name, value)  # the other key head's heads
            if name == "v":
                assert not got[first:, :2, 5].isfinite().any(), (j, value)
                assert torch.equal(got[first:, :2, 6:], clean[first:, :2, 6:])


@pytest.mark.parametrize("new,keys", [([1, 1], [90, 300]), ([150, 20], [150, 60])])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_strides(new, keys, shift):
    """q, k and v as columns of one wide row, at any element; heads in the other order; out with gaps."""
    s = inputs(new, keys, 4, 2, 80, BF16, seed=7)
    want = check(s, "dense")
    rows = s["k"].shape[0]
    wide = torch.randn(rows, shift + 2 * 2 * 96, device="cuda").to(BF16)
    for i, name in enumerate("kv"):
        view = wide[:, shift + i * 192:shift + (i + 1) * 192].unflatten(1, (2, 96))[:, :, :80]
        view.copy_(s[name])
        s[name] = view
    q = torch.zeros(4, sum(new), 88, dtype=BF16, device="cuda")[:, :, shift % 8:shift % 8 + 80].transpose(0, 1)
    q.copy_(s["q"])
    s["q"] = q
    wide = torch.full((sum(new), 4, 100), 3.0, dtype=BF16, device="cuda")
    got = edge.attend(**s, out=wide[:, :, shift:shift + 80])
    assert torch.equal(got, want)
    assert (wide[:, :, :shift] == 3).all() and (wide[:, :, shift + 80:] == 3).all()


def test_a_cache_whose_offsets_pass_32_bits():
    """Keys and values behind 2^32 bytes and 2^31 elements of their buffers."""
    rows, dim = (1 << 31) // 64 + 5000, 64
    s = inputs([1, 130], [300, 200], 2, 1, dim, BF16)
    big = torch.empty(rows, 2, 1, dim, dtype=BF16, device="cuda")
    old = s["key_start"].tolist()
    starts = [rows - 1000, rows - 600]
    for i, name in enumerate("kv"):
        for o, a, m in zip(old, starts, (300, 200)):
            big[a:a + m, i] = s[name][o:o + m]
        s[name] = big[:, i]
    want = check({**s, "k": s["k"][rows - 2000:], "v": s["v"][rows - 2000:],
                  "key_start": torch.tensor([a - rows + 2000 for a in starts], device="cuda")}, "near")
    s["key_start"] = torch.tensor(starts, device="cuda")
    assert torch.equal(edge.attend(**s), want)


def test_index_arrays_out_of_range_stay_within_the_buffers():
    s = inputs([3, 2], [40, 50], 2, 1, 64, BF16)
    s["query_start"] = torch.tensor([-5, 3, 90], dtype=torch.int32, device="cuda")
    s["key_start"] = torch.tensor([-3, 1 << 40], dtype=torch.int64, device="cuda")
    s["key_count"] = torch.tensor([1 << 30, -7], dtype=torch.int32, device="cuda")
    for most in (3, 200):
        s["max_queries"] = most
        assert edge.attend(**s).shape == (5, 2, 64)
    torch.cuda.synchronize()


@pytest.mark.parametrize("new,keys", [([1] * 3, [3000, 10, 700]), ([200, 3], [300, 40])])
def test_equal_calls_give_equal_bits_also_on_another_stream_and_in_a_graph(new, keys):
    s = inputs(new, keys, 8, 2, 128, F16, fill=0.0)
    first = check(s, new)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = edge.attend(**s, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(first, again) and torch.equal(first, edge.attend(**s))
    out = torch.empty_like(s["q"])
    space = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    with torch.cuda.stream(side):
        edge.attend(**s, out=out, workspace=space)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        edge.attend(**s, out=out, workspace=space)
    for seed in range(3):
        s["q"].copy_(torch.randn(s["q"].shape, device="cuda"))
        want = edge.attend(**s)
        out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_nothing_to_do():
    s = inputs([], [], 2, 1, 64, BF16)
    assert edge.attend(**s).shape == (0, 2, 64)
    s = inputs([0, 0], [4, 0], 2, 1, 64, BF16)
    assert edge.attend(**s).shape == (0, 2, 64)


def far_scores(kind, keys, dim, dtype):
    """Keys whose scores with the query of `far_query` are far from zero and equal, or so far apart that one wins:
    the weights are 0 or 1 / n exactly, in 64 bits as in any other."""
    j = torch.arange(keys, device="cuda", dtype=torch.float64)[:, None].expand(keys, dim)
    low = torch.finfo(dtype).min
    return {"lowest": j * 0 + low, "highest": j * 0 - low, "first": -(j + 1) * 2.0 ** 100, "last": (j + 1) * 2.0 ** 100,
            "lowest, then zeros": torch.where(j < keys // 2, low, 0.0), "zeros, then lowest": torch.where(j < keys // 2, 0.0, low),
            "large": j * 0 + 60000.0, "large, then larger": torch.where(j < keys // 2, 50000.0, 60000.0),
            "large and negative": j * 0 - 60000.0}[kind].to(dtype)


@pytest.mark.parametrize("new,keys", [([1], [300]), ([5, 2], [70, 2]), ([1], [3000]), ([100], [130]), ([200, 140], [200, 100]),
                                      ([300], [700])])
@pytest.mark.parametrize("kind,dtype", [("lowest", BF16), ("highest", BF16), ("first", BF16), ("last", BF16),
                                        ("lowest, then zeros", BF16), ("zeros, then lowest", BF16), ("lowest", F16),
                                        ("large", F16), ("large, then larger", F16), ("large and negative", F16)])
def test_scores_far_from_zero(new, keys, kind, dtype):
    """Scores that binary32 holds are scores, however far from zero: a row's weights are their softmax."""
    s = inputs(new, keys, 4, 2, 64, dtype, seed=sum(keys))
    other = edge.attend(**s)
    for first, m in zip(s["key_start"].tolist(), keys):
        s["k"][first:first + m, 0] = far_scores(kind, m, 64, dtype)
    s["q"][:, :2] = 60000.0 if dtype == F16 else 2.0 ** -10
    for scale in (None, 0.01, 7.3):
        got = edge.attend(**s, scale=scale)
        ref = {k: s[k] for k in ("q", "k", "v", "query_start", "key_start", "key_count")}
        out, size, _ = model.attend(**ref, scale=64 ** -0.5 if scale is None else scale)
        off = (got.double() - out).abs() - model.attend_bound(out, size, torch.zeros_like(out[:, :, 0]), 64, max(keys), dtype)
        assert not got.isnan().any() and off[:, :2].max() <= 0, (scale, off[:, :2].max())
        if scale is None:  # the other key head's heads are what they were
            assert torch.equal(got[:, 2:], other[:, 2:])


@pytest.mark.parametrize("new,keys", [(1, 300), (100, 130), (300, 700)])
def test_rows_far_from_zero_beside_ordinary_ones(new, keys):
    """A row's roundings do not depend on the rows beside it, large scores among them."""
    s = inputs([new], [keys], 4, 2, 64, F16, seed=5)
    s["k"][s["key_start"][0]:][:keys, :, :8] = 30000.0
    s["q"][:, :, :8] = 0
    plain = check(s, "ordinary")
    s["q"][::3, ::2, :8] = 60000.0
    got = edge.attend(**s)
    keep = torch.ones(got.shape[:2], dtype=torch.bool, device="cuda")
    keep[::3, ::2] = False
    assert torch.equal(got[keep], plain[keep]) and not got.isnan().any()


def test_more_rows_than_one_dimension_of_a_grid():
    """2^28 rows of eight heads, of which the last four see keys."""
    rows, dim = (1 << 28) + 3, 8
    s = inputs([4], [4], 8, 8, dim, BF16)
    want = check(s, "four rows")
    s["q"] = s["q"][:1].expand(rows, 8, dim)
    s["query_start"], s["max_queries"] = torch.tensor([0, rows], dtype=torch.int32, device="cuda"), rows
    got = edge.attend(**s)
    assert torch.equal(got[rows - 4], want[0])
    for at in range(0, rows - 4, 1 << 24):
        assert not got[at:min(at + (1 << 24), rows - 4)].any(), at


def test_the_longest_sequence():
    """2^31 - 1 keys: positions behind the last one pass 32 bits."""
    m = (1 << 31) - 1
    kv = torch.zeros(m, 1, 8, dtype=BF16, device="cuda")
    kv[m - 1], kv[m - 3] = 16.0, 12.0
    q = torch.full((3, 1, 8), 16.0, dtype=BF16, device="cuda")
    at = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    first, count = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.full((1,), m, dtype=torch.int32, device="cuda")
    got = edge.attend(q, kv, kv, at, first, count)
    assert got[:, 0, 0].tolist() == [12.0, 12.0, 16.0] and torch.equal(got, got[:, :, :1].expand(3, 1, 8))


def test_hints_beyond_32_bits():
    s = inputs([5, 3], [9, 700], 4, 2, 64, BF16)
    want = check(s, "exact hints")
    for most in (1 << 31, (1 << 32) + 1):
        check({**s, "max_queries": most}, most)
        assert torch.equal(edge.attend(**{**s, "max_queries": 5, "max_keys": 700}), want)
        check({**s, "max_keys": most}, most)
