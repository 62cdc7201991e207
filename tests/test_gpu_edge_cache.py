"""jdob_edge_cache_write and jdob_edge_cache_read against their definitions, and a run of them with the attention.

Codes and scales are binary32 divisions and compared bit by bit; what is read back is one rounding of code * scale."""

import pytest
import torch

from paper_2504_14611_amd import edge, jdob
from tests import edge_cache_model as model

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def fresh(s, garbage=True):
    """The cache's tensors with recognisable contents."""
    return {n: None if t is None else t.clone() for n, t in s["cache"].items()}


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def written(s, k, v):
    """The cache after the rows have been written, from the definition."""
    cache = fresh(s)
    pages, _, page, _ = cache["k"].shape
    stands, _ = model.rows_of(s["table"].tolist(), s["row_start"].tolist(), s["key_count"].tolist(), page, pages)
    if stands:
        row, at, slot = (torch.tensor(x, device=k.device) for x in zip(*stands))
        for name, x in (("k", k), ("v", v)):
            if cache[name].dtype is torch.int8:
                cache[name][at, :, slot], cache[name + "_scale"][at, :, slot] = model.quantised(x[row])
            else:
                cache[name][at, :, slot] = x[row]
    return cache


def read(s, cache, rows, dtype):
    pages, g, page, d = cache["k"].shape
    stands, belong = model.rows_of(s["table"].tolist(), s["row_start"].tolist(), s["key_count"].tolist(), page, pages)
    got = []
    for name in ("k", "v"):
        x = torch.full((rows, g, d), 5.0, dtype=dtype, device=cache["k"].device)
        if belong:
            x[torch.tensor([b[0] for b in belong], device=x.device)] = 0
        if stands:
            row, at, slot = (torch.tensor(t, device=x.device) for t in zip(*stands))
            x[row] = model.values(cache, name)[at, :, slot].float().to(dtype)  # (codes times scales: one rounding to binary32)
        got.append(x)
    return got


def rows(n, g, d, dtype, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    both = torch.randn(n, 2, g, d, generator=gen, device="cuda")
    both[:, :, :, ::16] *= 4
    both = both.to(dtype)
    return both[:, 0], both[:, 1]


def check(s, k, v, label):
    cache = fresh(s)
    edge.cache_write(k, v, cache, s["table"], s["row_start"], s["key_count"])
    want = written(s, k, v)
    for n, t in want.items():
        assert t is None or same(cache[n], t), (label, n)
    n, dtype = k.shape[0], k.dtype
    into = {x: torch.full((n, *cache["k"].shape[1::2]), 5.0, dtype=dtype, device="cuda") for x in "kv"}
    got = edge.cache_read(cache, s["table"], s["row_start"], s["key_count"], into=into)
    for a, b in zip(got, read(s, want, n, dtype)):
        # (which NaN a NaN is, is left open)
        assert torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(0.0), b.nan_to_num(0.0)), label
    return cache


CASES = [([1], [1]), ([1], [40]), ([3, 0, 5], [3, 9, 70]), ([20, 4, 1], [9, 0, 300]), ([130, 1], [130, 1]), ([0, 0, 65], [4, 4, 66])]


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("page", [16, 64, 20, 1])
@pytest.mark.parametrize("kv_heads,dim,dtype", [(8, 128, BF16), (3, 80, F16), (1, 8, F16), (2, 64, BF16), (5, 72, BF16)])
def test_write_and_read(page, kv_heads, dim, dtype, bits8):
    for new, keys in CASES:
        s = model.inputs(new, keys, page, kv_heads, dim, dtype, bits8, seed=sum(keys))
        check(s, *rows(sum(new), kv_heads, dim, dtype), (new, keys))


@pytest.mark.parametrize("bits8", [False, True])
def test_many_sequences(bits8):
    """As many as take several steps of the search, most of them without rows."""
    new = [(i * 7 + 3) % 5 if i % 9 == 0 else 0 for i in range(5000)]
    keys = [n + i % 3 for i, n in enumerate(new)]
    s = model.inputs(new, keys, 4, 1, 64, BF16, bits8)
    check(s, *rows(sum(new), 1, 64, BF16), "many")


@pytest.mark.parametrize("bits8", [False, True])
def test_rows_that_stand_nowhere(bits8):
    """Pages that are not there, rows before the first key, rows of no sequence, counts below zero."""
    new, keys = [30, 40, 6], [50, 25, 60]
    s = model.inputs(new, keys, 16, 2, 64, BF16, bits8, gone=[(0, 2), (1, 0), (2, 3)])
    k, v = rows(90, 2, 64, BF16)
    check(s, k, v, "gone")
    s["key_count"][1] = -4
    check(s, k, v, "below zero")
    s["row_start"] += 5  # rows before the first sequence, too
    check(s, k, v, "shifted")


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_codes(dtype):
    """Zeros, ties (half of the largest value lies between two codes), subnormals, the largest values, infinities and
    NaN: each row its own."""
    s = model.inputs([64], [64], 16, 2, 64, dtype, True)
    k, v = (x.contiguous() for x in rows(64, 2, 64, dtype))
    least, most = torch.finfo(dtype).smallest_normal, torch.finfo(dtype).max
    k[0] = 0
    k[1, 0, 5], k[2, 1, 63], k[3, 0, 0] = float("nan"), float("inf"), float("-inf")
    for i, top in enumerate(torch.linspace(1.0, 1.992, 40).to(dtype).tolist()):
        k[4 + i] = (k[4 + i].float() / 8).clamp(-top, top).to(dtype)
        k[4 + i, :, 0], k[4 + i, :, 1], k[4 + i, :, 2] = top, top / 2, -top / 2
    k[45] = k[45] * least
    k[46], k[46, 0, 3] = 0, least * torch.finfo(dtype).eps  # the smallest subnormal
    k[47] = most
    k[48, :, ::2], k[48, :, 1::2] = -most, 1.0
    cache = check(s, k, v, "codes")
    assert (cache["k"][s["table"][0, 0], :, 0] == 0).all() and (cache["k_scale"][s["table"][0, 0], :, 0] == 0).all()


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("shift", [0, 1, 4])
def test_strides(shift, bits8):
    """Rows as columns of a wide row at any element; caches in another order; read into wide rows."""
    new, keys, page, g, d = [40, 3], [60, 3], 16, 3, 72
    s = model.inputs(new, keys, page, g, d, BF16, bits8)
    wide = torch.randn(sum(new), 2, g, d + 8, device="cuda").to(BF16)[..., shift:shift + d]
    pages = s["cache"]["k"].shape[0]
    for name in ("k", "v"):
        old = s["cache"][name]
        s["cache"][name] = torch.zeros(pages, page, g, d + 8, dtype=old.dtype, device="cuda")[..., shift:shift + d].transpose(1, 2).copy_(old)
        if bits8:
            scale = s["cache"][name + "_scale"]
            s["cache"][name + "_scale"] = torch.zeros(page, g, pages, device="cuda").permute(2, 1, 0).copy_(scale)
    want = written(s, wide[:, 0], wide[:, 1])
    edge.cache_write(wide[:, 0], wide[:, 1], s["cache"], s["table"], s["row_start"], s["key_count"])
    for n, t in want.items():
        assert t is None or same(s["cache"][n].contiguous(), t.contiguous()), n
    into = torch.full((sum(new), 2, g, d + 8), 5.0, dtype=BF16, device="cuda")
    part = into[..., shift:shift + d]
    edge.cache_read(s["cache"], s["table"], s["row_start"], s["key_count"], into={"k": part[:, 0], "v": part[:, 1]})
    for a, b in zip((part[:, 0], part[:, 1]), read(s, want, sum(new), BF16)):
        assert torch.equal(a, b)
    assert (into[..., :shift] == 5).all() and (into[..., shift + d:] == 5).all()


@pytest.mark.parametrize("bits8", [False, True])
def test_index_arrays_out_of_range_stay_within_the_buffers(bits8):
    s = model.inputs([30, 10], [40, 50], 16, 2, 64, BF16, bits8)
    k, v = rows(40, 2, 64, BF16)
    for start, count in (([-7, 100, 60], [1 << 30, -5]), ([30, 10, 0], [40, 50]), ([0, 1 << 30, 1 << 30], [0x7fffffff, 3])):
        s["row_start"] = torch.tensor(start, dtype=torch.int32, device="cuda")
        s["key_count"] = torch.tensor(count, dtype=torch.int32, device="cuda")
        edge.cache_write(k, v, s["cache"], s["table"], s["row_start"], s["key_count"])
        edge.cache_read(s["cache"], s["table"], s["row_start"], s["key_count"], rows=40)
    torch.cuda.synchronize()


@pytest.mark.parametrize("bits8", [False, True])
def test_a_cache_whose_offsets_pass_32_bits(bits8):
    page, d = 64, 64
    pages = (1 << 33) // (page * d) // (1 if bits8 else 2) + 40
    cache = edge.make_cache(pages, page, 1, d, bits8=bits8)
    table = torch.tensor([[pages - 1, pages - 30, 0]], dtype=torch.int32, device="cuda")
    start, count = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 150], [150]))
    k, v = rows(150, 1, d, BF16)
    edge.cache_write(k, v, cache, table, start, count)
    a, b = edge.cache_read(cache, table, start, count, rows=150)
    small = edge.make_cache(3, page, 1, d, bits8=bits8)
    near = torch.tensor([[2, 1, 0]], dtype=torch.int32, device="cuda")
    edge.cache_write(k, v, small, near, start, count)
    for n, t in small.items():
        assert t is None or all(torch.equal(cache[n][i], t[j]) for i, j in ((pages - 1, 2), (pages - 30, 1)))
    c, e = edge.cache_read(small, near, start, count, rows=150)
    assert torch.equal(a, c) and torch.equal(b, e)


@pytest.mark.parametrize("bits8", [False, True])
def test_streams_and_graphs(bits8):
    """Written on another stream; captured and replayed on new rows."""
    new, keys = [30, 1], [50, 20]
    s = model.inputs(new, keys, 16, 2, 128, BF16, bits8)
    k, v = (x.contiguous() for x in rows(31, 2, 128, BF16))
    cache, side = fresh(s), torch.cuda.Stream()
    torch.cuda.synchronize()
    edge.cache_write(k, v, cache, s["table"], s["row_start"], s["key_count"], stream=side.cuda_stream)
    got = edge.cache_read(cache, s["table"], s["row_start"], s["key_count"], rows=31, stream=side.cuda_stream)
    side.synchronize()
    want = written(s, k, v)
    assert all(t is None or same(cache[n], t) for n, t in want.items())
    assert all(torch.equal(a, b) for a, b in zip(got, read(s, want, 31, BF16)))
    cache, into = fresh(s), {"k": torch.empty_like(k), "v": torch.empty_like(v)}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        edge.cache_write(k, v, cache, s["table"], s["row_start"], s["key_count"])
        edge.cache_read(cache, s["table"], s["row_start"], s["key_count"], into=into)
    for i in range(4):
        a, b = rows(31, 2, 128, BF16, seed=10 + i)
        k.copy_(a), v.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        want = written({**s, "cache": cache}, k, v)
        assert all(t is None or same(cache[n], t) for n, t in want.items())
        assert all(torch.equal(x, y) for x, y in zip((into["k"], into["v"]), read(s, want, 31, BF16)))


def test_refusals():
    s = model.inputs([4], [20], 16, 2, 64, BF16, True)
    k, v = rows(4, 2, 64, BF16)
    where = (s["table"], s["row_start"], s["key_count"])
    for args in ((k.cpu(), v, s["cache"]), (k, v[:3], s["cache"]), (k.float(), v.float(), s["cache"]), (k[..., :56], v[..., :56], s["cache"]),
                 (k[:, :1], v[:, :1], s["cache"]), (k, v, {**s["cache"], "v_scale": None}), (k, v, {**s["cache"], "k": s["cache"]["k"].bfloat16()}),
                 (k, v, {**s["cache"], "k": s["cache"]["k"][:, :1].expand(-1, 2, -1, -1)})):
        with pytest.raises(jdob.JdobError):
            edge.cache_write(*args, *where)
    with pytest.raises(jdob.JdobError):
        edge.cache_read(s["cache"], *where)
    with pytest.raises(jdob.JdobError):
        edge.cache_read(s["cache"], *where, rows=4, dtype=torch.float32)
    with pytest.raises(jdob.JdobError):
        edge.cache_read(s["cache"], *where, into={"k": k[:1].expand(4, -1, -1), "v": torch.empty(4, 2, 64, dtype=BF16, device="cuda")})
    with pytest.raises(jdob.JdobError):
        edge.make_cache(4, 16, 2, 60)
    with pytest.raises(jdob.JdobError):
        edge.make_cache(4, 0, 2, 64)


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("page", [16, 12])
def test_a_decode_is_the_attention_of_its_rows(page, bits8):
    """Prompts written, then tokens one by one, then a few at once: each step's attention over the pages is that of
    packed 16-bit rows that hold what the cache stands for; pages are taken as the sequences grow."""
    g, group, d, users = 2, 4, 128, 3
    free = list(range(80))[::-1]
    cache = edge.make_cache(80, page, g, d, bits8=bits8)
    table = torch.full((users, 20), -1, dtype=torch.int32, device="cuda")
    have, held, kept = [0] * users, [0] * users, [[torch.empty(0, g, d, dtype=BF16, device="cuda")] * 2 for _ in range(users)]
    gen = torch.Generator(device="cuda").manual_seed(4)
    for step, new in enumerate([(17, 0, 90), (1, 5, 1)] + [(1, 1, 1)] * 6 + [(4, 1, 0), (1, 1, 1)]):
        n = sum(new)
        qkv = torch.randn(n, g * (group + 2), d, generator=gen, device="cuda").bfloat16()
        q, k, v = qkv[:, :g * group], qkv[:, g * group:g * (group + 1)], qkv[:, g * (group + 1):]
        for u in range(users):
            have[u] += new[u]
            while held[u] * page < have[u]:
                table[u, held[u]] = free.pop()
                held[u] += 1
        start = torch.tensor([sum(new[:u]) for u in range(users + 1)], dtype=torch.int32, device="cuda")
        count = torch.tensor(have, dtype=torch.int32, device="cuda")
        edge.cache_write(k, v, cache, table, start, count)
        got = edge.attend_paged(q, cache, table, start, count, max_queries=max(new), max_keys=max(have))
        back = edge.cache_read(cache, table, start, count, rows=n)
        for i, x in enumerate((k, v)):
            if bits8:
                codes, scale = model.quantised(x)
                x = (codes.double() * scale.double()[..., None]).float().bfloat16()
            assert torch.equal(back[i], x)
        at = start.tolist()
        for u in range(users):
            kept[u] = [torch.cat([old, x[at[u]:at[u + 1]]]) for old, x in zip(kept[u], back)]
        ks, vs = (torch.cat([kept[u][i] for u in range(users)]) for i in range(2))
        first = torch.tensor([sum(have[:u]) for u in range(users)], device="cuda")
        want = edge.attend(q, ks, vs, start, first, count, max_queries=max(new), max_keys=max(have))
        # both round p and the output to bfloat16 (UNIT = 2^-8 each, relative to the weighted sums of |v|), and what has
        # been read back is rounded once more: its scores are off by 2^-8 of each product, its values by 2^-8
        out, mass, spread, most = model.attend(q, cache, table.tolist(), at, have, d ** -0.5)
        bound = model.attend_bound(out, mass, spread, most, d, max(have), BF16, bits8)
        assert ((got.double() - out).abs() <= bound).all(), step
        slack = mass * 2 * 2.0 ** -8 * (1 + (spread[..., None] + 1 if bits8 else 0))
        assert ((got.double() - want.double()).abs() <= 2 * bound + slack).all(), step
        full = torch.tensor([0] + [sum(have[:u + 1]) for u in range(users)], dtype=torch.int32, device="cuda")
        a, b = edge.cache_read(cache, table, full, count, rows=sum(have))
        assert torch.equal(a, ks) and torch.equal(b, vs)
