"""jdob_edge_attend_paged against its definition in 64 bits."""

import random

import pytest
import torch

from paper_2504_14611_amd import edge, jdob
from tests import edge_cache_model as model

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def call(s, new, keys, **kw):
    return edge.attend_paged(s["q"], s["cache"], s["table"], s["row_start"], s["key_count"],
                             **{"max_queries": max(new, default=0), "max_keys": max(keys, default=0), **kw})


def check(s, new, keys, label, got=None, scale=None, **kw):
    got = call(s, new, keys, scale=scale, **kw) if got is None else got
    d = s["q"].shape[2]
    out, mass, spread, most = model.attend(s["q"], s["cache"], s["table"].tolist(), s["row_start"].tolist(), keys,
                                           d ** -0.5 if scale is None else scale)
    bits8 = s["cache"]["k"].dtype is torch.int8
    bound = model.attend_bound(out, mass, spread, most, d, max(keys, default=0), got.dtype, bits8)
    # binary16 values may be infinite, and finite results may round to an infinity
    fine = out.isfinite()
    assert not got[~fine].isfinite().any(), label
    fine &= got.isfinite() | (out.abs() + bound < torch.finfo(got.dtype).max)
    assert not got[fine].isnan().any(), label
    off = ((got.double() - out).abs() - bound)[fine]
    assert off.numel() == 0 or off.max() <= 0, (label, off.max(), (off > 0).sum())
    return got


CASES = [
    # new rows, keys
    ([1], [1]), ([1], [2]), ([1], [31]), ([1], [32]), ([1], [33]), ([1], [129]), ([1, 1, 1], [5, 300, 64]),
    ([1] * 5, [0, 1, 700, 33, 257]), ([2, 3], [2, 130]), ([7, 0, 1], [300, 10, 0]), ([4, 9], [2, 40]), ([33], [40]),
]


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("page", [16, 64, 20, 7, 1])
@pytest.mark.parametrize("kv_heads,group,dim,dtype", [(4, 1, 64, BF16), (2, 4, 128, BF16), (2, 3, 80, F16), (1, 2, 8, F16),
                                                      (1, 16, 96, BF16), (3, 1, 40, BF16), (1, 24, 112, F16), (2, 7, 128, F16)])
def test_attend(page, kv_heads, group, dim, dtype, bits8):
    for new, keys in CASES:
        s = model.inputs(new, keys, page, kv_heads, dim, dtype, bits8, group, seed=sum(new) + sum(keys))
        check(s, new, keys, (new, keys))


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("page", [32, 128, 24, 5])
@pytest.mark.parametrize("new,keys", [([1], [20000]), ([3], [5000]), ([1, 1], [9000, 4]), ([1, 2, 1], [3000, 2900, 1])])
def test_long_histories(new, keys, page, bits8):
    """Keys that are split over workgroups."""
    check(model.inputs(new, keys, page, 2, 128, BF16, bits8, 4, seed=3), new, keys, (new, keys))


@pytest.mark.parametrize("seed", range(4))
def test_many_sequences(seed):
    r = random.Random(seed)
    n = r.choice([65, 130, 300])
    new = [r.choice([0, 0, 1, 2]) for _ in range(n)]
    keys = [max(0, x + r.randint(-3, 40)) for x in new]
    check(model.inputs(new, keys, r.choice([16, 4]), 2, 64, F16, seed % 2 == 1, 2, seed=seed), new, keys, (new, keys))


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("n,page", [(70, 16), (150, 12), (200, 64)])
def test_shares_of_many_sequences(n, page, bits8):
    """More sequences than lanes whose keys are dealt over workgroups: none, few and many keys, with and without rows."""
    r = random.Random(n)
    new = [r.choice([0, 1, 1, 2]) for _ in range(n)]
    keys = [r.choice([0, 3, 100, 700, 2000]) for _ in range(n)]
    new[n // 2], keys[n // 2], keys[n - 1] = 1, 7000, 4000
    check(model.inputs(new, keys, page, 2, 64, BF16, bits8, 3, seed=n), new, keys, (n, page))


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("page", [16, 48, 10])
def test_pages_that_have_been_given_back(page, bits8):
    """Keys on pages that are not there are not seen: at the beginning, in the middle, all of them."""
    new, keys = [1, 2, 1, 3], [400, 700, 90, 1000]
    held = [-(-m // page) for m in keys]
    gone = [(0, i) for i in range(3)] + [(1, 5), (1, 6), (1, held[1] - 1)] + [(2, i) for i in range(held[2])] + \
        [(3, i) for i in range(held[3] - 2)]
    s = model.inputs(new, keys, page, 2, 64, BF16, bits8, 4, gone=gone)
    got = check(s, new, keys, "gone")
    assert (got[3] == 0).all()


@pytest.mark.parametrize("bits8", [False, True])
def test_shared_pages(bits8):
    """Two sequences whose first pages are the same ones."""
    new, keys, page = [1, 1], [100, 70], 16
    s = model.inputs(new, keys, page, 2, 64, BF16, bits8, 4)
    s["table"][1, :3] = s["table"][0, :3]
    check(s, new, keys, "shared")


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("new", [1, 4])
def test_large_scores_and_growing_maxima(new, bits8):
    """Scores far apart, whose maximum grows along the keys; scores as far from zero as 2^30; a scale of its own."""
    keys = 600
    s = model.inputs([new], [keys], 16, 2, 64, BF16, bits8, 2)
    at = s["table"][0, :38].long()
    ramp = torch.linspace(0.1, 12, 38, device="cuda")
    if bits8:
        s["cache"]["k_scale"][at] *= ramp[:, None, None]
    else:
        s["cache"]["k"][at] *= ramp[:, None, None, None].to(BF16)
    check(s, [new], [keys], new)
    check(s, [new], [keys], new, scale=0.01)
    # one key's score is 2^30 above zero for every head, and the others' far below: the softmax is that key's value
    q = s["q"].abs() + 1
    s["q"] = q
    if bits8:
        s["cache"]["k"][at] = -1
        s["cache"]["k_scale"][at] = 1.0
    else:
        s["cache"]["k"][at] = -1.0
    s["cache"]["k"][at[3], :, 7] = 1
    if bits8:
        s["cache"]["k_scale"][at[3], :, 7] = 2.0 ** 24
    else:
        s["cache"]["k"][at[3], :, 7] = 2.0 ** 24
    got = call(s, [new], [keys])
    want = model.values(s["cache"], "v")[at[3], :, 7].repeat_interleave(2, dim=0).to(BF16).expand(new, 4, 64)
    assert torch.equal(got, want)
    # equal scores
    s["q"] = s["q"] * 0
    check(s, [new], [keys], new)


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("size", [2.0 ** -20, 1.0, 2.0 ** 12])
def test_values_of_any_size(size, dtype, bits8):
    """Values far from 1, some much larger than others."""
    s = model.inputs([1, 2], [300, 45], 16, 2, 128, dtype, bits8, 4, seed=5)
    loud = torch.where(torch.rand(s["cache"]["v"].shape[:3], device="cuda") < 0.02, 16.0, 0.25) * size
    if bits8:
        s["cache"]["v_scale"] *= loud
    else:
        s["cache"]["v"] = (s["cache"]["v"].float() * loud[..., None]).to(dtype)
    check(s, [1, 2], [300, 45], size)


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("new,keys", [(1, 1), (3, 70), (5, 5), (4, 700)])
@pytest.mark.parametrize("page", [16, 12])
def test_unseen_keys_and_values_change_nothing(new, keys, page, bits8):
    """Infinities and NaN in keys and values (8 bits: in scales) reach the rows that see them, and no others."""
    s = model.inputs([new], [keys], page, 2, 64, BF16, bits8, 4)
    clean = check(s, [new], [keys], "clean")
    table = s["table"].tolist()
    for j in {0, keys // 2, keys - 1, keys - 2 if keys > 1 else 0}:
        at, slot = table[0][j // page], j % page
        for name, value in (("k", float("nan")), ("k", float("inf")), ("v", float("nan")), ("v", float("-inf"))):
            cache = dict(s["cache"])
            if bits8:
                cache[name + "_scale"] = cache[name + "_scale"].clone()
                cache[name + "_scale"][at, 0, slot] = value
                cache[name] = cache[name].clone()
                cache[name][at, 0, slot, 5] = 3
            else:
                cache[name] = cache[name].clone()
                cache[name][at, 0, slot, 5] = value
            got = call({**s, "cache": cache}, [new], [keys])
            first = max(0, j - (keys - new))  # the first row that sees key j
            assert torch.equal(got[:first], clean[:first]), (j, name, value)
            assert torch.equal(got[first:, 4:], clean[first:, 4:]), (j, name, value)  # the other key head's heads
            if name == "v":
                assert not got[first:, :4, 5].isfinite().any(), (j, value)
                if not bits8:
                    assert torch.equal(got[first:, :4, 6:], clean[first:, :4, 6:])


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("shift", [0, 1, 8])
@pytest.mark.parametrize("order", ["slots before heads", "k and v interleaved", "pages inside"])
def test_strides(order, shift, bits8):
    """Caches in other orders, at any element; q as columns of a wide row; out with gaps."""
    new, keys, page, g, d = [1, 2, 1], [90, 300, 17], 16, 2, 80
    s = model.inputs(new, keys, page, g, d, BF16, bits8, 2, seed=7)
    want = check(s, new, keys, "dense")
    pages = s["cache"]["k"].shape[0]
    cache = {}
    for i, name in enumerate("kv"):
        old = s["cache"][name]
        if order == "slots before heads":
            wide = torch.zeros(pages, page, g, d + 16, dtype=old.dtype, device="cuda")[..., shift:shift + d].transpose(1, 2)
        elif order == "k and v interleaved":
            if i == 0:
                both = torch.zeros(pages, 2, g, page, d + 16, dtype=old.dtype, device="cuda")[..., shift:shift + d]
            wide = both[:, i]
        else:
            wide = torch.zeros(g, page, pages, d + 16, dtype=old.dtype, device="cuda")[..., shift:shift + d].permute(2, 0, 1, 3)
        wide.copy_(old)
        cache[name] = wide
        if bits8:
            scale = torch.zeros(page, g, pages, device="cuda").permute(2, 1, 0) if shift else torch.zeros(pages, g, page, device="cuda")
            cache[name + "_scale"] = scale.copy_(s["cache"][name + "_scale"])
    q = torch.zeros(4, sum(new), 96, dtype=BF16, device="cuda")[:, :, shift:shift + d].transpose(0, 1)
    q.copy_(s["q"])
    table = torch.full((len(new), s["table"].shape[1] + 5), 7, dtype=torch.int32, device="cuda")
    table[:, :-5] = s["table"]
    wide = torch.full((sum(new), 4, 100), 3.0, dtype=BF16, device="cuda")
    got = call({**s, "q": q, "cache": cache, "table": table[:, :-5]}, new, keys, out=wide[:, :, shift:shift + d])
    assert torch.equal(got, want)
    assert (wide[:, :, :shift] == 3).all() and (wide[:, :, shift + d:] == 3).all()


def test_scales_with_gaps():
    """Scales whose heads and pages start at any element, side by side within a page."""
    new, keys = [1, 2, 1], [90, 300, 17]
    s = model.inputs(new, keys, 16, 2, 64, BF16, True, 2, seed=7)
    want = check(s, new, keys, "dense")
    for name in ("k_scale", "v_scale"):
        old = s["cache"][name]
        s["cache"][name] = torch.full((old.shape[0], 2, 19), float("nan"), device="cuda")[:, :, 1:17].copy_(old)
    assert torch.equal(call(s, new, keys), want)


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("dim,dtype", [(64, BF16), (88, F16), (128, BF16)])
@pytest.mark.parametrize("page,shift", [(16, 0), (16, 1), (12, 0)])
def test_many_columns_after_many_keys(page, shift, dim, dtype, bits8):
    """More than 32 rows times heads of a key head, whose keys are read for 32 at once where the arrays allow."""
    new, keys = [5, 1, 3], [20000, 1, 300]
    s = model.inputs(new, keys, page, 8, dim, dtype, bits8, 8, seed=9)
    for name in ("k", "v"):
        old = s["cache"][name]
        wide = torch.zeros(*old.shape[:3], dim + 16, dtype=old.dtype, device="cuda")[..., shift:shift + dim]
        s["cache"][name] = wide.copy_(old)
    check(s, new, keys, "columns")


@pytest.mark.parametrize("bits8", [False, True])
@pytest.mark.parametrize("page", [64, 20, 9])
def test_a_cache_whose_offsets_pass_32_bits(page, bits8):
    """Pages behind 2^32 bytes and 2^31 elements of the cache."""
    d = 64
    pages = (1 << 33) // (page * d) // (1 if bits8 else 2) + 40
    s = model.inputs([1, 3], [300, 200], page, 1, d, BF16, bits8, 2)
    want = check(s, [1, 3], [300, 200], "near")
    small = s["cache"]["k"].shape[0]
    big = {n: None if t is None else torch.empty((pages, *t.shape[1:]), dtype=t.dtype, device="cuda") for n, t in s["cache"].items()}
    for n, t in s["cache"].items():
        if t is not None:
            big[n][pages - small:] = t
    table = torch.where((s["table"] >= 0) & (s["table"] < small), s["table"] + pages - small, -1)
    assert torch.equal(call({**s, "cache": big, "table": table}, [1, 3], [300, 200]), want)


def test_index_arrays_out_of_range_stay_within_the_buffers():
    s = model.inputs([3, 2], [40, 50], 16, 1, 64, BF16, False, 2, fill=0.0)
    s["row_start"] = torch.tensor([-5, 3, 90], dtype=torch.int32, device="cuda")
    s["key_count"] = torch.tensor([1 << 30, -7], dtype=torch.int32, device="cuda")
    for most in (3, 200):
        got = call(s, [most], [50])
        assert got.isfinite().all()
        assert most < 200 or (got[3:] == 0).all()


@pytest.mark.parametrize("bits8", [False, True])
def test_hints(bits8):
    """A cache that is longer than max_keys says; no hints at all; rows beyond the sequences stay as they were."""
    new, keys = [1, 1], [3000, 90]
    s = model.inputs(new, keys, 16, 2, 128, BF16, bits8, 4)
    want = check(s, new, keys, "hints")
    check(s, new, keys, "too few", got=call(s, new, keys, max_keys=1000))
    check(s, new, keys, "none", got=edge.attend_paged(s["q"], s["cache"], s["table"], s["row_start"], s["key_count"]))
    q = torch.cat([s["q"], s["q"]])
    out = torch.full_like(q, 5.0)
    call({**s, "q": q}, new, keys, out=out)
    assert torch.equal(out[:2], want) and (out[2:] == 5).all()


def test_nothing_to_do():
    s = model.inputs([1], [9], 16, 2, 64, BF16, False, 2)
    empty = {**s, "q": s["q"][:0]}
    assert call(empty, [0], [9]).shape == (0, 4, 64)
    none = {**s, "table": s["table"][:0], "row_start": s["row_start"][:1], "key_count": s["key_count"][:0]}
    call(none, [1], [9])
    # a cache without pages, a table without columns: rows see nothing
    bare = {n: None if t is None else t[:0] for n, t in s["cache"].items()}
    assert (call({**s, "cache": bare}, [1], [9]) == 0).all()
    assert (call({**s, "table": s["table"][:, :0].contiguous()}, [1], [9]) == 0).all()


@pytest.mark.parametrize("bits8", [False, True])
def test_equal_calls_give_equal_bits_whatever_stands_beside(bits8):
    """What a sequence's rows become does not depend on the call, nor on what its neighbours' rows, keys and values are
    (how the keys are split follows from all sequences' lengths)."""
    new, keys = [1, 1, 2], [5000, 77, 300]
    s = model.inputs(new, keys, 16, 2, 128, BF16, bits8, 4)
    want = call(s, new, keys)
    for _ in range(3):
        assert torch.equal(call(s, new, keys), want)
    at = s["row_start"].tolist()
    for u in range(3):
        mine = torch.zeros(s["cache"]["k"].shape[0], dtype=torch.bool, device="cuda")
        mine[s["table"][u, :-(-keys[u] // 16)].long()] = True
        cache = {n: None if t is None else t.clone() for n, t in s["cache"].items()}
        for n in ("v_scale", "k_scale") if bits8 else ("k", "v"):
            cache[n][~mine] *= 7
        q = s["q"] * 3
        q[at[u]:at[u + 1]] = s["q"][at[u]:at[u + 1]]
        got = call({**s, "q": q, "cache": cache}, new, keys)
        assert torch.equal(got[at[u]:at[u + 1]], want[at[u]:at[u + 1]]), u
        assert not torch.equal(got, want)


@pytest.mark.parametrize("bits8", [False, True])
def test_streams_graphs_and_workspaces(bits8):
    """On another stream; captured in two graphs that share a workspace and replayed with the program's own work between."""
    new, keys = [1, 1], [4000, 600]
    s, t = (model.inputs(new, keys, 16, 2, 128, BF16, bits8, 4, seed=i) for i in (1, 2))
    want = [call(x, new, keys) for x in (s, t)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = call(s, new, keys)
    side.synchronize()
    assert torch.equal(got, want[0])
    handle = side.cuda_stream
    got = call(s, new, keys, stream=handle)
    side.synchronize()
    assert torch.equal(got, want[0])
    space = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(x) for x in want]
    graphs = []
    for x, out in zip((s, t), outs):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(x, new, keys, out=out, workspace=space)
        graphs.append(graph)
    for _ in range(4):
        for graph, out, w in zip(graphs, outs, want):
            out.fill_(9)
            space.fill_(255)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, w)
            assert torch.equal(call(t, new, keys), want[1])


@pytest.mark.parametrize("bits8", [False, True])
def test_two_calls_at_once(bits8):
    """Two batches over one cache on two streams, neither waiting for the other."""
    new, keys = [1, 2], [6000, 300]
    s = model.inputs(new, keys, 16, 4, 128, BF16, bits8, 4, seed=1)
    t = {**s, "q": torch.randn_like(s["q"].float()).to(BF16)}
    want = [call(x, new, keys) for x in (s, t)]
    sides = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for x, side in zip((s, t), sides):
            with torch.cuda.stream(side):
                got.append(call(x, new, keys))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i % 2]) for i, g in enumerate(got))


def test_refusals():
    s = model.inputs([1], [90], 16, 2, 64, BF16, True, 2)
    none = {"k": s["cache"]["k"], "v": s["cache"]["v"]}
    for bad in ({**s, "q": s["q"].cpu()}, {**s, "q": s["q"].float()}, {**s, "q": s["q"][:, :3]}, {**s, "q": s["q"][..., :56]},
                {**s, "cache": none}, {**s, "cache": {**s["cache"], "v": s["cache"]["v"][:1]}},
                {**s, "cache": {**s["cache"], "k_scale": s["cache"]["k_scale"].half()}},
                {**s, "table": s["table"].long()}, {**s, "table": s["table"][0]}, {**s, "key_count": s["key_count"].long()},
                {**s, "row_start": s["row_start"][:1]}, {**s, "table": s["table"].expand(1, -1).cpu()}):
        with pytest.raises(jdob.JdobError):
            call(bad, [1], [90])
    with pytest.raises(jdob.JdobError):
        call(s, [1], [90], max_keys=-1)
    with pytest.raises(jdob.JdobError):
        call(s, [1], [90], scale=0.0)
