"""Inputs of the attentions whose scores are whole numbers that binary32 holds in any order of their sums, with the outputs
in 64 bits and how far a kernel may be from them: what shows is what the softmax and the values' sums lose.

Every key's score is `base` + its `scores` (whole numbers to 127), for all heads and rows; scale is 1."""

import torch

from tests import edge_cache_model as model

BF16, F16 = torch.bfloat16, torch.float16
HALF = {t: torch.finfo(t).eps / 2 for t in (BF16, F16)}  # half a step, relative
LEAST = {BF16: 2.0 ** -134, F16: 2.0 ** -25}             # half a step of the smallest numbers
U32 = 2.0 ** -24


def query(rows, heads, dim, dtype, base, device):
    q = torch.zeros(rows, heads, dim, dtype=dtype, device=device)
    q[..., :8], q[..., 8] = base / 512, 1
    assert (q[..., 0].double() * 512 == base).all()
    return q


def keys_of(scores, dim):
    """Keys [keys, dim]: 8 * 64 * base / 512 + the score."""
    x = torch.zeros(len(scores), dim, dtype=torch.float64, device=scores.device)
    x[:, :8], x[:, 8] = 64, scores
    return x


def paged(scores, v, base, new, page, kv_heads, group, dtype, bits8, v_scale=None):
    """One sequence of len(scores) keys, the last `new` of them its rows.  v [keys, dim]; with 8 bits whole numbers to 127,
    times v_scale [keys]."""
    m, dim, device = len(scores), v.shape[1], v.device
    s = model.inputs([new], [m], page, kv_heads, dim, dtype, bits8, group, device=device)
    s["q"] = query(new, kv_heads * group, dim, dtype, base, device)
    j = torch.arange(m, device=device)
    at = s["table"][0].long()[j // page], slice(None), j % page
    for name, x, scale in (("k", keys_of(scores, dim), None), ("v", v, v_scale)):
        held = x.to(s["cache"][name].dtype)
        assert torch.equal(held.double(), x.double()), name
        s["cache"][name][at] = held[:, None].expand(-1, kv_heads, -1)
        if bits8:
            scale = torch.ones(m, device=device) if scale is None else scale.float()
            s["cache"][name + "_scale"][at] = scale[:, None].expand(-1, kv_heads)
    return s


def packed(scores, v, base, new, kv_heads, group, dtype):
    """The same for packed keys: q, k, v, query_start, key_start, key_count."""
    m, dim, device = len(scores), v.shape[1], v.device
    k, v16 = (x.to(dtype)[:, None].repeat(1, kv_heads, 1) for x in (keys_of(scores, dim), v))
    assert torch.equal(v16[:, 0].double(), v.double())
    starts = (torch.tensor([0, new], dtype=torch.int32, device=device), torch.zeros(1, dtype=torch.int64, device=device),
              torch.tensor([m], dtype=torch.int32, device=device))
    return query(new, kv_heads * group, dim, dtype, base, device), k, v16, *starts


def outputs(scores, values, new):
    """For each of the last `new` keys as a row: the output and the weighted sum of |v| in 64 bits, [new, dim]."""
    out, mass = [], []
    for i in range(new):
        sees = len(scores) - new + i + 1
        p = torch.softmax(scores[:sees].double(), dim=0)
        out.append(p @ values[:sees].double())
        mass.append(p @ values[:sees].double().abs())
    return torch.stack(out), torch.stack(mass)


def bound(out, mass, keys, dtype, part, reach=128):
    """`part`: how far the weight that goes into the product may be from p, relative.  A difference of two scores, exact,
    is multiplied by scale * log2(e), which has been rounded, and rounds: an exponent to `reach` is off by reach * 2^-23, p
    by 0.7 of that, relative.  Waves and workgroups are joined by three more such factors: 4 * 0.7 * reach * 2^-23, and
    reach * 2^-21 stands for it and the exponentials' own steps.  Sums are binary32, numerator and denominator."""
    return out.abs() * HALF[dtype] * 1.01 + LEAST[dtype] + mass * (part + reach * 2.0 ** -21 + 2 * (keys + 64) * U32)


def over(got, scores, values, new, dtype, part, reach=128):
    """By how much the worst element of got [new, heads, dim] passes its bound (not above 0: none)."""
    out, mass = outputs(scores, values, new)
    off = (got.double() - out[:, None]).abs() - bound(out, mass, len(scores), dtype, part, reach)[:, None]
    assert not got.isnan().any() and not off.isnan().any()
    return off.max().item()


# ---- what the tests run, here and on the CPU

def far_scores(keys, seed, device, dim=16):
    """Scores within 12 of each other (seed 0: the first half's one above the others'); values that show weights."""
    gen = torch.Generator().manual_seed(seed)
    r = torch.randint(0, 13, (keys,), generator=gen) if seed else (torch.arange(keys) < keys // 2).int()
    v = torch.randint(0, 3, (keys, dim), generator=gen).float()
    v[:, 0] = torch.arange(keys) >= keys // 2
    return r.to(device), v.to(device)


def rising_scores(keys, seed, device, dim=16):
    """Tiles of 64 keys each 7 above the one before, so that the maximum has to follow; values that show each tile's weight."""
    tile = torch.arange(keys) // 64
    v = (tile[:, None] % dim == torch.arange(dim)).float()
    return (tile * 7).to(device), v.to(device)


def small_weights(keys, above, device, dim=16):
    """The first key's value is zero and its score `above` the others', whose large values show what small weights are."""
    gen = torch.Generator().manual_seed(above)
    r = (torch.arange(keys) == 0).int() * above
    v = torch.randint(64, 128, (keys, dim), generator=gen).float() * (r == 0)[:, None]
    return r.to(device), v.to(device), torch.full((keys,), 256.0, device=device)


def huge_values(keys, seed, device, dim=16):
    """Values near the end of bfloat16's range, of either sign in some columns, with scores that rise slowly: sums of values
    times weights that nobody has divided yet pass binary32."""
    gen = torch.Generator().manual_seed(seed)
    r = torch.arange(keys) * 5 // keys
    v = torch.randint(64, 128, (keys, dim), generator=gen).float()
    v[:, dim // 2:] *= torch.randint(0, 2, (keys, dim - dim // 2), generator=gen) * 2 - 1
    return r.to(device), v.to(device), torch.full((keys,), 2.0 ** 121, device=device)


def cancelling_values(keys, seed, dtype, bits8, device, dim=16):
    """The last key's values are chosen so that the output is next to nothing beside what is summed: it shows each weight's
    own rounding, not the output's.  For one row."""
    gen = torch.Generator().manual_seed(seed)
    r = torch.randint(0, 7, (keys,), generator=gen)
    r[0], r[-1] = 6, 5
    v = (torch.rand(keys, dim, generator=gen) * 254 - 127).round()
    v[-1] = 0
    p = torch.softmax(r.double(), dim=0)
    last = -(p @ v.double()) / p[-1]
    scale = torch.ones(keys)
    if bits8:
        scale[-1] = last.abs().max() / 127
        v[-1] = (last / scale[-1].double()).round()
    else:
        v[-1] = last.to(dtype).float()
    return r.to(device), v.to(device), scale.to(device)
