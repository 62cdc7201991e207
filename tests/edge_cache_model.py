"""The operators on a paged cache in 64 bits, from their definitions, inputs for them, and how far an output may be off.

A cache is a dict of k and v [pages, heads, page size, columns] and, with 8 bits, k_scale and v_scale.  Bounds follow
from the roundings that include/jdob_edge.h states, as in edge_model: inputs (codes and scales among them) are taken as
they are, sums are binary32 with a factor of two for the matrix units' own order, outputs are rounded once."""

import torch

from tests.edge_model import LEAST, U32, UNIT

BF16, F16 = torch.bfloat16, torch.float16


def place(table, page_size, pages, u, j):
    """Page and slot of key j of sequence u, None where it is absent."""
    i = j // page_size
    if j < 0 or i >= len(table[u]) or not 0 <= table[u][i] < pages:
        return None
    return table[u][i], j % page_size


def rows_of(table, row_start, key_count, page_size, pages):
    """(row, page, slot) of every row that stands somewhere, and (row, u, key) of those that belong to a sequence."""
    stands, belong = [], []
    for u in range(len(key_count)):
        n = row_start[u + 1] - row_start[u]
        for i in range(n):
            j = key_count[u] - n + i
            belong.append((row_start[u] + i, u, j))
            at = place(table, page_size, pages, u, j)
            if at is not None:
                stands.append((row_start[u] + i, *at))
    return stands, belong


def quantised(x):
    """Codes and scales of rows [..., columns], by binary32 divisions (a 64-bit quotient of binary32 numbers, rounded
    to binary32, is the binary32 quotient: 53 bits are more than 2 * 24 + 2)."""
    x = x.double()
    top = x.abs().amax(dim=-1)
    scale = (top / 127).float()
    fine = top.isfinite()
    q = (x / torch.where(scale > 0, scale, 1.0).double()[..., None]).float().double()
    codes = torch.where((fine & (scale > 0))[..., None], q.round().clamp(-127, 127).nan_to_num(0.0), 0.0)
    return codes.to(torch.int8), torch.where(fine, scale, float("nan"))


def values(cache, name):
    """What k or v stands for, in 64 bits."""
    x = cache[name].double()
    return x if cache.get(name + "_scale") is None else x * cache[name + "_scale"].double()[..., None]


def attend(q, cache, table, row_start, key_count, scale):
    """out, the weighted sums of |v|, the scores' largest sums of absolute products of a row, the largest |v| seen."""
    k, v = values(cache, "k"), values(cache, "v")
    pages, g, size, d = k.shape
    h = q.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    mass, most = torch.zeros_like(out), torch.zeros_like(out)
    spread = torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    for u in range(len(key_count)):
        n = row_start[u + 1] - row_start[u]
        if n <= 0:
            continue
        there = [(j, *place(table, size, pages, u, j)) for j in range(max(0, key_count[u])) if place(table, size, pages, u, j)]
        if not there:
            continue
        j, page, slot = (torch.tensor(x, device=q.device) for x in zip(*there))
        for i in range(n):
            sees = int((j <= key_count[u] - n + i).sum())
            if not sees:
                continue
            kk, vv = (t[page[:sees], :, slot[:sees]].transpose(0, 1).contiguous() for t in (k, v))  # [g, sees, d]
            qq = q[row_start[u] + i].double().view(g, h // g, d)
            p = torch.softmax(scale * torch.bmm(qq, kk.transpose(1, 2).contiguous()), dim=2)
            row = row_start[u] + i
            out[row] = torch.bmm(p, vv).reshape(h, d)
            mass[row] = torch.bmm(p, vv.abs()).reshape(h, d)
            most[row] = vv.abs().amax(dim=1).repeat_interleave(h // g, dim=0)
            spread[row] = abs(scale) * torch.bmm(qq.abs(), kk.abs().transpose(1, 2).contiguous()).amax(dim=2).reshape(h)
    return out, mass, spread, most


def attend_bound(out, mass, spread, most, dim, keys, dtype, bits8):
    # A score is off by (2 dim + 8) roundings of its products' sum (the key's scale among them), and the exponential by
    # as much again, relative.  p is rounded to dtype, in the numerator only; to a binary16 not below 2^-25, relative to
    # the largest of at least 1.  With 8 bits it is held as two bfloat16 parts: what is left of it is at most 2^-16 of it.
    off = 2 * (2 * dim + 10) * U32 * spread[..., None] + (2 * keys + 64) * U32
    part = 2.0 ** -16 if bits8 else UNIT[dtype]
    tiny = keys * 2.0 ** -25 * most if dtype is F16 and not bits8 else 0
    return out.abs() * (UNIT[dtype] + off) + mass * (part + off) + tiny + LEAST[dtype] * 4


def inputs(new, keys, page, kv_heads, dim, dtype, bits8, group=0, seed=0, device="cuda", gone=(), fill=float("nan"), spare=3):
    """Sequences whose pages lie anywhere in a cache; `gone`: (sequence, entry) that are no page; slots in use hold normal
    values (8 bits: codes), all others `fill` (8 bits: scales of it)."""
    gen = torch.Generator(device=device).manual_seed(seed)
    held = [-(-m // page) for m in keys]
    width = max(held, default=0) + 2
    pages = sum(held) + spare
    order = torch.randperm(pages, generator=gen, device=device).tolist()
    absent = [-1, pages, 1 << 30, -(1 << 31)]
    table = [[absent[(u + i) % 4] for i in range(width)] for u in range(len(keys))]
    at = 0
    for u, h in enumerate(held):
        for i in range(h):
            if (u, i) not in gone:
                table[u][i] = order[at]
                at += 1

    def normal(*size):
        return torch.randn(*size, generator=gen, device=device)

    shape = (pages, kv_heads, page, dim)
    cache = {"k_scale": None, "v_scale": None}
    used = torch.zeros(pages, page, dtype=torch.bool)
    for u, m in enumerate(keys):
        for i in range(held[u]):
            if 0 <= table[u][i] < pages:
                used[table[u][i], :m - i * page] = True
    used = used.to(device)[:, None]
    for name in ("k", "v"):
        if bits8:
            cache[name] = normal(*shape).mul_(40).round_().clamp_(-127, 127).to(torch.int8)
            scale = torch.rand(shape[:3], generator=gen, device=device).add_(0.2).mul_(1 / 40)
            cache[name + "_scale"] = torch.where(used.expand(shape[:3]), scale, fill)
        else:
            cache[name] = torch.where(used[..., None].expand(shape), normal(*shape), fill).to(dtype)
    s = {"cache": cache, "table": torch.tensor(table, dtype=torch.int32, device=device).view(len(keys), width),
         "row_start": torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device=device),
         "key_count": torch.tensor(keys, dtype=torch.int32, device=device)}
    if group:
        s["q"] = normal(sum(new), kv_heads * group, dim).to(dtype)
    return s
