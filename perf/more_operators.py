"""Timed cases of the edge operators on a paged cache of keys and values: what the edge GPU keeps of its users' histories.

`write` puts new rows' keys and values into the pages of a cache, 16-bit rows as they are or in 8 bits with a scale for
every row and key head; `read` brings histories back as packed 16-bit rows, as a chunk's attention takes them; `attend`
is the attention of every sequence's newest rows (one token, or a few that are checked at once) over its pages; `step`
is what one token takes: its row written, its attention.

A sequence's keys stand on the pages that its row of `table` names, `page` keys on each: pages lie anywhere in the
cache, and those that stand behind a window have been given back (-1).  Sequence u's rows row_start[u] ..
row_start[u + 1] are the last of its key_count[u] keys.

The plain forms are elementary torch operations in 32 bits, sequences padded to the longest one.
"""

import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def _case(name, op, users, new_lo, new_hi, old_lo, old_hi, kv_heads, dim, page, bits8, dtype="bf16", group=0, window=0, mix=0):
    """`users` sequences with new_lo..new_hi rows after old_lo..old_hi keys (below 0: fewer keys than rows, whose first
    rows stand nowhere); `group` heads read a key head; `window`: whole pages more than so many keys back are gone
    (0: none); the lengths follow from `mix`."""
    return dict(name=name, op=op, users=users, new_lo=new_lo, new_hi=new_hi, old_lo=old_lo, old_hi=old_hi, kv_heads=kv_heads,
                dim=dim, page=page, bits8=bits8, dtype=dtype, group=group, window=window, mix=mix)


def listed():
    return [
        # one new token of each of 32 users: a call whose latency counts
        _case("write_tokens", "write", 32, 1, 1, 15, 1023, 8, 128, 16, False),
        # a batch of prompts, quantised as they are written
        _case("write_prompts_8bit", "write", 32, 40, 1000, 0, 0, 8, 128, 64, True),
        # chunks of a small model after histories, pages and heads that fit no tile, rows that stand nowhere
        _case("write_odd", "write", 9, 0, 300, -20, 700, 3, 80, 24, True, dtype="f16"),
        # histories of 16 users, ahead of their next chunks
        _case("read_chunks", "read", 16, 0, 8192, 0, 0, 4, 64, 16, False, dtype="f16"),
        # one very long history out of 8 bits
        _case("read_long_8bit", "read", 1, 131072, 131072, 0, 0, 8, 128, 256, True),
        # one new token of each of four users with short histories: a call whose latency counts
        _case("attend_short_8bit", "attend", 4, 1, 1, 19, 400, 4, 128, 16, True, group=4),
        # one new token of each of 32 users with histories of very different lengths
        _case("attend_tokens", "attend", 32, 1, 1, 15, 8191, 8, 128, 16, False, group=4),
        # one user's new token after a very long history: few rows, one long axis
        _case("attend_token_long_8bit", "attend", 1, 1, 1, 131071, 131071, 8, 128, 128, True, group=4),
        # a few drafted tokens at once, pages that end inside tiles, a head size between two tiles, rows that see nothing
        _case("attend_drafts", "attend", 24, 1, 5, -2, 3000, 2, 96, 20, False, dtype="f16", group=7),
        # long histories of which a window is kept
        _case("attend_window_8bit", "attend", 16, 1, 1, 20000, 32767, 2, 64, 32, True, dtype="f16", group=8, window=4096),
        # many users of a large model, 8 bits: a token's row written, its attention
        _case("step_many_8bit", "step", 256, 1, 1, 511, 4095, 8, 128, 64, True, group=8),
    ]


def draw(rng):
    def log_int(lo, hi):
        return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    op = rng.choice(["write", "write", "read", "attend", "attend", "attend", "step"])
    kv_heads, dim = rng.choice([1, 2, 3, 4, 8, 8]), rng.choice([64, 64, 80, 96, 128, 128, 128, 8 * rng.randint(1, 16)])
    page = rng.choice([16, 16, 32, 64, 64, 128, 256, 8, log_int(1, 200)])
    bits8, dtype, mix = rng.random() < 0.55, rng.choice(["bf16", "bf16", "f16"]), rng.randrange(1 << 20)
    users = log_int(1, 256)
    if op in ("attend", "step"):
        group = rng.choice([1, 2, 4, 4, 7, 8, 8, 16])
        rows = 1 if op == "step" else rng.choice([1, 1, 1, 2, log_int(2, 8)])
        keys = log_int(16, min(131072, 524288 // users))
        old = keys - rows if rng.random() < 0.5 else 0  # all of one length, or any
        window = rng.choice([0, 0, 0, log_int(16, keys)])
        c = _case("", op, users, rng.choice([0, 1, rows]), rows, old if old > 0 else -min(2, rows - 1), max(0, keys - rows),
                  kv_heads, dim, page, bits8, dtype, group, window, mix)
    else:
        most = log_int(1, min(65536, 262144 // users))
        chunk = op == "write" and rng.random() < 0.5
        old = log_int(1, most) if chunk else 0
        c = _case("", op, users, rng.choice([0, most // 4, most]), most, -min(4, old), old, kv_heads, dim, page, bits8, dtype, 0,
                  log_int(16, most) if op == "read" and most > 16 and rng.random() < 0.2 else 0, mix)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------- inputs

def _lengths(case):
    """New rows and keys of every sequence."""
    r = random.Random(case["mix"] * 7919 + case["users"])
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["users"])]
    old = [r.randint(case["old_lo"], case["old_hi"]) for _ in range(case["users"])]
    new[0], old[0] = case["new_hi"], case["old_hi"]
    return new, [max(0, n + o) for n, o in zip(new, old)]


def _first_key(case, keys):
    """The first key of `keys` whose page has not been given back."""
    return 0 if not case["window"] else max(0, keys - case["window"]) // case["page"] * case["page"]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt, g, d, page = TYPES[case["dtype"]], case["kv_heads"], case["dim"], case["page"]
    new, keys = _lengths(case)
    # every sequence has its pages and some room to grow; pages in use lie anywhere among those of the cache
    held = [-(-m // page) for m in keys]
    gone = [_first_key(case, m) // page for m in keys]
    width = max(held) + 2
    pages = sum(h - o for h, o in zip(held, gone)) + len(held) + 1
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    host, at = [], 0
    for h, o in zip(held, gone):
        host.append([-1] * o + list(range(at, at + h - o)) + [-1] * (width - h))
        at += h - o
    host = torch.tensor(host, device="cuda")
    shape = (pages, g, page, d)

    def normal(*size):
        return torch.randn(*size, generator=gen, device="cuda")

    s = {"case": dict(case), "k_scale": None, "v_scale": None}
    for name, loud in (("k", 1.0), ("v", 0.5)):
        if case["bits8"]:
            s[name + "_pages"] = normal(*shape).mul_(36).round_().clamp_(-127, 127).to(torch.int8)
            s[name + "_scale"] = torch.rand(shape[:3], generator=gen, device="cuda").add_(0.5).mul_(loud / 36)
        else:
            s[name + "_pages"] = normal(*shape).mul_(loud).to(dt)
        # the new rows stand beside each other as a projection leaves them
    s["rows"] = sum(new)
    s["row_start"] = torch.tensor([sum(new[:u]) for u in range(len(new) + 1)], dtype=torch.int32, device="cuda")
    s["key_count"] = torch.tensor(keys, dtype=torch.int32, device="cuda")
    s["table"] = torch.where(host >= 0, order[host.clamp_min(0)], -1).to(torch.int32)
    s["max_queries"], s["max_keys"] = max(new), max(keys)
    if case["op"] in ("write", "step"):
        both = normal(max(1, sum(new)), 2, g, d)
        both[:, 1] *= 0.5
        both[:, :, :, :: 16] *= 4  # some channels carry larger values
        both = both.to(dt)[:sum(new)]
        s["k"], s["v"] = both[:, 0], both[:, 1]
    if case["op"] in ("attend", "step"):
        s["q"] = normal(max(1, sum(new)), g * case["group"], d).to(dt)[:sum(new)]
    return s


# ---------------------------------------------------------------------------------------------- the operators

def run(s):
    op = s["case"]["op"]
    if own:
        from paper_2504_14611_amd import edge
        dt = TYPES[s["case"]["dtype"]]
        cache = {"k": s["k_pages"], "v": s["v_pages"], "k_scale": s["k_scale"], "v_scale": s["v_scale"]}
        where = (s["table"], s["row_start"], s["key_count"])
        r = {}
        if op in ("write", "step"):
            edge.cache_write(s["k"], s["v"], cache, *where)
        if op in ("attend", "step"):
            r["out"] = edge.attend_paged(s["q"], cache, *where, max_queries=s["max_queries"], max_keys=s["max_keys"])
        if op == "write" and not s["case"]["bits8"]:
            r["k"], r["v"] = s["k_pages"], s["v_pages"]
        elif op != "attend":  # the 8-bit rows, as the values that they stand for
            r["k"], r["v"] = edge.cache_read(cache, *where, rows=s["rows"], dtype=dt)
        return r
    r = {}
    if op in ("write", "step"):
        _write(s)
    if op in ("attend", "step"):
        r["out"] = _attend(s)
    if op == "write" and not s["case"]["bits8"]:
        r["k"], r["v"] = s["k_pages"], s["v_pages"]
    elif op != "attend":
        r["k"], r["v"] = _read(s)
    return r


def _places(s):
    """Page and slot of every row, and whether it stands anywhere."""
    start, page = s["row_start"].long(), s["case"]["page"]
    row = torch.arange(s["rows"], device=start.device)
    user = torch.searchsorted(start[1:].contiguous(), row, right=True)
    key = s["key_count"][user] - start[user + 1] + row
    at = torch.where(key >= 0, s["table"][user, key.clamp_min(0) // page].long(), -1)
    return at, key % page, at >= 0


def _write(s):
    at, slot, there = _places(s)
    at, slot = at[there], slot[there]
    for name in ("k", "v"):
        x = s[name][there]
        if s["case"]["bits8"]:
            x = x.float()
            # (a division by a number is a product with its reciprocal in 32 bits: codes next to a border would change)
            scale = (x.abs().amax(dim=2).double() / 127).float()
            s[name + "_pages"][at, :, slot] = torch.round(x / torch.where(scale > 0, scale, 1.0)[:, :, None]).to(torch.int8)
            s[name + "_scale"][at, :, slot] = scale
        else:
            s[name + "_pages"][at, :, slot] = x


def _read(s):
    at, slot, there = _places(s)
    got = []
    for name in ("k", "v"):
        x = s[name + "_pages"][at.clamp_min(0), :, slot].float()
        if s["case"]["bits8"]:
            x = x * s[name + "_scale"][at.clamp_min(0), :, slot][:, :, None]
        got.append(x.masked_fill(~there[:, None, None], 0.0).to(TYPES[s["case"]["dtype"]]))
    return got


def _attend(s):
    q, page, g = s["q"], s["case"]["page"], s["case"]["kv_heads"]
    h, d = q.shape[1:]
    users, most, longest = s["key_count"].shape[0], s["max_queries"], max(1, s["max_keys"])
    start = s["row_start"].long()
    row = torch.arange(most, device=q.device)
    col = torch.arange(longest, device=q.device)
    new = start[1:] - start[:-1]
    have = row < new[:, None]                                                     # [users, most]
    rows = torch.where(have, start[:-1, None] + row, 0)
    at = s["table"][:, col // page].long()                                        # [users, longest]
    there = (at >= 0) & (col < s["key_count"][:, None])
    at, slot = torch.where(there, at, 0), (col % page).expand(users, -1)
    kv = []
    for name in ("k", "v"):
        x = s[name + "_pages"][at, :, slot].float()                               # [users, longest, g, d]
        if s["case"]["bits8"]:
            x = x * s[name + "_scale"][at, :, slot][..., None]
        kv.append(x.permute(0, 2, 1, 3).contiguous())
    qs = q.float()[rows].reshape(users, most, g, h // g, d).permute(0, 2, 3, 1, 4).reshape(users, g, -1, d)
    sees = there[:, None] & (col < (s["key_count"][:, None] - new[:, None] + row + 1)[:, :, None])
    sees = sees[:, None, None]                                                    # [users, 1, 1, most, longest]
    p = (qs @ kv[0].transpose(2, 3).contiguous()).mul_(d ** -0.5).reshape(users, g, h // g, most, longest)
    p.masked_fill_(~sees, -math.inf)
    top = p.amax(dim=-1, keepdim=True)
    p = p.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(dim=-1, keepdim=True)
    p = p.div_(torch.where(total > 0, total, 1.0))
    o = (p.reshape(users, g, -1, longest) @ kv[1]).reshape(users, h, most, d).permute(0, 2, 1, 3)
    return o[have].to(q.dtype)


# ---------------------------------------------------------------------------------------------- what they cannot do without

def work(case):
    new, keys = _lengths(case)
    g, d, h, op = case["kv_heads"], case["dim"], case["kv_heads"] * case["group"], case["op"]
    first = [_first_key(case, m) for m in keys]
    rows16 = 4 * g * d * sum(new)                                         # keys and values as 16-bit rows
    a_key = g * (2 * d + 8) if case["bits8"] else 4 * g * d               # in the cache
    there = sum(min(n, m - f) for n, m, f in zip(new, keys, first))       # rows that stand somewhere
    bytes_, flops = 0, 0
    if op in ("write", "step"):
        bytes_ += rows16 + there * a_key
        flops += 4 * there * g * d if case["bits8"] else 0
    if op in ("read", "step") or (op == "write" and case["bits8"]):
        bytes_ += there * a_key + rows16
        flops += 2 * there * g * d if case["bits8"] else 0
    if op in ("attend", "step"):
        bytes_ += 4 * sum(new) * h * d + sum(m - f for n, m, f in zip(new, keys, first) if n) * a_key
        flops += 4 * h * d * sum(max(0, m - n + i + 1 - f) for n, m, f in zip(new, keys, first) for i in range(n))
    return {"bytes": bytes_, "flops": flops}


# ---------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    new, keys = _lengths(case)
    table, g, d, page, bits8 = s["table"].tolist(), case["kv_heads"], case["dim"], case["page"], case["bits8"]

    # the cache as rows of values: key j of user u is row table[u][j // page] * page + j % page
    def values(name):
        x = s[name + "_pages"].permute(0, 2, 1, 3).reshape(-1, g, d)
        if not bits8:
            return x.double()
        return x.double() * s[name + "_scale"].permute(0, 2, 1).reshape(-1, g).double()[:, :, None]

    def spots(u, lo, hi):
        """The rows of keys lo .. hi - 1, and which of these keys there are."""
        j = [j for j in range(lo, hi) if j >= 0 and table[u][j // page] >= 0]
        return torch.tensor([table[u][i // page] * page + i % page for i in j], dtype=torch.int64, device="cuda"), j

    def coded(x):
        """Rows as their codes and scale stand for them; the scale and the quotients are binary32 by definition."""
        x = x.double()
        scale = (x.abs().amax(dim=-1, keepdim=True) / 127).float().double()
        quotient = (x / scale.clamp_min(1e-300)).float().double()
        return torch.where(scale > 0, quotient.round() * scale, 0.0)

    cache, r, at = {name: values(name) for name in ("k", "v")}, {}, s["row_start"].tolist()
    if case["op"] in ("write", "step"):
        for u, (n, m) in enumerate(zip(new, keys)):
            rows, j = spots(u, m - n, m)
            pick = torch.tensor([at[u] + i - (m - n) for i in j], dtype=torch.int64, device="cuda")
            for name in ("k", "v"):
                x = s[name][pick]
                cache[name][rows] = coded(x) if bits8 else x.double()
    if case["op"] in ("attend", "step"):
        q, group = s["q"].double(), case["group"]
        r["out"] = torch.zeros_like(q)
        for u, (n, m) in enumerate(zip(new, keys)):
            rows, j = spots(u, 0, m)
            if not n or not j:
                continue
            kk = cache["k"][rows].permute(1, 2, 0).contiguous()            # [g, d, keys]
            vv = cache["v"][rows].permute(1, 0, 2).contiguous()            # [g, keys, d]
            j = torch.tensor(j, device="cuda")
            for i in range(n):
                score = torch.bmm(q[at[u] + i].reshape(g, group, d), kk) / math.sqrt(d)
                score = score.masked_fill(j > m - n + i, -math.inf)
                p = torch.nan_to_num(torch.softmax(score, dim=2), nan=0.0)  # (a row that sees nothing is zero)
                r["out"][at[u] + i] = torch.bmm(p, vv).reshape(g * group, d)
    if case["op"] == "write" and not bits8:
        for name in ("k", "v"):
            r[name] = cache[name].reshape(-1, page, g, d).permute(0, 2, 1, 3)
    elif case["op"] != "attend":
        for name in ("k", "v"):
            r[name] = torch.zeros(s["rows"], g, d, dtype=torch.float64, device="cuda")
            for u, (n, m) in enumerate(zip(new, keys)):
                rows, j = spots(u, m - n, m)
                r[name][torch.tensor([at[u] + i - (m - n) for i in j], dtype=torch.int64, device="cuda")] = cache[name][rows]
    return r
