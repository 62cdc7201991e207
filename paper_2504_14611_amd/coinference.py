"""Co-inference of a decoder chain, planned and carried out: `python -m paper_2504_14611_amd.coinference`.

The chain's sub-tasks are decoder blocks that all users share, each user with a low-rank adapter of their own.
The planner (jdob.solve_batch) takes the latency of a batch of b users on the edge GPU as alpha_l + beta_l * b per
sub-task; here the edge operators (edge.norm, edge.project, edge.attend) are that latency and the carrying out:

1. `profile` times the blocks on this GPU for batches of users and fits alpha and beta of one,
2. `instance` puts them with the devices, uplinks and deadlines into a problem, which jdob.solve_batch decides:
   the partition point s, the GPU level, and which users offload,
3. `Edge` computes blocks s+1..L for the offloaded users' rows in one batch, all users' rows packed one after the
   other, and keeps their keys and values, so that it can go on with single tokens: in a slab a user, or on pages that
   all users share, 16-bit or in 8 bits (edge.cache_write, edge.cache_read, edge.attend_paged).

A block:  h += x;  q, k, v = norm(h) Wqkv;  x = attend(q, k, v) Wo;  h += x;  x = gelu(norm(h) Wup) Wdown.
Wqkv and Wup take the norm's 8-bit rows and have 8-bit weights; Wo and Wdown are 16-bit.  Weights and rows are
random (synthetic); the devices' share of the chain is computed with the same operators, one user at a time.
"""

from __future__ import annotations

import argparse
import dataclasses
import itertools
import time
from typing import Dict, List, Optional, Sequence

import numpy as np

from . import edge, jdob


@dataclasses.dataclass(frozen=True)
class Shape:
    blocks: int = 8
    width: int = 2048
    heads: int = 16
    kv_heads: int = 4
    inner: int = 8192      # of the block's second half
    rank: int = 16         # of the users' adapters

    @property
    def head_dim(self) -> int:
        return self.width // self.heads

    @property
    def qkv(self) -> int:
        return (self.heads + 2 * self.kv_heads) * self.head_dim

    def multiplications(self, tokens: int) -> float:
        """Of one block for one user's prompt (the causal half of the attention)."""
        per_row = self.width * (self.qkv + self.width + 2 * self.inner)
        return float(tokens) * per_row + float(tokens) * (tokens + 1) * self.width


def make_chain(shape: Shape, users: int, device="cuda", seed: int = 0) -> List[dict]:
    """Random weights of every block: 16-bit matrices, 8-bit ones with a scale a row, adapters of all users."""
    import torch
    gen = torch.Generator(device=device).manual_seed(seed)

    def normal(*size, scale=1.0):
        return torch.randn(*size, generator=gen, device=device).mul_(scale)

    def wide(out, inner, bits8):
        w = normal(out, inner, scale=inner ** -0.5)
        if not bits8:
            return {"weight": w.bfloat16()}
        scale = w.abs().amax(dim=1) / 127
        return {"weight": torch.round(w / scale[:, None]).to(torch.int8), "weight_scale": scale}

    def adapters(out, inner):
        return {"down": normal(users, shape.rank, inner, scale=inner ** -0.5).bfloat16(),
                "up": normal(users, out, shape.rank, scale=0.25 * shape.rank ** -0.5).bfloat16(),
                "gain": torch.ones(users, device=device)}

    sizes = {"qkv": (shape.qkv, shape.width, True), "o": (shape.width, shape.width, False),
             "up": (shape.inner, shape.width, True), "down": (shape.width, shape.inner, False)}
    return [{"first": (1 + normal(shape.width, scale=0.1)).bfloat16(),
             "second": (1 + normal(shape.width, scale=0.1)).bfloat16(),
             **{name: {**wide(*size), "adapters": adapters(*size[:2])} for name, size in sizes.items()}}
            for _ in range(shape.blocks)]


class Edge:
    """Blocks first..L of the chain for a batch of users, with their keys and values.

    Every user has a slab of `room` rows in each block's cache; new keys and values are written behind those that
    stand there already.  With `page` the cache is made of `pages` pages of so many keys (default: as many as all users
    may fill), which users take as they grow; it holds 8-bit rows with bits8, and then all rows attend to what the cache
    stands for, their own and the other new ones' keys and values among it.  Users with up to FEW new rows attend over the
    pages as they are, the others to rows that are read back, each user for itself: what a user's rows see does not depend on
    who else is in the batch."""

    FEW = 8

    def __init__(self, shape: Shape, chain: Sequence[dict], users: Sequence[int], first: int, room: int, device="cuda",
                 page: int = 0, bits8: bool = False, pages: Optional[int] = None):
        import torch
        self.shape, self.chain, self.users, self.device = shape, list(chain[first:]), list(users), device
        self.room, self.count, self.page, self.bits8 = room, [0] * len(self.users), page, bits8
        if page < 0:
            raise ValueError(f"pages of {page} keys")
        if page:
            each = -(-room // page)
            pages = len(self.users) * each if pages is None else pages
            self.free, self.held = list(range(pages))[::-1], [[] for _ in self.users]
            self.cache = [edge.make_cache(pages, page, shape.kv_heads, shape.head_dim, bits8=bits8, device=device)
                          for _ in self.chain]
            return
        if bits8 or pages is not None:
            raise ValueError("slabs are 16-bit and have no pages")
        n = len(self.users) * room
        self.cache = [torch.zeros((n, 2, shape.kv_heads, shape.head_dim), dtype=torch.bfloat16, device=device)
                      for _ in self.chain]

    def _take_pages(self, counts: Sequence[int]):
        """Pages for so many keys of every user (the same ones in all blocks), and the table of all users' pages."""
        import torch
        need = [-(-m // self.page) - len(held) for m, held in zip(counts, self.held)]
        if sum(max(0, n) for n in need) > len(self.free):
            raise ValueError(f"the cache has {len(self.free)} pages left")
        for n, held in zip(need, self.held):
            held += [self.free.pop() for _ in range(n)]
        width = max(map(len, self.held), default=0)
        return torch.tensor([held + [-1] * (width - len(held)) for held in self.held], dtype=torch.int32,
                            device=self.device).view(len(self.users), width)

    def _plan(self, lengths: Sequence[int], counts: Sequence[int]) -> dict:
        """Where the new rows go, and for the users with few and with many of them: their rows (None: all there are),
        tables, starts of their rows and of all their keys."""
        import torch

        def on_device(x, dtype=torch.int32):
            return torch.tensor(x, dtype=dtype, device=self.device)

        def starts(x):
            return [0, *itertools.accumulate(x)]

        table, first, groups = self._take_pages(counts), starts(lengths), []
        query_start, key_count = on_device(first), on_device(counts)
        for few in (True, False):
            users = [u for u, m in enumerate(lengths) if m and (m <= self.FEW) == few]
            if not users:
                continue
            new, keys = [lengths[u] for u in users], [counts[u] for u in users]
            g = {"rows": None, "table": table, "query_start": query_start, "key_count": key_count}
            if sum(new) < first[-1]:
                g["rows"] = on_device([first[u] + i for u in users for i in range(lengths[u])], torch.int64)
            if len(users) < len(lengths):
                g.update(table=table[on_device(users, torch.int64)], query_start=on_device(starts(new)), key_count=on_device(keys))
            key_start = None if few else on_device(starts(keys))
            # (rows without a history are read back as they are out of 16 bits)
            groups.append({**g, "few": few, "read": not few and (self.bits8 or new != keys), "key_start": key_start,
                           "most": max(new), "longest": max(keys), "keys": sum(keys)})
        return {"table": table, "query_start": query_start, "key_count": key_count, "groups": groups}

    def _attend_pages(self, q, k, v, cache, plan):
        """The rows' keys and values into the cache, and their attention."""
        import torch
        edge.cache_write(k, v, cache, plan["table"], plan["query_start"], plan["key_count"])
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if len(plan["groups"]) > 1 else None
        for g in plan["groups"]:
            rows, where = g["rows"], (g["table"], g["query_start"], g["key_count"])
            qg = q if rows is None else q[rows]
            most = {"max_queries": g["most"], "max_keys": g["longest"]}
            if g["few"]:
                y = edge.attend_paged(qg, cache, *where, **most)
            else:
                if g["read"]:
                    kg, vg = edge.cache_read(cache, g["table"], g["key_start"], g["key_count"], rows=g["keys"], dtype=q.dtype)
                else:
                    kg, vg = (k, v) if rows is None else (k[rows], v[rows])
                y = edge.attend(qg, kg, vg, g["query_start"], g["key_start"][:-1].long(), g["key_count"], **most)
            if out is None:
                return y
            out[rows] = y
        return torch.empty(q.shape, dtype=q.dtype, device=q.device) if out is None else out

    def run(self, rows, lengths: Sequence[int]):
        """`rows` [sum of lengths, width]: each user's new rows behind each other, as they enter the first block.
        Returns the rows that leave the last one."""
        import torch
        import torch.nn.functional as F
        s, dev, n = self.shape, self.device, len(self.users)
        if len(lengths) != n or sum(lengths) != rows.shape[0]:
            raise ValueError("a length for every user, and a row for each")
        if any(c + m > self.room for c, m in zip(self.count, lengths)):
            raise ValueError(f"the cache has room for {self.room} rows a user")
        if not self.chain:
            return rows
        counts = [c + m for c, m in zip(self.count, lengths)]
        row_adapter = torch.tensor(np.repeat(np.asarray(self.users, dtype=np.int32), lengths), device=dev)
        if self.page:
            plan = self._plan(lengths, counts)
        else:
            query_start = torch.tensor([0, *itertools.accumulate(lengths)], dtype=torch.int32, device=dev)
            key_start = torch.arange(n, device=dev) * self.room
            key_count = torch.tensor(counts, dtype=torch.int32, device=dev)
            slots = torch.tensor(np.concatenate([u * self.room + c + np.arange(m) for u, (c, m) in
                                                 enumerate(zip(self.count, lengths))]).astype(np.int64), device=dev)

        def project(part, x, scale=None):
            return edge.project(x, part["weight"], x_scale=scale, weight_scale=part.get("weight_scale"),
                                adapters=part["adapters"], row_adapter=row_adapter)

        h, x = rows, None
        for block, cache in zip(self.chain, self.cache):
            r = edge.norm(h if x is None else x, block["first"], residual=None if x is None else h, bits8=True)
            h = h if x is None else r["sum"]
            qkv = project(block["qkv"], r["q"], r["scale"]).view(-1, s.heads + 2 * s.kv_heads, s.head_dim)
            if self.page:
                y = self._attend_pages(qkv[:, :s.heads], qkv[:, s.heads:s.heads + s.kv_heads], qkv[:, s.heads + s.kv_heads:],
                                       cache, plan)
            else:
                cache[slots] = qkv[:, s.heads:].reshape(-1, 2, s.kv_heads, s.head_dim)
                y = edge.attend(qkv[:, :s.heads], cache[:, 0], cache[:, 1], query_start, key_start, key_count,
                                max_queries=max(lengths), max_keys=max(counts))
            r = edge.norm(project(block["o"], y.view(-1, s.width)), block["second"], residual=h, bits8=True)
            h = r["sum"]
            x = project(block["down"], F.gelu(project(block["up"], r["q"], r["scale"])))
        self.count = counts
        return h if x is None else h + x


def fit(batches: Sequence[int], seconds: Sequence[float]) -> tuple:
    """alpha, beta >= 0 of the least squares of alpha + beta * b."""
    b, t = np.asarray(batches, dtype=np.float64), np.asarray(seconds, dtype=np.float64)
    beta = max(0.0, float(np.sum((b - b.mean()) * (t - t.mean())) / max(np.sum((b - b.mean()) ** 2), 1e-30)))
    return max(0.0, float(t.mean() - beta * b.mean())), beta


def profile(shape: Shape, chain: Sequence[dict], users: int, tokens: int, repeats: int = 5, device="cuda") -> tuple:
    """alpha, beta in seconds of one block for b users' prompts of `tokens` rows, timed on this GPU: the whole chain's
    time over its blocks, as a batch brings its index arrays to the GPU once and not for every block."""
    import torch
    batches = sorted({1, *[max(1, users * k // 4) for k in (1, 2, 3, 4)]})
    seconds = []
    for b in batches:
        rows = torch.randn(b * tokens, shape.width, device=device).bfloat16()
        times = []
        for _ in range(repeats + 2):
            e = Edge(shape, chain, list(range(b)), 0, tokens, device)
            torch.cuda.synchronize()
            t = time.perf_counter()
            e.run(rows, [tokens] * b)
            torch.cuda.synchronize()
            times.append(time.perf_counter() - t)
        seconds.append(sorted(times[2:])[repeats // 2] / len(chain))
    return fit(batches, seconds)


def instance(shape: Shape, users: int, tokens: int, alpha: float, beta: float, seed: int = 0) -> Dict[str, object]:
    """The planning problem: `users` devices with a prompt of `tokens` rows each before the chain's blocks, on the
    edge GPU whose top level is the one that alpha and beta were timed at.

    Devices do 4 multiplications a cycle, from 0.5 to 2 GHz; the rows between two blocks are 16-bit, the prompt is
    16 bits a token; uplinks of 50 to 500 Mbit/s; deadlines of 1.2 to 4 times the chain's local latency."""
    r = np.random.RandomState(seed)
    L, cycles = shape.blocks, shape.multiplications(tokens) / 4
    bits = np.full((1, L + 1), tokens * shape.width * 16.0, dtype=np.float32)
    bits[0, 0] = tokens * 16.0
    f = np.linspace(0.5e9, 2.0e9, 8, dtype=np.float32)
    local = L * cycles / float(f[-1])
    return {"N": users, "L": L, "K": 8, "J": 8, "dtype": "f32", "mode": 0,
            "cycles": np.full((1, L), cycles, dtype=np.float32), "bits": bits,
            "alpha": np.full((1, L), alpha, dtype=np.float32), "beta": np.full((1, L), beta, dtype=np.float32),
            "rate": r.uniform(5e7, 5e8, (1, users)).astype(np.float32),
            "deadline": (local * r.uniform(1.2, 4.0, (1, users))).astype(np.float32),
            "t_free": np.zeros(1, dtype=np.float32), "local_freq": f,
            "gpu_freq": np.linspace(0.8e9, 2.0e9, 8, dtype=np.float32),
            "kappa": 2.25e-26, "p_tx": 0.5, "gpu_c": 3.125e-26, "gpu_p_static": 50.0}


def carry_out(shape: Shape, chain: Sequence[dict], cut: int, offloaders: Sequence[int], rows: dict, more: int = 0,
              device="cuda", page: int = 0, bits8: bool = False):
    """The offloaders' prompts (`rows`: user -> [tokens, width]) through the chain: blocks 1..cut each on their own
    device, the others in one batch on the edge, then `more` further single rows a user the same way, each the row
    that left the last block before it.  `page` and `bits8` are the edge's cache.  Returns user -> the rows that left
    the last block."""
    import torch
    lengths = [rows[u].shape[0] for u in offloaders]
    devices = [Edge(shape, chain[:cut], [u], 0, n + more, device) for u, n in zip(offloaders, lengths)]
    e = Edge(shape, chain, offloaders, cut, max(lengths) + more, device, page, bits8,
             sum(-(-(n + more) // page) for n in lengths) if page else None)

    def through(entering):
        sent = [d.run(x, [x.shape[0]]) for d, x in zip(devices, entering)]
        new = [x.shape[0] for x in sent]
        return e.run(torch.cat(sent), new).split(new)

    out = [through([rows[u] for u in offloaders])]
    for _ in range(more):
        out.append(through([x[-1:] for x in out[-1]]))
    return {u: torch.cat(parts) for u, parts in zip(offloaders, zip(*out))}


def main(argv=None) -> Dict[str, object]:
    import torch
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--users", type=int, default=16)
    p.add_argument("--tokens", type=int, default=256, help="of the longest prompt")
    p.add_argument("--more", type=int, default=8, help="single tokens after the prompts")
    p.add_argument("--page", type=int, default=0, help="keys on a page of the edge's cache (0: a slab a user)")
    p.add_argument("--cache-bits", type=int, choices=(8, 16), default=16, help="of the keys and values on its pages")
    for field in dataclasses.fields(Shape):
        p.add_argument("--" + field.name.replace("_", "-"), type=int, default=field.default)
    a = p.parse_args(argv)
    if not 0 <= a.page <= edge.MAX_PAGE_SIZE:
        p.error(f"--page: 0 to {edge.MAX_PAGE_SIZE} keys")
    if a.cache_bits == 8 and not a.page:
        p.error("--cache-bits 8: 8-bit keys and values stand on pages (--page)")
    shape = Shape(*[getattr(a, field.name) for field in dataclasses.fields(Shape)])
    chain = make_chain(shape, a.users)
    alpha, beta = profile(shape, chain, a.users, a.tokens)
    print(f"a block on this GPU: {alpha * 1e6:.1f} us + {beta * 1e6:.2f} us a user ({a.tokens} tokens)")
    prob = instance(shape, a.users, a.tokens, alpha, beta)
    policy = jdob.to_host(jdob.solve_batch(jdob.to_device(prob)))
    if policy["status"][0]:
        print("no feasible policy")
        return {"alpha": alpha, "beta": beta, "policy": policy}
    cut = int(policy["cut"][0])
    offloaders = [int(u) for u in np.flatnonzero(policy["user_offload"][0])]
    print(f"policy: {len(offloaders)} of {a.users} users offload after block {cut} of {shape.blocks}, GPU level "
          f"{int(policy['gpu_level'][0])}, {float(policy['energy'][0]):.4g} J")
    out = {}
    if offloaders:
        r = np.random.RandomState(1)
        rows = {u: torch.randn(int(r.randint(max(1, a.tokens // 4), a.tokens + 1)), shape.width, device="cuda").bfloat16()
                for u in offloaders}
        kept = {"page": a.page, "bits8": a.cache_bits == 8}
        carry_out(shape, chain, cut, offloaders, rows, 1, **kept)
        torch.cuda.synchronize()
        t = time.perf_counter()
        out = carry_out(shape, chain, cut, offloaders, rows, a.more, **kept)
        torch.cuda.synchronize()
        t = time.perf_counter() - t
        print(f"carried out: {sum(map(len, rows.values()))} rows and {a.more} further ones a user in {t * 1e3:.2f} ms; "
              f"all finite: {all(bool(torch.isfinite(o).all()) for o in out.values())}")
    return {"alpha": alpha, "beta": beta, "policy": policy, "out": out}


if __name__ == "__main__":
    main()
