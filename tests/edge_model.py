"""The edge operators in 64 bits, from their definitions, and how far a kernel's output may be from them.

Bounds follow from the roundings that include/jdob_edge.h states: inputs are taken as they are, sums are binary32
(unit roundoff 2^-24 a step; a factor of two for products that are summed in an order and with roundings of the
matrix units' own), and the output is rounded once to its type (UNIT).
"""

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
LEAST = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -149}  # smallest subnormals
U32 = 2.0 ** -24


def norm(x, weight, eps, residual=None):
    """h and y."""
    h = x.double() + (0 if residual is None else residual.double())
    return h, h * weight.double() / torch.sqrt((h * h).mean(dim=1, keepdim=True) + eps)


def norm_bound(y, dtype):
    # h, its square, at most 64 terms a thread and 10 steps between threads, division, root, two products
    return y.abs() * (UNIT[dtype] + 90 * U32) + LEAST[dtype]


def project(x, weight, x_scale=None, weight_scale=None, adapters=None, row_adapter=None):
    """y, the sums of absolute values of the shared part's and of the low-rank part's products."""
    x, w = x.double(), weight.double()
    if x_scale is not None:
        x, w = x * x_scale.double()[:, None], w * weight_scale.double()[:, None]
    y, s = x @ w.T, x.abs() @ w.abs().T
    low = torch.zeros_like(y)
    if adapters is not None:
        n, most = adapters["down"].shape[:2]
        rank = adapters["rank"].tolist() if adapters.get("rank") is not None else [most] * n
        for a in range(n):
            rows = (row_adapter == a).nonzero()[:, 0]
            r = max(0, min(most, rank[a]))
            d, u, g = adapters["down"][a, :r].double(), adapters["up"][a, :, :r].double(), adapters["gain"][a].double()
            y[rows] += g * ((x[rows] @ d.T) @ u.T)
            low[rows] += g.abs() * ((x[rows].abs() @ d.abs().T) @ u.abs().T)
    return y, s, low


def project_bound(y, s, low, in_dim, rank, dtype):
    # the low-rank rows as two 16-bit parts: what is left of either is at most UNIT squared
    return (y.abs() * UNIT[dtype] + s * (2 * in_dim + 8) * U32 +
            low * (2 * (in_dim + rank + 16) * U32 + 2 * UNIT[dtype] ** 2) + LEAST[dtype])


def attend(q, k, v, query_start, key_start, key_count, scale):
    """out, the weighted sums of |v|, and the scores' sums of absolute products (largest of a row)."""
    h, g = q.shape[1], k.shape[1]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    size, spread = torch.zeros_like(out), torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    at, first, count = query_start.tolist(), key_start.tolist(), key_count.tolist()
    for u in range(len(count)):
        n, m = at[u + 1] - at[u], count[u]
        for i in range(n):
            sees = m - n + i + 1
            if sees <= 0:
                continue
            for head in range(h):
                kk = k[first[u]:first[u] + sees, head * g // h].double()
                vv = v[first[u]:first[u] + sees, head * g // h].double()
                qq = q[at[u] + i, head].double()
                p = torch.softmax(scale * (kk @ qq), dim=0)
                out[at[u] + i, head] = p @ vv
                size[at[u] + i, head] = p @ vv.abs()
                spread[at[u] + i, head] = abs(scale) * (kk.abs() @ qq.abs()).max()
    return out, size, spread


def attend_bound(out, size, spread, dim, keys, dtype):
    # a score is off by (2 dim + 4) roundings of its products' sum and the exponential by as much again, relative;
    # p is rounded to the type, once in the numerator only
    off = 2 * (2 * dim + 8) * U32 * spread[..., None] + (2 * keys + 64) * U32
    return out.abs() * (UNIT[dtype] + off) + size * (UNIT[dtype] + off) + LEAST[dtype] * 4
