"""The key-value cache calls in 64 bits on the CPU, loop by loop from their definitions, and the makers of small cases."""
import math

import torch

SPINE = (1, 3, -1, 5, -1, 7, -1, -1, -1)
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def parents(k, N, table=None):
    """Parent of every node, -1 for roots, by the rule of first_child tables."""
    parent = [-1] * N
    for n in range(N):
        c = k * n + 1 if table is None else table[n]
        if c > n and c + k <= N:
            for j in range(k):
                parent[c + j] = max(parent[c + j], n)
    return parent


def levels(parent):
    out = []
    for p in parent:
        out.append(out[p] + 1 if p >= 0 else 0)
    return out


def ancestors(parent, n):
    got = set()
    while n >= 0:
        got.add(n)
        n = parent[n]
    return got


def place(table, page_size, pages, s):
    """(page, slot) of a sequence's slot s, None if it has no page."""
    e = s // page_size
    if s < 0 or e >= len(table) or not 0 <= table[e] < pages:
        return None
    return table[e], s % page_size


def attention(k_pages, v_pages, table, lengths, counts, parent, q, scale, shared=0, shared_pages=None):
    """[B, N, heads, dim] results in 64 bits, and a bound of what fp32 sums and rounded weights may be off by; None rows
    (not to be written) hold NaN in both.  k_pages: [pages, page_size, heads, dim] of one layer."""
    k_pages, v_pages, q = (x.detach().cpu() for x in (k_pages, v_pages, q))
    dtype = q.dtype
    pages, page_size, H, D = k_pages.shape
    B, N, heads, _ = q.shape
    G = heads // H
    out = torch.full((B, N, heads, D), math.nan, dtype=torch.float64)
    off = torch.zeros((B, N, heads, D), dtype=torch.float64)
    u_weight = half_step(dtype) if dtype != torch.float32 else 0.0
    for b in range(B):
        if lengths[b] < 0:
            continue
        c = max(0, min(N, counts[b]))
        row = list(table[b])
        prefix = min(shared, lengths[b])
        for n in range(c):
            at = []
            capacity = len(row) * page_size
            for s in range(min(lengths[b], capacity)):
                own = list(shared_pages) if s < prefix else row
                at.append(place(own, page_size, pages, s))
            at += [place(row, page_size, pages, lengths[b] + m) for m in sorted(ancestors(parent, n))]
            at = [a for a in at if a is not None]
            if not at:
                out[b, n] = 0.0
                continue
            p, s = (torch.tensor(x) for x in zip(*at))
            for h in range(heads):
                kk, vv = k_pages[p, s, h // G].double(), v_pages[p, s, h // G].double()
                x = kk @ q[b, n, h].double() * scale
                w = torch.softmax(x, 0)
                # a weight is positive, however small: infinities and NaNs of the values come through even where
                # the 64-bit exponential is zero (scores more than 745 below the largest), which would make 0 * inf = NaN
                plain = torch.where(torch.isfinite(vv), vv, 0.0)
                out[b, n, h] = w @ plain + torch.where(torch.isfinite(vv), 0.0, vv).sum(0)
                spread = w @ plain.abs()
                # scores: D products summed in fp32, one multiplication, one exponential of about an ulp, twice (the
                # weight and the sum it is divided by); sums of len(at) terms, rescaled once a tile; weights rounded once
                size = (kk.abs() @ q[b, n, h].double().abs()).max() * scale
                rel = 2 * ((D + 4) * 2.0 ** -24 * size + 2.0 ** -22) + (len(at) + 64) * 2.0 ** -24 + u_weight
                if dtype == torch.float16:  # weights below the normal range: half a step of 2^-24, the largest being 2^7
                    off[b, n, h] += w.max() * plain.abs().sum(0) * 2.0 ** -32
                off[b, n, h] += spread * rel + (half_step(dtype) + 2.0 ** -22) * out[b, n, h].abs() + 1e-30
    if dtype == torch.float16:
        off += 2.0 ** -24  # numbers below fp16's normal range
    return out, off


def rotated(x, t, inv_freq, neighbours):
    """One head's vector (64 bits) at position t."""
    y = x.clone()
    half = len(inv_freq)
    for i in range(half):
        a = t * float(inv_freq[i])
        c, s = math.cos(a), math.sin(a)
        i0, i1 = (2 * i, 2 * i + 1) if neighbours else (i, i + half)
        y[..., i0] = x[..., i0] * c - x[..., i1] * s
        y[..., i1] = x[..., i0] * s + x[..., i1] * c
    return y


def path_of(outcome, accept_depth, depth, k, N, count, table=None):
    if count == 0:
        return []
    node, path = 0, [0]
    while len(path) <= min(accept_depth, depth - 1):
        c = k * node + 1 if table is None else table[node]
        if not 0 <= outcome[node] < k or c <= node or c + k > N or c + outcome[node] >= count:
            break
        node = c + outcome[node]
        path.append(node)
    return path


def make_pages(lengths, N, page_size, *, layers=1, heads=2, dim=64, dtype=torch.float32, order="slots", spare=2,
               shared=0, seed=0, device="cuda", used=True):
    """Pools full of NaN but for the slots in use (those of the nodes too, where `used`), and the sequences' tables.
    The first shared // page_size pages are common to all."""
    gen = torch.Generator().manual_seed(seed)
    B = len(lengths)
    common = shared // page_size
    need = [max(common, -(-(max(n, 0) + N) // page_size)) for n in lengths]
    pages = common + sum(n - common for n in need) + spare
    mixed = torch.randperm(pages, generator=gen).tolist()
    first, rest = mixed[:common], mixed[common:]
    table = []
    for n in need:
        table.append(first + [rest.pop() for _ in range(n - common)])
    width = max(need) + 1
    shape = (layers, pages, page_size, heads, dim) if order == "slots" else (layers, pages, heads, page_size, dim)
    pools = []
    for _ in range(2):
        pool = torch.full(shape, math.nan, dtype=dtype, device=device)
        pool = pool if order == "slots" else pool.transpose(2, 3)
        values = torch.randn((layers, pages, page_size, heads, dim), generator=gen).to(dtype).to(device)
        for b, n in enumerate(lengths):
            for s in range(max(n, 0) + (N if used else 0)):
                p = table[b][s // page_size]
                pool[:, p, s % page_size] = values[:, p, s % page_size]
        pools.append(pool)
    filled = torch.tensor([t + [-7] * (width - len(t)) for t in table], dtype=torch.int32, device=device)
    return pools[0], pools[1], filled, table
