"""A cache in 4 bits, slots' weights and eviction in 64 bits on the CPU, from their definitions."""
import math

import torch

from kv_reference import ancestors, half_step, place

VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EXPONENTS = {torch.float32: (-125, 125), torch.bfloat16: (-125, 125), torch.float16: (-23, 13)}


def block_of(x, dtype):
    """32 numbers -> (16 bytes, scale byte): by distances, the even code where two values are as near."""
    if not all(math.isfinite(v) for v in x):
        return [0] * 16, 255
    lo, hi = EXPONENTS[dtype]
    most, e = max(abs(v) for v in x), lo
    while e < hi and most > 7 * 2.0 ** e:
        e += 1
    codes = []
    for v in x:
        off = [(abs(abs(v) / 2.0 ** e - w), c & 1, c) for c, w in enumerate(VALUES)]
        codes.append(min(off)[2] + (8 if math.copysign(1.0, v) < 0 else 0))
    return [codes[2 * i] + 16 * codes[2 * i + 1] for i in range(16)], e + 127


def in_four(x, dtype):
    """[..., dim] -> codes [..., dim / 2], scales [..., dim / 32] uint8."""
    rows = x.double().reshape(-1, 32).tolist()
    got = [block_of(r, dtype) for r in rows]
    codes = torch.tensor([g[0] for g in got], dtype=torch.uint8).reshape(*x.shape[:-1], x.shape[-1] // 2)
    return codes, torch.tensor([g[1] for g in got], dtype=torch.uint8).reshape(*x.shape[:-1], x.shape[-1] // 32)


def values_of(codes, scales):
    """What codes and scales stand for, in 64 bits."""
    codes, scales = codes.cpu(), scales.cpu()
    table = torch.tensor(VALUES + tuple(-v for v in VALUES), dtype=torch.float64)
    x = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], -1).flatten(-2)
    unit = torch.tensor([2.0 ** (s - 127) if s < 255 else math.nan for s in range(256)], dtype=torch.float64)[scales.long()]
    return x * unit.repeat_interleave(32, -1)


def slots_seen(table, page_size, pages, length, seen_nodes):
    """[(slot, page, slot of it)] of what a row sees; `seen_nodes`: [(place behind the length, node)]."""
    capacity = len(table) * page_size
    got = [(s, place(table, page_size, pages, s)) for s in range(min(length, capacity))]
    got += [(length + i, place(table, page_size, pages, length + n)) for i, n in seen_nodes]
    return [(s, *at) for s, at in got if at is not None]


def lse_of(k_pages, table, lengths, counts, parent, q, scale):
    """[B, N, heads] logarithms of rows' sums in 64 bits, and a bound of what fp32 may be off by; NaN where there is no row.
    k_pages: [pages, page_size, heads, dim] of one layer, as numbers."""
    k_pages, q = k_pages.detach().cpu().double(), q.detach().cpu().double()
    pages, page_size, H, D = k_pages.shape
    B, N, heads, _ = q.shape
    want = torch.full((B, N, heads), math.nan, dtype=torch.float64)
    off = torch.zeros((B, N, heads), dtype=torch.float64)
    for b in range(B):
        for n in range(max(0, min(N, counts[b])) if lengths[b] >= 0 else 0):
            at = slots_seen(list(table[b]), page_size, pages, lengths[b], [(m, m) for m in sorted(ancestors(parent, n))])
            if not at:
                want[b, n] = -math.inf
                continue
            _, p, s = (torch.tensor(x) for x in zip(*at))
            for h in range(heads):
                kk = k_pages[p, s, h // (heads // H)]
                want[b, n, h] = torch.logsumexp(kk @ q[b, n, h] * scale, 0)
                size = (kk.abs() @ q[b, n, h].abs()).max() * scale
                # scores (D products summed in fp32, one multiplication), weights of an exponential, their sum, its logarithm
                # and the sum of that with the score it goes by, times ln 2
                off[b, n, h] = (D + 4) * 2.0 ** -24 * size + (len(at) + 64) * 2.0 ** -24 + 2.0 ** -21 + 2.0 ** -22 * (want[b, n, h].abs() + size)
    return want, off


def weigh(k_pages, table, lengths, counts, parent, q, lse, scale, width, paths=None):
    """[B, width] sums of weights in 64 bits and a bound for each; paths: the accepted ones, or None."""
    k_pages, q, lse = k_pages.detach().cpu().double(), q.detach().cpu().double(), lse.detach().cpu().double()
    pages, page_size, H, D = k_pages.shape
    B, N, heads, _ = q.shape
    want = torch.zeros((B, width), dtype=torch.float64)
    off = torch.zeros((B, width), dtype=torch.float64)
    for b in range(B):
        if lengths[b] < 0:
            continue
        nodes = list(range(max(0, min(N, counts[b])))) if paths is None else paths[b]
        for i, n in enumerate(nodes):
            see = [(m, m) for m in sorted(ancestors(parent, n))] if paths is None else list(enumerate(nodes[:i + 1]))
            at = [a for a in slots_seen(list(table[b]), page_size, pages, lengths[b], see) if a[0] < width]
            if not at:
                continue
            slot, p, s = (torch.tensor(x) for x in zip(*at))
            for h in range(heads):
                if lse[b, n, h] == -math.inf:
                    continue
                kk = k_pages[p, s, h // (heads // H)]
                x = kk @ q[b, n, h] * scale
                w = torch.exp(x - lse[b, n, h])
                size = kk.abs() @ q[b, n, h].abs() * scale
                # a score of D products in fp32, the sum's logarithm times log2(e) and the difference to it, an exponential
                rel = (D + 4) * 2.0 ** -24 * size + 2.0 ** -22 * lse[b, n, h].abs() + 2.0 ** -23 * x.abs() + 2.0 ** -22
                want[b].index_add_(0, slot, w)
                off[b].index_add_(0, slot, w * (rel + (N * heads + 20) * 2.0 ** -24))
    return want, off + 1e-30


def kept_of(weights, length, budget, first, recent):
    """The slots that a sequence keeps, in order."""
    if length <= budget:
        return list(range(max(length, 0)))

    def weight(s):
        w = weights[s] if s < len(weights) else 0.0
        return -math.inf if math.isnan(w) else w, not (s < len(weights) and math.isnan(weights[s]))
    middle = sorted(range(first, length - recent), key=lambda s: (tuple(-x for x in weight(s)), s))
    return list(range(first)) + sorted(middle[:budget - first - recent]) + list(range(length - recent, length))
