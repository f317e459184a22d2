"""The key-value cache of token trees, measured: appending, attending and committing.

One step of a decoder that verifies token trees runs the target model over the nodes of each tree.  Its
attention layers put the nodes' keys and values behind the sequence's in a paged cache, rotated to the
nodes' positions (`append`); every node attends to the sequence and to its ancestors (`attend`); and once
the trees are verified, the keys and values of the accepted path stay and the others go (`commit`).  A
prompt is a tree of one branch, a single token a tree of one node.
"""
import math

import torch

own = False

# First children of a tree of nine nodes: a left spine, as a tree search over acceptance rates gives it.
SPINE = (1, 3, -1, 5, -1, 7, -1, -1, -1)


def _case(name, op, B, tree, k, depth, heads, kv_heads, dim, lo, hi, dtype, *, page=64, order="slots", layers=1,
          shared=0, counts="full", rot=0, pairs="halves"):
    return dict(name=name, op=op, B=B, tree=tree, k=k, depth=depth, heads=heads, kv_heads=kv_heads, dim=dim, lo=lo,
                hi=hi, dtype=dtype, page=page, order=order, layers=layers, shared=shared, counts=counts,
                rot=rot or dim, pairs=pairs)


def listed():
    return [
        # one user far into a conversation, a 15-node tree in fp32: nothing but latency
        _case("append_one_sequence", "append", 1, "complete", 2, 4, 8, 8, 64, 90000, 90000, "fp32", page=16),
        # a serving batch: 64 sequences of all lengths, 31-node trees
        _case("append_serving", "append", 64, "complete", 2, 5, 32, 8, 128, 512, 4096, "bf16"),
        # prompts of different lengths, padded to the longest; half of each head is rotated, pair by pair
        _case("append_prompts", "append", 8, "chain", 1, 4096, 32, 8, 128, 0, 1024, "fp16", order="heads",
              counts="ragged", rot=64, pairs="neighbours"),
        # one token of one user
        _case("attend_token", "attend", 1, "chain", 1, 1, 32, 8, 128, 8192, 8192, "bf16"),
        # a batch that decodes token by token: bandwidth
        _case("attend_tokens", "attend", 64, "chain", 1, 1, 32, 8, 128, 512, 8192, "bf16", order="heads"),
        # a serving batch of 31-node trees: 124 rows for every key
        _case("attend_serving", "attend", 64, "complete", 2, 5, 32, 8, 128, 512, 4096, "bf16"),
        # two users with book-length contexts
        _case("attend_long", "attend", 2, "complete", 2, 4, 32, 8, 128, 100001, 131072, "bf16", page=16),
        # 64 requests behind one long system prompt
        _case("attend_shared_prefix", "attend", 64, "complete", 2, 4, 32, 8, 128, 1, 1024, "fp16", shared=16384),
        # prompts, some of them in their second part: causal attention, the largest amount of work
        _case("attend_prompts", "attend", 4, "chain", 1, 4096, 32, 8, 128, 0, 1024, "bf16", counts="ragged"),
        # fp32, a tree of its own shape, heads of 80, a page that is no power of two
        _case("attend_odd", "attend", 48, "spine", 2, 5, 12, 12, 80, 1, 2000, "fp32", page=48),
        # the serving batch after its trees are verified, all layers at once
        _case("commit_serving", "commit", 64, "complete", 2, 5, 32, 8, 128, 16, 128, "bf16", page=16, layers=32),
        # one user's cache
        _case("commit_one_sequence", "commit", 1, "complete", 2, 4, 32, 8, 128, 777, 777, "fp16", page=16, layers=32),
    ]


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "commit"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    dim = rng.choice([64, 128, 128, 128, 80, 96, 192, 256])
    kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
    heads = kv_heads * rng.choice([1, 2, 4, 4, 8])
    kind = rng.choice(["complete", "complete", "spine", "token", "chain"])
    if op == "commit" and kind in ("token", "chain"):
        kind = "complete"
    tree, k, depth = "complete", 2, rng.randint(2, 5)
    if kind == "spine":
        tree, depth = "spine", 5
    elif kind == "token":
        tree, k, depth = "chain", 1, 1
    elif kind == "chain":
        tree, k, depth = "chain", 1, _between(rng, 2, 4096)
    elif rng.random() < 0.3:
        k, depth = rng.choice([3, 4]), rng.choice([2, 3])
    N = _nodes(dict(tree=tree, k=k, depth=depth))
    # lengths and batch within what the largest listed cases take
    layers = rng.choice([1, 4, 16]) if op == "commit" else 1
    hi = _between(rng, 1, 131072 if op == "attend" and N <= 64 else 4096)
    if op == "append" and rng.random() < 0.3:
        hi = _between(rng, 4096, 200000)
    per_sequence = layers * kv_heads * dim * (hi + N)
    most = min(2.0e8 / per_sequence, 4.0e8 / (heads * N * (hi + N)) if op == "attend" else 2.0e8 / (heads * N * dim), 256)
    B = _between(rng, 1, max(1.0, most))
    shared = 0
    page = rng.choice([16, 16, 32, 64, 64, 128, 24, 1])
    if op == "attend" and hi > 64 and rng.random() < 0.3:
        shared = _between(rng, 32, hi) // page * page
    lo = rng.choice([0, hi // 2, hi])
    return dict(op=op, B=B, tree=tree, k=k, depth=depth, heads=heads, kv_heads=kv_heads, dim=dim,
                lo=max(0, lo - shared), hi=max(1, hi - shared), dtype=dtype, page=page,
                order=rng.choice(["slots", "heads"]), layers=layers, shared=shared,
                counts="ragged" if rng.random() < 0.3 and op != "commit" else "full",
                rot=rng.choice([dim, dim, dim // 2]), pairs=rng.choice(["halves", "neighbours"]))


def _nodes(case):
    if case["tree"] == "spine":
        return len(SPINE)
    k, depth = case["k"], case["depth"]
    return depth if k == 1 else (k ** depth - 1) // (k - 1)


def _parents(case):
    N, k = _nodes(case), case["k"]
    if case["tree"] != "spine":
        return [(n - 1) // k if n else -1 for n in range(N)]
    parent = [-1] * N
    for n, c in enumerate(SPINE):
        for j in range(k if c >= 0 else 0):
            parent[c + j] = n
    return parent


def _depths(case):
    parent, depth = _parents(case), []
    for p in parent:
        depth.append(depth[p] + 1 if p >= 0 else 0)
    return depth


def _spread(lo, hi, B):
    """B whole numbers from lo to hi in equal steps (a batch of one has the last)."""
    return [hi if B == 1 else lo + (hi - lo) * b // (B - 1) for b in range(B)]


def _lengths(case):
    return [case["shared"] + x for x in _spread(case["lo"], case["hi"], case["B"])]


def _counts(case):
    N = _nodes(case)
    return _spread(max(1, N // 4), N, case["B"]) if case["counts"] == "ragged" else [N] * case["B"]


def _accepted(case):
    """Accepted drafts of each sequence: every number that the tree allows, in turn."""
    return [b % case["depth"] if case["B"] > 1 else case["depth"] - 1 for b in range(case["B"])]


TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    on_host = torch.Generator().manual_seed(seed)
    B, N, page, layers = case["B"], _nodes(case), case["page"], case["layers"]
    H, G, D, dtype = case["kv_heads"], case["heads"] // case["kv_heads"], case["dim"], TYPES[case["dtype"]]
    mixed = torch.randperm(B, generator=on_host)
    lengths = torch.tensor(_lengths(case))[mixed]
    counts = torch.tensor(_counts(case))[mixed]

    # pages of a pool in no order; the shared ones stand first in every sequence's list
    common = case["shared"] // page
    need = (lengths + N + page - 1) // page
    listed_pages = int(need.max())
    pages = common + int((need - common).sum())
    order = torch.randperm(pages, generator=on_host)
    table = torch.full((B, listed_pages), -1, dtype=torch.int32)
    table[:, :common] = order[:common].to(torch.int32)
    place = torch.arange(listed_pages)[None, :]
    table[(place >= common) & (place < need[:, None])] = order[common:].to(torch.int32)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)

    def pool():
        if case["order"] == "slots":
            return normal(layers, pages, page, H, D)
        return normal(layers, pages, H, page, D).transpose(2, 3)

    first = torch.tensor(SPINE, dtype=torch.int32, device="cuda") if case["tree"] == "spine" else None
    state = dict(op=case["op"], k_pages=pool(), v_pages=pool(), table=table.cuda(),
                 lengths=lengths.to(torch.int32).cuda(), longest=int(lengths.max()), k=case["k"], depth=case["depth"],
                 first_child=first, counts=counts.to(torch.int32).cuda() if case["counts"] == "ragged" else None,
                 depths=torch.tensor(_depths(case), device="cuda"), layer=layers // 2, neighbours=case["pairs"] == "neighbours",
                 shared=case["shared"], scale=D ** -0.5)
    if case["op"] == "commit":
        # walks of the numbers of accepted drafts that a verification gives, the first child more often than not
        parent = torch.tensor(_parents(case))
        accepted = torch.tensor(_accepted(case))[mixed]
        children = torch.tensor(SPINE) if case["tree"] == "spine" else torch.where(
            torch.arange(N) * case["k"] + case["k"] < N, torch.arange(N) * case["k"] + 1, -1)
        outcome = (torch.rand((B, N), generator=on_host).square() * case["k"]).to(torch.int64).clamp(max=case["k"] - 1)
        if case["tree"] == "spine":
            outcome.zero_()            # only first children have children
        at = torch.zeros(B, dtype=torch.int64)
        for level in range(case["depth"]):
            stop = accepted == level
            outcome[torch.arange(B)[stop], at[stop]] = -1
            step = (children[at] >= 0) & ~stop & (level < accepted)
            at = torch.where(step, children[at] + outcome[torch.arange(B), at].clamp(min=0), at)
        state.update(outcome=outcome.to(torch.int32).cuda(), accept_depth=accepted.to(torch.int32).cuda(),
                     parent=parent.cuda(), new_lengths=torch.zeros(B, dtype=torch.int32, device="cuda"))
        return state
    if case["tree"] == "chain":
        visible = torch.ones((N, N), dtype=torch.bool, device="cuda").tril_()
    else:
        visible = torch.eye(N, dtype=torch.bool)
        for n, p in enumerate(_parents(case)):
            if p >= 0:
                visible[n] |= visible[p]
        visible = visible.cuda()
    state.update(visible=visible, out=torch.zeros((B, N, H * G, D), dtype=dtype, device="cuda"))
    if case["op"] == "append":
        # queries, keys and values as one projection gives them
        qkv = normal(B, N, (G + 2) * H, D)
        state.update(q=qkv[:, :, :G * H], new_k=qkv[:, :, G * H:(G + 1) * H], new_v=qkv[:, :, (G + 1) * H:])
        half = case["rot"] // 2
        state["inv_freq"] = 10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float32) / half)
    else:
        state["q"] = normal(B, N, H * G, D) * 2.0
    return state


def _rotated(x, cos, sin, neighbours):
    half = cos.shape[-1]
    x = x.float()
    if neighbours:
        a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:2 * half]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, x[..., 2 * half:]], -1)


def _new_rows(s, B, N):
    """Which of the N rows of every sequence there are."""
    if s["counts"] is None:
        return torch.ones((B, N), dtype=torch.bool, device="cuda")
    return torch.arange(N, device="cuda") < s["counts"][:, None]


def _places(s, slots):
    """Page and slot within the page of every [B, n] slot of the sequences."""
    page = s["k_pages"].shape[2]
    return s["table"].long().gather(1, slots // page), slots % page


def _append(s):
    B, N = s["q"].shape[:2]
    position = s["lengths"].long()[:, None] + s["depths"]
    # positions of several ten thousand: the angle's whole turns would take an fp32 angle's last digits
    angle = position.double()[..., None] * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    new = _new_rows(s, B, N)
    dtype = s["q"].dtype
    s["out"].copy_(torch.where(new[..., None, None], _rotated(s["q"], cos, sin, s["neighbours"]).to(dtype), s["out"]))
    at, slot = _places(s, s["lengths"].long()[:, None] + torch.arange(N, device="cuda"))
    at, slot = at[new], slot[new]
    s["k_pages"][s["layer"]][at, slot] = _rotated(s["new_k"], cos, sin, s["neighbours"]).to(dtype)[new]
    s["v_pages"][s["layer"]][at, slot] = s["new_v"][new]
    return {"q": s["out"], "k": s["k_pages"], "v": s["v_pages"]}


def _attend(s):
    B, N, heads, D = s["q"].shape
    H = s["k_pages"].shape[3]
    slots = torch.arange(s["longest"] + N, device="cuda")[None].expand(B, -1)
    at, slot = _places(s, slots)
    keys = s["k_pages"][s["layer"]][at.clamp(min=0), slot].float().permute(0, 2, 3, 1).contiguous()
    values = s["v_pages"][s["layer"]][at.clamp(min=0), slot].float().transpose(1, 2).contiguous()
    node = slots - s["lengths"].long()[:, None]
    seen = s["visible"].t()[node.clamp(0, N - 1)].transpose(1, 2) & (node < N)[:, None] | (node < 0)[:, None]
    q = s["q"].float().view(B, N, H, heads // H, D).permute(0, 2, 3, 1, 4).reshape(B, heads, N, D)
    scores = torch.matmul(q.reshape(B, H, -1, D), keys).view(B, heads, N, -1).mul_(s["scale"])
    scores.masked_fill_(~seen[:, None], -math.inf)
    weights = scores.sub_(scores.amax(-1, keepdim=True)).exp_()
    total = weights.sum(-1, keepdim=True)
    o = torch.matmul(weights.view(B, H, -1, weights.shape[-1]), values).view(B, heads, N, D) / total
    new = _new_rows(s, B, N)
    s["out"].copy_(torch.where(new[..., None, None], o.transpose(1, 2).to(s["out"].dtype), s["out"]))
    return s["out"]


def _commit(s):
    B, N = s["outcome"].shape
    parent, outcome = s["parent"], s["outcome"].long()
    # the edge into a node is taken where its parent's outcome is the node's place among the children
    if s["first_child"] is None:
        place = (torch.arange(N, device="cuda") - 1) % s["k"]
    else:
        place = torch.arange(N, device="cuda") - s["first_child"].long()[parent.clamp(min=0)]
    on = (outcome[:, parent.clamp(min=0)] == place) | (parent < 0)
    level = s["depths"]
    for _ in range(s["depth"] - 1):
        on = on & (on[:, parent.clamp(min=0)] | (parent < 0))
    on = on & (level <= s["accept_depth"][:, None])
    base = s["lengths"].long()[:, None]
    at, slot = _places(s, base + torch.arange(N, device="cuda"))
    to, to_slot = _places(s, base + level)
    at, slot, to, to_slot = at[on], slot[on], to[on], to_slot[on]
    for pages in (s["k_pages"], s["v_pages"]):
        pages[:, to, to_slot] = pages[:, at, slot]
    s["new_lengths"].copy_(s["lengths"] + s["accept_depth"] + 1)
    return {"lengths": s["new_lengths"], "k": s["k_pages"], "v": s["v_pages"]}


def run(state):
    s = state
    if own:
        from paper_2411_05289_amd import binding
        cache = binding.KVCache(s["k_pages"], s["v_pages"], s["table"], s["lengths"])
        tree = binding.TokenTree(s["k"], s["depth"], s["first_child"], s["counts"])
        if s["op"] == "append":
            q = binding.kv_append(cache, tree, s["new_k"], s["new_v"], s["q"], s["inv_freq"], layer=s["layer"],
                                  neighbours=s["neighbours"], out=s["out"])
            return {"q": q, "k": s["k_pages"], "v": s["v_pages"]}
        if s["op"] == "attend":
            return binding.tree_attention(cache, tree, s["q"], layer=s["layer"], scale=s["scale"], shared=s["shared"],
                                          longest=s["longest"], out=s["out"])
        lengths = binding.kv_commit(cache, tree, s["outcome"], s["accept_depth"], out=s["new_lengths"])
        return {"lengths": lengths, "k": s["k_pages"], "v": s["v_pages"]}
    return {"append": _append, "attend": _attend, "commit": _commit}[s["op"]](s)


def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    B, N, D, heads, kv = case["B"], _nodes(case), case["dim"], case["heads"], case["kv_heads"]
    lengths, counts, depths = _lengths(case), _counts(case), _depths(case)
    rows = sum(counts)
    if case["op"] == "append":
        # queries, keys and values in and out; a rotation is 6 operations a pair
        return {"bytes": 2 * rows * (heads + 2 * kv) * D * size, "flops": 3 * rows * (heads + kv) * case["rot"]}
    if case["op"] == "attend":
        slots = case["shared"] + sum(x - case["shared"] for x in lengths) + rows
        pairs = sum(x * c + sum(depths[:c]) + c for x, c in zip(lengths, counts))
        return {"bytes": (2 * slots * kv + 2 * rows * heads) * D * size, "flops": 4 * pairs * heads * D}
    # rows that move: the first child of the root stays where it is, of the others in the mean about
    # every one moves
    p = 1 - (1 / case["k"]) ** 0.5 if case["tree"] == "complete" else 0.0
    moved = sum(p * (a > 0) + max(0, a - 1) for a in _accepted(case))
    return {"bytes": moved * case["layers"] * kv * D * size * 4 + 4 * (B * (N + 3)), "flops": 0}


# ---------------------------------------------------------------- the same in 64 bits
def _slot_of(s, b, n):
    page = s["k_pages"].shape[2]
    return s["table"][b].long()[n // page], n % page


def exact(case, seed):
    s = prepare(case, seed)
    lengths, N = s["lengths"].tolist(), _nodes(case)
    B = len(lengths)
    counts = s["counts"].tolist() if s["counts"] is not None else [N] * B
    if case["op"] == "append":
        half = case["rot"] // 2
        q, k, v = s["q"].double(), s["new_k"].double(), s["new_v"].double()
        if s["neighbours"]:
            first = torch.arange(half, device="cuda") * 2
            second = first + 1
        else:
            first = torch.arange(half, device="cuda")
            second = first + half
        out, keys, values = s["out"].double(), s["k_pages"].double(), s["v_pages"].double()
        for b in range(B):
            c = counts[b]
            turn = torch.outer((lengths[b] + s["depths"][:c]).double(), s["inv_freq"].double())
            unit = torch.polar(torch.ones_like(turn), turn)[:, None]
            at, slot = _slot_of(s, b, lengths[b] + torch.arange(c, device="cuda"))
            for x, into in ((q, out), (k, None)):
                z = torch.complex(x[b, :c][..., first], x[b, :c][..., second]) * unit
                y = x[b, :c].clone()
                y[..., first], y[..., second] = z.real, z.imag
                if into is not None:
                    into[b, :c] = y
                else:
                    keys[s["layer"]].index_put_((at, slot), y)
            values[s["layer"]].index_put_((at, slot), v[b, :c])
        return {"q": out, "k": keys, "v": values}
    if case["op"] == "attend":
        out = s["out"].double()
        G = case["heads"] // case["kv_heads"]
        for b in range(B):
            c, L = counts[b], lengths[b]
            at, slot = _slot_of(s, b, torch.arange(L + c, device="cuda"))
            for h in range(case["kv_heads"]):
                k = s["k_pages"][s["layer"], :, :, h][at, slot].double()
                v = s["v_pages"][s["layer"], :, :, h][at, slot].double()
                for g in range(h * G, (h + 1) * G):
                    x = (s["q"][b, :c, g].double() * s["scale"]) @ k.t()
                    x[:, L:] = torch.where(s["visible"][:c, :c], x[:, L:], -math.inf)
                    out[b, :c, g] = torch.softmax(x, -1) @ v
        return out
    keys, values = s["k_pages"].double(), s["v_pages"].double()
    outcome, accepted = s["outcome"].tolist(), s["accept_depth"].tolist()
    for b in range(B):
        node, path = 0, [0]
        for _ in range(accepted[b]):
            node = (SPINE[node] if case["tree"] == "spine" else case["k"] * node + 1) + outcome[b][node]
            path.append(node)
        at, slot = _slot_of(s, b, lengths[b] + torch.tensor(path, device="cuda"))
        to, to_slot = _slot_of(s, b, lengths[b] + torch.arange(len(path), device="cuda"))
        for pages in (keys, values):
            pages[:, to, to_slot] = pages[:, at, slot]
    return {"lengths": s["lengths"] + s["accept_depth"] + 1, "k": keys, "v": values}
