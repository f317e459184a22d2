"""The key-value cache of token trees: what the calls refuse (CPU), and appending, attending and committing against
64-bit references (GPU)."""
import ctypes as C
import math

import pytest
import torch

from paper_2411_05289_amd import binding as B
from kv_reference import SPINE, TYPES, attention, half_step, levels, make_pages, parents, path_of, rotated

gpu = pytest.mark.gpu
DEV = "cuda"


# ---------------------------------------------------------------- refusals (nothing is launched)
def _cache(**kw):
    c = B._Cache()
    c.k, c.v = 0x10000, 0x20000     # never dereferenced
    c.ld_layer, c.ld_page, c.ld_slot, c.ld_head = 1 << 20, 16 * 2 * 64, 2 * 64, 64
    c.dtype, c.layers, c.pages, c.page_size, c.heads, c.dim, c.table_pages = B.BF16, 2, 8, 16, 2, 64, 4
    c.table, c.ld_table, c.lengths = 0x30000, 4, 0x40000
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _tree(**kw):
    t = B._Tree()
    t.B, t.N, t.k, t.depth = 1, 7, 2, 3
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def _heads(n=2, **kw):
    h = B._Heads()
    h.p, h.ld_tree, h.ld_node, h.ld_head, h.heads = 0x50000, 7 * n * 64, n * 64, 64, n
    for k, v in kw.items():
        setattr(h, k, v)
    return h


def _append(cache=None, tree=None, k=None, v=None, q=None, q_out=None, inv_freq=0x60000, rot=64, style=0, layer=0, flags=None):
    ref = lambda x: None if x is None else C.byref(x)  # noqa: E731
    return B.lib().mdsd_kv_append(ref(cache or _cache()), layer, ref(tree or _tree()), ref(k or _heads()), ref(v or _heads()),
                                  ref(q), ref(q_out), inv_freq, rot, style, flags, None)


def _attend(cache=None, tree=None, q=None, out=None, scale=0.125, shared_pages=None, shared=0, longest=0, layer=0, flags=None,
            ws=None, ws_bytes=0):
    return B.lib().mdsd_tree_attention(C.byref(cache or _cache()), layer, C.byref(tree or _tree()), C.byref(q or _heads(4)),
                                       C.byref(out or _heads(4, p=0x70000)), scale, shared_pages, shared, longest, flags, ws,
                                       ws_bytes, None)


def _commit(cache=None, tree=None, outcome=0x80000, accept_depth=0x90000, new_lengths=0xA0000, flags=None):
    return B.lib().mdsd_kv_commit(C.byref(cache or _cache()), C.byref(tree or _tree()), outcome, accept_depth, new_lengths, flags,
                                  None)


@pytest.mark.parametrize("call", [_append, _attend, _commit])
@pytest.mark.parametrize("kw,code", [
    (dict(k=None), -1), (dict(v=None), -1), (dict(table=None), -1), (dict(lengths=None), -1), (dict(dtype=3), -5),
    (dict(layers=0), -2), (dict(pages=0), -2), (dict(page_size=0), -2), (dict(heads=0), -2), (dict(table_pages=0), -2),
    (dict(dim=0), -2), (dict(dim=60), -2), (dict(dim=264), -2), (dict(ld_table=3), -2), (dict(page_size=1 << 29), -2),
    (dict(k=0x10008), -6), (dict(v=0x20002), -6), (dict(ld_slot=65), -6), (dict(ld_page=-16), -6), (dict(ld_head=4), -6),
    (dict(ld_page=1 << 35), -2), (dict(ld_slot=1 << 35), -2), (dict(ld_layer=1 << 47), -6),
    (dict(table=0x30001), -6), (dict(lengths=0x40002), -6),
])
def test_bad_caches_are_refused(call, kw, code):
    assert call(cache=_cache(**kw)) == code


@pytest.mark.parametrize("call", [_append, _attend, _commit])
@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), -2), (dict(N=0), -2), (dict(N=6), -2), (dict(depth=0), -2), (dict(k=0, N=1), -3), (dict(k=9), -3),
    (dict(k=1), -2), (dict(N=4097, first_child=0xB0000), -2), (dict(B=1 << 20, N=1 << 20, k=1, depth=1 << 20), -2),
])
def test_bad_trees_are_refused(call, kw, code):
    assert call(tree=_tree(**kw)) == code


@pytest.mark.parametrize("call", [_append, _attend, _commit])
@pytest.mark.parametrize("kw", [dict(first_child=0xB0001), dict(first_child=0xB0002), dict(counts=0xC0002), dict(counts=0xC0003)])
def test_trees_that_are_not_aligned_are_refused(call, kw):
    assert call(tree=_tree(**kw)) == -6


@pytest.mark.parametrize("call", [
    lambda: _append(tree=_tree(B=1 << 12, N=1 << 12, k=1, depth=1 << 12)), lambda: _append(tree=_tree(B=1 << 24, N=1, k=1, depth=1)),
    lambda: _commit(tree=_tree(B=1 << 23), new_lengths=1 << 40), lambda: _attend(tree=_tree(B=1 << 23, N=1, k=1, depth=1)),
    lambda: _attend(tree=_tree(B=1 << 23, N=1, k=1, depth=1), ws=0x1000, ws_bytes=1 << 62),
    lambda: _attend(tree=_tree(B=1, N=1 << 29, k=1, depth=1 << 29), out=_heads(4, p=1 << 48)),
])
def test_calls_that_no_launch_can_hold_are_refused(call):
    assert call() == -2


@pytest.mark.parametrize("scale,code", [(2.3e38, -2), (2.4e38, -4), (3.0e38, -4), (1e-44, -2)])
def test_scales_whose_exponent_to_two_is_no_number_are_refused(scale, code):
    assert _attend(scale=scale, tree=_tree(B=1 << 23, N=1, k=1, depth=1)) == code      # (too large a call: nothing is launched)


ROW = 6 * 128      # of 6 heads of 64 bf16 elements, of which the queries are the first ones


@pytest.mark.parametrize("heads,off,strides,refused", [
    (4, 0, {}, False), (4, 0, dict(ld_node=4 * 64, ld_tree=28 * 64), True), (4, 0, dict(ld_tree=1 << 20), True),
    (4, 128, {}, True), (4, 2 * 128, {}, True), (4, -128, {}, True), (4, 16, {}, True), (4, ROW, {}, True), (4, 7 * ROW, {}, True),
    (4, -7 * ROW - 112, {}, True), (4, 4 * 128, {}, True), (4, 14 * ROW, {}, False), (4, 2 * 128 - 14 * ROW, {}, False),
    (4, 13 * ROW + 4 * 128, {}, False), (4, 13 * ROW + 4 * 128 - 16, {}, True), (2, 2 * 128, {}, False), (2, 4 * 128, {}, False),
    (2, 5 * 128, {}, True), (2, ROW + 2 * 128, {}, False), (2, ROW + 128, {}, True), (2, -ROW - 2 * 128, {}, False),
])
def test_results_that_overlap_the_queries_are_refused(heads, off, strides, refused):
    """Two trees of 7 nodes; the queries themselves and what lies between or behind them may be written."""
    own = dict(ld_node=ROW // 2, ld_tree=7 * ROW // 2)
    q, out = _heads(heads, p=0x50000, **own), _heads(heads, p=0x50000 + off, **{**own, **strides})
    # (an argument that is looked at later is wrong too: nothing is launched)
    assert _attend(tree=_tree(B=2), q=q, out=out, scale=0.0) == (-6 if refused else -4)
    assert _append(tree=_tree(B=2), q=q, q_out=out, style=7) == (-6 if refused else -5)


@pytest.mark.parametrize("dims", [dict(B=1), dict(B=2, N=1, k=1, depth=1), dict(B=1, N=1, k=1, depth=1)])
def test_results_in_the_queries_place_go_by_the_strides_that_matter(dims):
    """Strides of an axis of one element may be anything."""
    N = dims.get("N", 7)
    any_ = {**(dict(ld_tree=0) if dims["B"] == 1 else {}), **(dict(ld_node=0) if N == 1 else {})}
    q, out = _heads(4, p=0x50000, ld_tree=28 * 64, ld_node=256), _heads(4, p=0x50000, **{"ld_tree": 28 * 64, "ld_node": 256, **any_})
    assert _attend(tree=_tree(**dims), q=q, out=out, scale=0.0) == -4


def test_empty_batches_and_missing_structures():
    for call in (_append, _attend, _commit):
        assert call(cache=_cache(k=None, dtype=9), tree=_tree(B=0)) == 0
    L = B.lib()
    assert L.mdsd_kv_append(None, 0, C.byref(_tree()), None, None, None, None, None, 0, 0, None, None) == -1
    assert L.mdsd_kv_append(C.byref(_cache()), 0, None, None, None, None, None, None, 0, 0, None, None) == -1
    assert L.mdsd_tree_attention(C.byref(_cache()), 0, C.byref(_tree()), None, None, 1.0, None, 0, 0, None, None, 0, None) == -1
    assert L.mdsd_kv_commit(None, C.byref(_tree()), 8, 8, 8, None, None) == -1


@pytest.mark.parametrize("kw,code", [
    (dict(layer=2), -2), (dict(layer=-1), -2), (dict(k=_heads(3)), -2), (dict(v=_heads(1)), -2), (dict(k=_heads(p=None)), -1),
    (dict(k=_heads(p=0x50004)), -6), (dict(v=_heads(ld_node=100)), -6), (dict(q=_heads(4)), -1), (dict(q_out=_heads(4)), -1),
    (dict(q=_heads(4), q_out=_heads(2)), -2), (dict(q=_heads(4, ld_head=-64), q_out=_heads(4)), -6), (dict(rot=63), -2),
    (dict(rot=66), -2), (dict(rot=-2), -2), (dict(inv_freq=None), -1), (dict(inv_freq=0x60002), -6), (dict(style=2), -5),
    (dict(flags=0x61), -6), (dict(cache=_cache(ld_head=0)), -2), (dict(cache=_cache(ld_page=0)), -2),
    (dict(q=_heads(4), q_out=_heads(4, ld_node=0)), -2),
])
def test_appends_that_are_refused(kw, code):
    assert _append(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(layer=2), -2), (dict(q=_heads(3), out=_heads(3)), -2), (dict(out=_heads(2)), -2), (dict(q=_heads(4, p=None)), -1),
    (dict(out=_heads(4, p=0x70002)), -6), (dict(scale=0.0), -4), (dict(scale=-1.0), -4), (dict(scale=math.inf), -4),
    (dict(scale=math.nan), -4), (dict(shared=-1), -2), (dict(shared=65, shared_pages=0x100), -2), (dict(shared=16), -1),
    (dict(shared=16, shared_pages=0x102), -6), (dict(longest=-1), -2), (dict(flags=0x61), -6), (dict(ws=0x1008, ws_bytes=1 << 30), -6),
    (dict(out=_heads(4, p=0x70000, ld_head=0)), -2), (dict(tree=_tree(B=2), out=_heads(4, p=0x70000, ld_tree=0)), -2),
])
def test_attentions_that_are_refused(kw, code):
    assert _attend(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(outcome=None), -1), (dict(accept_depth=None), -1), (dict(new_lengths=None), -1), (dict(outcome=0x80001), -6),
    (dict(new_lengths=0x80002), -6), (dict(flags=0x61), -6),
    (dict(cache=_cache(ld_layer=0)), -2), (dict(cache=_cache(ld_slot=0)), -2),
    (dict(new_lengths=0x40004, tree=_tree(B=2)), -6), (dict(new_lengths=0x3FFFC, tree=_tree(B=2)), -6),
])
def test_commits_that_are_refused(kw, code):
    assert _commit(**kw) == code


@pytest.mark.parametrize("B_,N,q_heads,heads,dim,dtype,shared", [(8500, 1, 8, 8, 64, 1, 1040), (100000, 1, 8, 1, 128, 1, 4096),
                                                                 (20000, 1, 1, 1, 256, 0, 2048), (3000, 15, 8, 2, 128, 2, 16384)])
def test_workspaces_go_by_the_trees_rows(B_, N, q_heads, heads, dim, dtype, shared):
    """Behind a prefix that is met once a tree's own part and the prefix's have its results in fp32 and two words a row, whatever the
    kernels' tiles; 512 workgroups have a part each besides, of 128 rows at most."""
    cache = _cache(dtype=dtype, heads=heads, dim=dim, table_pages=shared // 16 + 1, ld_table=shared // 16 + 1,
                   ld_slot=heads * dim, ld_head=dim, ld_page=16 * heads * dim)
    tree = _tree(B=B_, N=N, k=1, depth=N)
    size = B.lib().mdsd_tree_attention_workspace_bytes(C.byref(cache), C.byref(tree), q_heads, shared, 0)
    assert size > B.lib().mdsd_tree_attention_workspace_bytes(C.byref(cache), C.byref(tree), q_heads, 0, 0)
    results = B_ * N * q_heads * (4 * dim + 8 + 8)
    assert size <= 2 * results + (2 * 512 + heads) * 128 * (4 * dim + 8) + 4096


@pytest.mark.parametrize("B_,N,shared,once", [
    (64, 1, 1024, True), (64, 8, 1024, False), (64, 8, 2048, True), (128, 15, 2048, False), (128, 15, 3200, False), (64, 15, 4096, True),
    (64, 31, 6144, True), (128, 31, 8192, False), (64, 15, 16384, True),
])
def test_prefixes_that_are_met_once(B_, N, shared, once):
    """Only where that was measured to be the faster (32 query heads on 8 of 128): a workspace of another size."""
    entries = (shared + 512) // 16
    cache = _cache(heads=8, dim=128, table_pages=entries, ld_table=entries, ld_slot=1024, ld_head=128, ld_page=16 * 1024)
    size = [B.lib().mdsd_tree_attention_workspace_bytes(C.byref(cache), C.byref(_tree(B=B_, N=N, k=1, depth=N)), 32, s, 0)
            for s in (0, shared)]
    assert (size[0] != size[1]) == once


def test_binding_refuses_what_is_not_on_the_gpu():
    pool = torch.zeros((1, 4, 16, 2, 64), dtype=torch.bfloat16)
    cache = B.KVCache(pool, pool.clone(), torch.zeros((1, 4), dtype=torch.int32), torch.zeros(1, dtype=torch.int32))
    x = torch.zeros((1, 7, 2, 64), dtype=torch.bfloat16)
    for call in (lambda: B.kv_append(cache, B.TokenTree(2, 3), x, x), lambda: B.tree_attention(cache, B.TokenTree(2, 3), x),
                 lambda: B.kv_commit(cache, B.TokenTree(2, 3), torch.zeros((1, 7), dtype=torch.int32), torch.zeros(1, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call()


@gpu
@pytest.mark.parametrize("native", [True, False])
def test_binding_refuses_what_does_not_fit(native, monkeypatch):
    if not native:
        monkeypatch.setattr(B, "_native", lambda: None)
    k, v, table, _ = make_pages([5, 9], 7, 16, dim=64, dtype=torch.bfloat16)
    cache = B.KVCache(k, v, table, torch.tensor([5, 9], dtype=torch.int32, device=DEV))
    x = torch.zeros((2, 7, 2, 64), dtype=torch.bfloat16, device=DEV)
    tree = B.TokenTree(2, 3)
    bad = [dict(k=x.float()), dict(k=x[:1]), dict(k=x[:, :, :, :32]), dict(v=x[:, :6]), dict(q=x.cpu()), dict(q=x, out=x[:, :3]),
           dict(inv_freq=torch.ones(32, dtype=torch.float64, device=DEV)), dict(flags=torch.zeros(3, dtype=torch.int32, device=DEV))]
    for kw in bad:
        with pytest.raises(ValueError):
            B.kv_append(cache, tree, kw.pop("k", x), kw.pop("v", x), **kw)
    with pytest.raises(B.MdsdError):
        B.kv_append(cache, B.TokenTree(2, 4), x, x)
    with pytest.raises(B.MdsdError):
        B.kv_append(cache, tree, x, x, layer=1)
    for kw in (dict(out=x.float()), dict(shared=40, shared_pages=table[0, :2]), dict(workspace=torch.zeros(64, device=DEV))):
        with pytest.raises(ValueError):
            B.tree_attention(cache, tree, x, **kw)
    with pytest.raises(B.MdsdError):
        B.tree_attention(cache, tree, x, scale=0.0)
    with pytest.raises(ValueError):
        B.kv_commit(cache, tree, torch.zeros((2, 7), dtype=torch.int64, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError):
        B.tree_attention(B.KVCache(k, v.transpose(2, 3), table, cache.lengths), tree, x)


@gpu
@pytest.mark.parametrize("native", [True, False])
def test_binding_refuses_numbers_that_do_not_fit(native, monkeypatch):
    """Beyond 32 bits: not another layer, prefix or tree by the low ones."""
    if not native:
        monkeypatch.setattr(B, "_native", lambda: None)
    k, v, table, _ = make_pages([5, 9], 7, 16, dim=64, dtype=torch.bfloat16)
    cache = B.KVCache(k, v, table, torch.tensor([5, 9], dtype=torch.int32, device=DEV))
    x = torch.zeros((2, 7, 2, 64), dtype=torch.bfloat16, device=DEV)
    tree, far = B.TokenTree(2, 3), 2 ** 32
    before = k.nan_to_num(9.0)
    outcome, accept = torch.zeros((2, 7), dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    calls = [lambda: B.kv_append(cache, tree, x, x, layer=far), lambda: B.kv_append(cache, B.TokenTree(2 + far, 3), x, x),
             lambda: B.tree_attention(cache, tree, x, layer=-far), lambda: B.tree_attention(cache, tree, x, longest=far + 9),
             lambda: B.tree_attention(cache, tree, x, shared=far + 16), lambda: B.tree_attention(cache, B.TokenTree(2, 3 + far), x),
             lambda: B.attention_workspace(cache, tree, x, longest=far), lambda: B.attention_workspace(cache, tree, x, shared=far),
             lambda: B.kv_commit(cache, B.TokenTree(2, 3 + far), outcome, accept)]
    for call in calls:
        with pytest.raises(ValueError):
            call()
    assert torch.equal(k.nan_to_num(9.0), before)


# ---------------------------------------------------------------- attention
def _tree_of(name, N=None):
    """(k, depth, table or None, N) of a named tree."""
    if name == "spine":
        return 2, 5, SPINE, 9
    if name == "roots":      # node 3's entry is malformed, nodes 5 and 6 are claimed by none, 3 and 4 by two
        return 2, 3, (1, 3, 3, 3, -1, 9, -1), 7
    if name == "chain":
        return 1, N, None, N
    if name == "chain_table":
        return 1, N, tuple(n + 1 if n + 1 < N else -1 for n in range(N)), N
    k, depth = {"binary": (2, 4), "binary5": (2, 5), "binary7": (2, 7), "ternary": (3, 3), "four": (4, 3), "eight": (8, 2),
                "one": (2, 1)}[name]
    return k, depth, None, (k ** depth - 1) // (k - 1)


def _queries(B_, N, heads, dim, dtype, seed, fused=False):
    gen = torch.Generator().manual_seed(seed + 31)
    if fused:   # a slice of a wider projection: strides of their own
        x = (2 * torch.randn((B_, N, heads + 3, dim), generator=gen)).to(dtype).to(DEV)
        return x[:, :, 1:1 + heads]
    return (2 * torch.randn((B_, N, heads, dim), generator=gen)).to(dtype).to(DEV)


def _check_attention(dtype, dim, heads, G, tree, lengths, *, N=None, page_size=16, order="slots", counts=None, layers=1, fused=False,
                     shared=0, workspace="own", seed=0, change=None, longest=0, flags=None):
    dt = TYPES[dtype]
    k, depth, first, N = _tree_of(tree, N)
    kp, vp, table, _ = make_pages(lengths, N, page_size, layers=layers, heads=heads, dim=dim, dtype=dt, order=order, shared=shared,
                                  seed=seed)
    len_t = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    q = _queries(len(lengths), N, heads * G, dim, dt, seed, fused)
    if change is not None:
        change(kp, vp, table, len_t, q)
    cache = B.KVCache(kp, vp, table, len_t)
    t = B.TokenTree(k, depth, None if first is None else torch.tensor(first, dtype=torch.int32, device=DEV),
                    None if counts is None else torch.tensor(counts, dtype=torch.int32, device=DEV))
    layer = layers - 1
    # the call is cut by the longest that sequences may be: once as told, and with tables that would hold long ones, whose further
    # entries are no pages, shared out and not
    wider = torch.cat([table, torch.full((len(lengths), 140000 // page_size), -1, dtype=torch.int32, device=DEV)], 1)
    outs = [torch.full((len(lengths), N, heads * G, dim), 7.5, dtype=dt, device=DEV) for _ in range(3)]
    if workspace == "none":
        _attend_without_workspace(cache, t, q, outs[0], layer, shared, flags)
    else:
        B.tree_attention(cache, t, q, layer=layer, shared=shared, out=outs[0], longest=longest, flags=flags)
    wide = B.KVCache(kp, vp, wider, len_t)
    B.tree_attention(wide, t, q, layer=layer, shared=shared, shared_pages=table[0], out=outs[1], flags=flags)
    _attend_without_workspace(wide, t, q, outs[2], layer, shared, flags)
    torch.cuda.synchronize()
    parent = parents(k, N, first)
    c = counts or [N] * len(lengths)
    rows = table.cpu().tolist()
    want, off = attention(kp[layer], vp[layer], rows, len_t.tolist(), c, parent, q, dim ** -0.5, shared, rows[0])
    for out in outs:
        got = out.double().cpu()
        for b in range(len(lengths)):
            m = max(0, min(N, c[b])) if len_t[b] >= 0 else 0
            assert (got[b, m:] == 7.5).all(), ("rows behind the last", b)
            w, g, o = want[b, :m], got[b, :m], off[b, :m]
            fine = torch.isfinite(w)
            assert torch.equal(torch.isnan(w), torch.isnan(g)) and torch.equal(w[~fine & ~torch.isnan(w)], g[~fine & ~torch.isnan(w)])
            wrong = (w - g).abs() > o
            assert not (wrong & fine).any(), (b, wrong.nonzero()[:4].tolist(), float(((w - g).abs() / o)[fine].max()))
    return outs[0]


def _attend_without_workspace(cache, tree, q, out, layer, shared, flags=None):
    c, t = B._c_cache(cache), B._c_tree(tree, q.shape[0], q.shape[1])
    qh, oh = B._c_heads("q", q, cache), B._c_heads("out", out, cache)
    rc = B.lib().mdsd_tree_attention(C.byref(c), layer, C.byref(t), C.byref(qh), C.byref(oh), q.shape[3] ** -0.5,
                                     B._ptr(cache.table[0]), shared, 0, B._ptr(flags), None, 0, B._stream())
    assert rc == 0


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim", [8, 64, 80, 128, 192, 256])
def test_attention_types_and_dims(dtype, dim):
    _check_attention(dtype, dim, 2, 4, "binary", [0, 1, 63, 64, 65, 200], seed=dim)


@gpu
@pytest.mark.parametrize("tree,N", [("one", None), ("binary5", None), ("binary7", None), ("ternary", None), ("four", None), ("eight", None),
                                    ("spine", None), ("roots", None), ("chain", 1), ("chain", 2), ("chain", 70), ("chain", 200),
                                    ("chain_table", 150)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_trees(tree, N, dtype):
    _check_attention(dtype, 64, 2, 2, tree, [0, 30, 129], N=N, seed=3)


@gpu
@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("bf16", 256), ("fp32", 256)])
def test_attention_largest_table(dtype, dim):
    """As many nodes as a table may have, one below the other, beside a tree of none."""
    _check_attention(dtype, dim, 1, 1, "chain_table", [33, 5], N=4096, counts=[4096, 0], seed=4)


@gpu
def test_empty_batch():
    """No sequences: nothing happens, with a prefix and without."""
    pool = torch.zeros((2, 1, 4, 16, 2, 64), device=DEV)
    none = torch.empty((0,), dtype=torch.int32, device=DEV)
    cache, tree = B.KVCache(pool[0], pool[1], none.reshape(0, 4), none), B.TokenTree(2, 2)
    x = torch.empty((0, 3, 2, 64), device=DEV)
    assert B.kv_append(cache, tree, x, x, x).shape == B.tree_attention(cache, tree, x, shared=32).shape == x.shape
    assert B.kv_commit(cache, tree, none.reshape(0, 3), none).shape == (0,)


@gpu
@pytest.mark.parametrize("heads,G", [(1, 1), (1, 8), (3, 1), (2, 7), (8, 16), (1, 40)])
def test_attention_head_layouts(heads, G):
    _check_attention("bf16", 128, heads, G, "binary", [0, 77], seed=heads, fused=True)
    _check_attention("fp16", 64, heads, G, "chain", [5, 40], N=3, seed=heads, fused=True, order="heads")


@gpu
@pytest.mark.parametrize("dtype,dim,heads,G,tree,N,lengths,shared", [
    ("bf16", 128, 2, 4, "one", None, [3000], 0), ("bf16", 128, 8, 4, "one", None, [30, 500, 7], 0),
    ("bf16", 128, 2, 4, "binary5", None, [700, 0, 41], 0), ("fp16", 64, 8, 4, "binary5", None, [5000, 3, 900], 0),
    ("fp32", 80, 2, 3, "spine", None, [2000, 5], 0), ("bf16", 64, 2, 4, "chain", 300, [500, 0], 0),
    ("bf16", 256, 1, 2, "binary5", None, [2500, 8], 0), ("bf16", 128, 2, 4, "binary", None, [2300, 2290, 2240, 2301, 2310, 2250], 2240),
])
def test_attention_in_the_queries_place(dtype, dim, heads, G, tree, N, lengths, shared):
    """out=q: the same bits as results of their own give, whichever way the work is cut."""
    dt = TYPES[dtype]
    k, depth, first, N = _tree_of(tree, N)
    kp, vp, table, _ = make_pages(lengths, N, 16, heads=heads, dim=dim, dtype=dt, shared=shared, seed=dim)
    cache = B.KVCache(kp, vp, table, torch.tensor(lengths, dtype=torch.int32, device=DEV))
    t = B.TokenTree(k, depth, None if first is None else torch.tensor(first, dtype=torch.int32, device=DEV))
    for longest in (0, max(lengths)):
        q = _queries(len(lengths), N, heads * G, dim, dt, N, fused=True)
        want = B.tree_attention(cache, t, q, shared=shared, longest=longest)
        alone = torch.empty_like(want)
        _attend_without_workspace(cache, t, q, alone, 0, shared)
        again = q.clone(memory_format=torch.contiguous_format)
        assert B.tree_attention(cache, t, q, shared=shared, longest=longest, out=q) is q and torch.equal(q, want)
        _attend_without_workspace(cache, t, again, again, 0, shared)
        assert torch.equal(again, alone)


@gpu
@pytest.mark.parametrize("page_size", [1, 3, 16, 48, 64, 100, 257])
@pytest.mark.parametrize("order", ["slots", "heads"])
def test_attention_pages(page_size, order):
    _check_attention("bf16", 64, 2, 2, "binary", [0, 15, 100, 300], page_size=page_size, order=order, layers=2, seed=page_size)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_of_fewer_nodes(dtype):
    _check_attention(dtype, 64, 2, 2, "binary", [10, 10, 70, 0, 3], counts=[15, 0, 1, 9, 99], seed=5)
    _check_attention(dtype, 64, 1, 4, "chain", [10, 0, 70], N=90, counts=[1, 90, 64], seed=6)


@gpu
def test_attention_sees_nothing_of_what_is_not_there():
    """Infinities and NaNs in keys and values of nodes that a row does not see, and in those it sees."""
    def change(kp, vp, table, lengths, q):
        def at(s):
            return 0, int(table[0, s // 16]), s % 16
        kp[at(70 + 2)] = math.nan          # node 2 and what is below it: NaN
        vp[at(70 + 3)][:, 5] = math.inf    # node 3 and below: one element
        vp[at(70 + 4)][:, 6] = -math.inf
        vp[at(70 + 9)][:, 6] = math.nan
        kp[at(70 + 10)] = -300.0
    for dtype in ("bf16", "fp16", "fp32"):
        _check_attention(dtype, 64, 2, 2, "binary", [70, 20], seed=8, change=change)

    def in_sequence(kp, vp, table, lengths, q):
        vp[0, int(table[0, 1]), 3, :, 7] = math.inf
        kp[0, int(table[1, 0]), 3] = math.nan
    _check_attention("bf16", 64, 2, 2, "binary", [70, 20, 9], seed=9, change=in_sequence)


@gpu
def test_attention_large_scores():
    def change(kp, vp, table, lengths, q):
        q.mul_(60.0)
    for dtype in ("bf16", "fp32"):
        _check_attention(dtype, 128, 2, 2, "binary", [0, 40, 200], seed=10, change=change)


@gpu
@pytest.mark.parametrize("dtype,most", [("bf16", 100), ("fp16", 30), ("fp32", 104), ("bf16", 22), ("fp16", 24), ("fp32", 26)])
@pytest.mark.parametrize("tree,G,heads,dim,lengths,shared", [
    ("one", 1, 2, 64, [0, 1, 300], 0), ("one", 4, 1, 128, [5000], 0), ("spine", 3, 2, 80, [40, 2000], 0), ("binary5", 4, 2, 128, [3, 900], 0),
    ("binary5", 2, 2, 64, [4000, 700], 0), ("binary", 4, 2, 256, [2300, 2240, 2241, 2240, 2250, 17], 2240), ("one", 2, 2, 64, [90] * 200, 0),
])
def test_attention_of_far_scores(dtype, most, tree, G, heads, dim, lengths, shared):
    """Scores times the scale up to 2^most, of both signs, rows of small ones between them: beyond 2^24 their steps in fp32 are larger
    than the range of a weight's exponent.  A row's scores are equal or differ by a quarter of the largest at least."""
    dt = TYPES[dtype]
    k, depth, first, N = _tree_of(tree)
    kp, vp, table, _ = make_pages(lengths, N, 16, heads=heads, dim=dim, dtype=dt, shared=shared, seed=most)
    gen = torch.Generator().manual_seed(most + N)
    high = most // 2
    # every key is one vector a number of times, every query one of a few multiples of another: their signs agree
    signs = torch.randint(0, 2, (dim,), generator=gen).to(torch.float32) * 2 - 1
    level = torch.tensor([0.25, 0.5, 0.75, 1.0, -1.0, -0.5])[torch.randint(0, 6, kp.shape[:4], generator=gen)]
    there = ~torch.isnan(kp[..., 0])
    kp.copy_(torch.where(there.cpu()[..., None], level[..., None] * signs * 1.25 * 2.0 ** (most - high), math.nan).to(dt))
    q = torch.tensor([1.0, -1.0, 2.0 ** -high, 2.0 ** (2 - most), -2.0 ** (3 - most)])[
        torch.randint(0, 5, (len(lengths), N, heads * G), generator=gen)]
    q = (q[..., None] * signs * 2.0 ** high * dim ** -0.5).to(dt).to(DEV)
    len_t = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    cache = B.KVCache(kp, vp, table, len_t)
    t = B.TokenTree(k, depth, None if first is None else torch.tensor(first, dtype=torch.int32, device=DEV))
    rows = table.cpu().tolist()
    scale = dim ** -0.5
    want, off = attention(kp[0], vp[0], rows, lengths, [N] * len(lengths), parents(k, N, first), q, scale, shared, rows[0])
    # a far row's largest scores are equal, or alone: their weights are one, the others' nothing, and what is left of the bound is the
    # sums' and the weights' rounding (the values are below 6); a near row's is as ever
    size = (q.double().abs().sum(-1).cpu() * 1.25 * 2.0 ** (most - high) * scale)[..., None]
    far = (max(lengths) + N + 64) * 2.0 ** -24 + 2 * half_step(dt) + 2.0 ** -20
    off = torch.where(size > 2.0 ** 12, 6.0 * far, off)
    wide = B.KVCache(kp, vp, torch.cat([table, torch.full((len(lengths), 140000 // 16), -1, dtype=torch.int32, device=DEV)], 1), len_t)
    alone = torch.empty_like(q)
    _attend_without_workspace(wide, t, q, alone, 0, shared)
    for got in (B.tree_attention(cache, t, q, shared=shared), alone,
                B.tree_attention(wide, t, q, shared=shared, shared_pages=table[0])):
        wrong = ~((got.double().cpu() - want).abs() <= off)
        assert not wrong.any(), (wrong.nonzero()[:4].tolist(), got.cpu()[wrong][:4], want[wrong][:4], off[wrong][:4])


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("G", [1, 5])
def test_attention_of_many_small_weights(dtype, G):
    """One key whose weight is 2^25 times each other's, which together are not nothing: its value is zero, theirs are large."""
    def change(kp, vp, table, lengths, q):
        q.fill_(0.5)
        kp.zero_()
        vp.mul_(20.0).add_(900.0)
        p = int(table[0, 2]), 5
        kp[0, p[0], p[1]] = 4.375      # 64 * 0.5 * 4.375 / 8 = 17.5
        vp[0, p[0], p[1]] = 0.0
    _check_attention(dtype, 64, 1, G, "binary", [5000], seed=21, change=change)


@gpu
@pytest.mark.parametrize("workspace", ["own", "none"])
@pytest.mark.parametrize("page_size,shared", [(16, 64), (16, 80), (16, 100), (1, 33), (64, 128), (16, 256), (3, 301), (64, 2100)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_shared_prefix(workspace, page_size, shared, dtype):
    """Slots below `shared` come from the first sequence's pages; a sequence may be shorter than that."""
    def change(kp, vp, table, lengths, q):
        # where the prefix ends inside a page, every sequence has its own copy of that page
        whole = shared // page_size * page_size
        for b in range(1, table.shape[0]):
            for s in range(whole, min(shared, int(lengths[b]))):
                for pool in (kp, vp):
                    pool[:, int(table[b, s // page_size]), s % page_size] = pool[:, int(table[0, s // page_size]), s % page_size]
    _check_attention(dtype, 64, 2, 3, "binary", [shared, shared + 1, shared + 70, shared + 200, 20], page_size=page_size,
                     shared=shared, workspace=workspace, seed=shared, change=change, longest=shared + 200)


@gpu
@pytest.mark.parametrize("tree,N,G,shared", [("one", None, 1, 1040), ("one", None, 8, 1040), ("binary5", None, 4, 2064), ("spine", None, 7, 2064), ("binary5", None, 4, 6160),
                                             ("chain", 16, 2, 1040), ("chain", 33, 2, 2064)])
@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("fp16", 80), ("fp32", 64), ("bf16", 256), ("fp32", 256)])
def test_attention_shared_prefix_trees(tree, N, G, shared, dtype, dim):
    """Prefixes long enough to be met once: rows of several trees in one tile, trees that lie across two, trees of fewer nodes."""
    N_ = _tree_of(tree, N)[3]
    _check_attention(dtype, dim, 2, G, tree, [shared, shared, shared + 12, shared + 1, shared + 113, shared, shared + 32], N=N,
                     shared=shared, counts=[N_, 1, 0, N_, min(N_, 2), 99, N_], seed=G, longest=shared + 113)


@gpu
def test_attention_shared_prefix_of_very_many():
    """More trees and heads than a launch has places along its second side."""
    n, heads, shared = 8500, 8, 1040
    gen = torch.Generator(device=DEV).manual_seed(17)
    pool = torch.randn((2, 1, 65 + n, 16, heads, 64), generator=gen, device=DEV).bfloat16()
    table = torch.cat([torch.arange(65, dtype=torch.int32, device=DEV).repeat(n, 1),
                       65 + torch.arange(n, dtype=torch.int32, device=DEV)[:, None]], 1)
    lengths = torch.randint(shared, shared + 16, (n,), generator=gen, device=DEV, dtype=torch.int32)
    cache, tree = B.KVCache(pool[0], pool[1], table, lengths), B.TokenTree(1, 1)
    q = torch.randn((n, 1, heads, 64), generator=gen, device=DEV).bfloat16()
    out = B.tree_attention(cache, tree, q, shared=shared)
    some = [0, 1, 127, 128, 4000, n - 1]
    want, off = attention(pool[0, 0], pool[1, 0], table[some].tolist(), lengths[some].tolist(), [1] * len(some), [-1], q[some], 0.125)
    assert ((out[some].double().cpu() - want).abs() <= off).all()
    alone = torch.empty_like(out)
    _attend_without_workspace(cache, tree, q, alone, 0, 0)
    # either is off by half a step of the result and of the weights, whose values are below 0.8 in the mean: 2^-8 (|x| + 0.8), twice
    assert ((out.float() - alone.float()).abs() <= 2.0 ** -6 * (0.5 + alone.float().abs())).all()


@gpu
@pytest.mark.parametrize("tree,N,G,shared", [("spine", None, 7, 4112), ("chain", 16, 2, 2064), ("binary", None, 4, 4096)])
@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("fp32", 80), ("bf16", 256)])
def test_attention_longer_shared_prefix(tree, N, G, shared, dtype, dim):
    """As above, where trees of some more rows have their prefix met once."""
    N_ = _tree_of(tree, N)[3]
    _check_attention(dtype, dim, 2, G, tree, [shared, shared, shared + 12, shared + 1, shared + 113, 20, shared + 32], N=N,
                     shared=shared, counts=[N_, 1, 0, N_, min(N_, 2), 99, N_], seed=G, longest=shared + 113)


@gpu
@pytest.mark.parametrize("dtype,dim,N,G,shared", [("bf16", 64, 1, 4, 1024), ("fp32", 80, 3, 2, 1040), ("fp16", 128, 15, 4, 4112),
                                                  ("bf16", 256, 31, 4, 6160)])
def test_attention_prefix_that_fills_the_table(dtype, dim, N, G, shared):
    """Tables that end with the prefix: the nodes of sequences as long as that have no slot, and their trees no keys of their own.  What
    the workspace holds does not matter."""
    dt, page, heads = TYPES[dtype], 16, 2
    lengths = [shared, shared + 1, shared - 1, shared - N, shared - N + 1, 40, 2 ** 31 - 1, -1]
    counts = [N, N, N, N, N, N, max(1, N // 2), N]
    gen = torch.Generator().manual_seed(shared)
    pages = shared // page
    pool = torch.randn((2, 1, pages, page, heads, dim), generator=gen).to(dt).to(DEV)
    rows = torch.randperm(pages, generator=gen).to(torch.int32)
    table = rows.repeat(len(lengths), 1).to(DEV)
    cache = B.KVCache(pool[0], pool[1], table, torch.tensor(lengths, dtype=torch.int32, device=DEV))
    tree = B.TokenTree(1, N, None, torch.tensor(counts, dtype=torch.int32, device=DEV))
    q = _queries(len(lengths), N, heads * G, dim, dt, shared)
    want, off = attention(pool[0, 0], pool[1, 0], table.tolist(), lengths, counts, parents(1, N), q, dim ** -0.5, shared, rows.tolist())
    ws = B.attention_workspace(cache, tree, q, shared=shared)
    assert ws.numel() != B.attention_workspace(cache, tree, q).numel()      # (the prefix is met once)
    for fill in (0, 0x3f, 0xff):
        ws.fill_(fill)
        flags = torch.zeros(len(lengths), dtype=torch.int32, device=DEV)
        out = torch.full(q.shape, 7.5, dtype=dt, device=DEV)
        B.tree_attention(cache, tree, q, shared=shared, out=out, flags=flags, workspace=ws)
        got = out.double().cpu()
        for b, n in enumerate(counts):
            n = n if lengths[b] >= 0 else 0
            assert (got[b, n:] == 7.5).all() and ((got[b, :n] - want[b, :n]).abs() <= off[b, :n]).all(), (fill, b)
        assert flags.tolist() == [32 if n < 0 or n + c > shared else 0 for n, c in zip(lengths, counts)]


@gpu
@pytest.mark.parametrize("G,shared", [(2, 1120), (8, 2240)])
def test_attention_shared_prefix_sees_nothing_of_what_is_not_there(G, shared):
    """A shorter sequence's rows stand beside others that see the whole prefix, whose values have infinities and NaNs."""
    def change(kp, vp, table, lengths, q):
        vp[0, int(table[0, 58]), 3, :, 7] = math.inf      # slot 931
        vp[0, int(table[0, 2]), 3, :, 9] = math.nan       # slot 35
        kp[0, int(table[0, 57]), 1] = math.nan            # slot 913
    _check_attention("bf16", 64, 2, G, "binary", [shared, 932, 912, 920, 30, 0], shared=shared, seed=14, change=change, longest=shared)


@gpu
@pytest.mark.parametrize("workspace", ["own", "none"])
def test_attention_without_pages(workspace):
    """Entries outside the pool, slots behind the table, negative lengths: the keys are not there, and a flag says so."""
    flags = torch.zeros(6, dtype=torch.int32, device=DEV)

    def change(kp, vp, table, lengths, q):
        table[1, 2] = -1
        table[2, 1] = kp.shape[1]
        table[3] = -5
        lengths[4] = -3
        lengths[5] = table.shape[1] * 16 - 4    # the last nodes have no slot
        for s in range(100, int(lengths[5])):
            p = int(table[5, s // 16])
            if p >= 0:
                kp[0, p, s % 16], vp[0, p, s % 16] = 0.5, 0.25
    _check_attention("bf16", 64, 2, 2, "binary", [50, 100, 60, 40, 30, 100], seed=11, change=change, workspace=workspace, flags=flags)
    assert flags.tolist() == [0, 32, 32, 32, 32, 32]


@gpu
@pytest.mark.parametrize("dtype,G,tree,N", [("bf16", 4, "one", None), ("bf16", 4, "binary", None), ("fp16", 8, "binary5", None),
                                            ("fp32", 2, "spine", None), ("bf16", 1, "chain", 130)])
def test_attention_long_sequences(dtype, G, tree, N):
    """Sequences of several thousand slots in one call with short ones."""
    _check_attention(dtype, 64, 2, G, tree, [3000, 0, 17, 5001, 700], N=N, page_size=32, seed=12)


@gpu
@pytest.mark.parametrize("tree,G,n,heads", [("one", 3, 70, 4), ("one", 1, 256, 2), ("one", 1, 257, 2), ("one", 2, 140, 5), ("spine", 4, 70, 4),
                                            ("spine", 4, 140, 4), ("binary", 8, 33, 8)])
def test_attention_of_many_trees(tree, G, n, heads):
    """Trees enough to be taken by their lengths: equal ones, none, negative ones, trees of no nodes."""
    gen = torch.Generator().manual_seed(n)
    lengths = torch.randint(0, 300, (n,), generator=gen).tolist()
    lengths[3], lengths[5], lengths[-1], lengths[7] = 0, lengths[4], 300, 64
    N = _tree_of(tree)[3]
    counts = [N if i % 5 else i % 3 for i in range(n)]
    flags = torch.zeros(n, dtype=torch.int32, device=DEV)

    def change(kp, vp, table, lengths, q):
        lengths[2] = lengths[11] = -1
    _check_attention("bf16", 64, heads, G, tree, lengths, counts=counts, seed=n, change=change, flags=flags)
    assert [b for b in range(n) if flags[b]] == [2, 11]


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim", [72, 128, 192, 256])
@pytest.mark.parametrize("G", [2, 6])
def test_attention_long_sequences_of_long_heads(dtype, dim, G):
    """Few rows of heads of all lengths, their keys shared out in the tiles that each takes."""
    _check_attention(dtype, dim, 1, G, "ternary" if G == 2 else "one", [2500, 0, 17, 1100], page_size=32, seed=dim, order="heads")


@gpu
def test_attention_offsets_beyond_32_bits():
    """A pool of 9 GB whose last pages are in use."""
    dim, heads, page = 128, 8, 64
    pages = 5 * 2 ** 30 // (page * heads * dim)
    k = torch.empty((1, pages, page, heads, dim), dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    small_k, small_v, _, rows = make_pages([150], 3, page, heads=heads, dim=dim, dtype=torch.bfloat16, seed=13)
    used = rows[0]
    table = torch.tensor([[pages - 1 - i for i in range(len(used))]], dtype=torch.int32, device=DEV)
    for i, p in enumerate(used):
        k[0, pages - 1 - i], v[0, pages - 1 - i] = small_k[0, p], small_v[0, p]
    q = _queries(1, 3, heads, dim, torch.bfloat16, 13)
    lengths = torch.tensor([150], dtype=torch.int32, device=DEV)
    tree = B.TokenTree(1, 3)
    got = B.tree_attention(B.KVCache(k, v, table, lengths), tree, q)
    want = B.tree_attention(B.KVCache(small_k, small_v, torch.tensor([used], dtype=torch.int32, device=DEV), lengths), tree, q)
    assert torch.equal(got, want)
    new = torch.randn((1, 3, heads, dim), device=DEV).to(torch.bfloat16)
    B.kv_append(B.KVCache(k, v, table, lengths), tree, new, new)
    for n in range(3):
        assert torch.equal(v[0, table[0, (150 + n) // page].item(), (150 + n) % page], new[0, n])
    outcome = torch.tensor([[1, -1, -1]], dtype=torch.int32, device=DEV)     # the root, then its second child
    accepted = torch.tensor([1], dtype=torch.int32, device=DEV)
    assert B.kv_commit(B.KVCache(k, v, table, lengths), B.TokenTree(2, 2), outcome, accepted).tolist() == [152]
    for x in (k, v):
        for n, slot in ((0, 150), (2, 151)):
            assert torch.equal(x[0, table[0, slot // page].item(), slot % page], new[0, n])


# ---------------------------------------------------------------- appending
@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim,rot,neighbours", [(64, 64, False), (64, 64, True), (128, 32, False), (80, 80, False), (80, 40, True),
                                                (72, 12, False), (72, 6, True), (16, 0, False), (256, 256, False), (8, 2, False)])
def test_append(dtype, dim, rot, neighbours):
    _check_append(dtype, dim, rot, neighbours, "binary", [0, 1, 37, 123456, 900000])


@gpu
@pytest.mark.parametrize("tree,N", [("spine", None), ("roots", None), ("eight", None), ("chain", 40), ("chain_table", 40), ("one", None)])
def test_append_trees(tree, N):
    _check_append("bf16", 64, 64, False, tree, [5, 18, 0], N=N, page_size=3, order="heads", layers=3)
    _check_append("fp32", 64, 64, True, tree, [5, 18, 0], N=N, counts=[1, 0, 77], fused=True, in_place=True)


def _check_append(dtype, dim, rot, neighbours, tree, positions, *, N=None, page_size=16, order="slots", layers=1, counts=None,
                  fused=False, in_place=False, heads=2, G=3, seed=0):
    dt = TYPES[dtype]
    k, depth, first, N = _tree_of(tree, N)
    # far positions: only the entries behind them have pages
    small = [n % 50 for n in positions]
    base = [(n - s) // page_size * page_size for n, s in zip(positions, small)]
    kp, vp, _, rows = make_pages(small, N, page_size, layers=layers, heads=heads, dim=dim, dtype=dt, order=order, seed=seed, used=False)
    lengths = [s + f for s, f in zip(small, base)]
    width = max(f // page_size + len(r) for f, r in zip(base, rows))
    table = torch.full((len(rows), width), -1, dtype=torch.int32)
    for b, r in enumerate(rows):
        table[b, base[b] // page_size:base[b] // page_size + len(r)] = torch.tensor(r, dtype=torch.int32)
    len_t = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    cache = B.KVCache(kp, vp, table.to(DEV), len_t)
    t = B.TokenTree(k, depth, None if first is None else torch.tensor(first, dtype=torch.int32, device=DEV),
                    None if counts is None else torch.tensor(counts, dtype=torch.int32, device=DEV))
    new = _queries(len(lengths), N, heads * (G + 2), dim, dt, seed, fused)
    q, nk, nv = new[:, :, :heads * G], new[:, :, heads * G:heads * (G + 1)], new[:, :, heads * (G + 1):]
    inv = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float32) / max(1, rot // 2))
    before_k, before_v, before_q = kp.clone(), vp.clone(), q.clone()
    layer = layers - 1
    flags = torch.zeros(len(lengths), dtype=torch.int32, device=DEV)
    out = q if in_place else torch.full(q.shape, 7.5, dtype=dt, device=DEV)
    got = B.kv_append(cache, t, nk, nv, q, inv.to(DEV) if rot else None, layer=layer, neighbours=neighbours, out=out, flags=flags)
    assert got is out and not flags.any()
    level = levels(parents(k, N, first))
    want_k, want_v = before_k.double().cpu(), before_v.double().cpu()
    # each product and its sum is rounded in fp32, cosine and sine are off by 2 ulp and half an ulp of their argument:
    # 5 half steps of (|x| + |y|), then one rounding to the type
    slack = torch.zeros_like(want_k)
    c = counts or [N] * len(lengths)
    for b, n0 in enumerate(lengths):
        for n in range(N):
            if n >= c[b]:
                assert (out[b, n] == (before_q[b, n] if in_place else 7.5)).all()
                continue
            s = n0 + n
            at = (layer, int(table[b, s // page_size]), s % page_size)
            x = nk[b, n].double().cpu()
            want_k[at] = rotated(x, n0 + level[n], inv, neighbours)
            slack[at] = want_k[at].abs() * half_step(dt) + 5 * 2.0 ** -24 * 2 * x.abs().max() if rot else 0.0
            want_v[at] = nv[b, n].double().cpu()
            x = before_q[b, n].double().cpu()
            w = rotated(x, n0 + level[n], inv, neighbours)
            room = w.abs() * half_step(dt) + (5 * 2.0 ** -24 * 2 * x.abs().max() if rot else 0.0)
            assert ((out[b, n].double().cpu() - w).abs() <= room).all(), (b, n)
    got_k, got_v = kp.double().cpu(), vp.double().cpu()
    assert torch.equal(torch.isnan(got_k), torch.isnan(want_k))
    assert ((got_k - want_k).abs() <= slack)[~torch.isnan(want_k)].all()
    assert torch.equal(got_v.nan_to_num(9.0), want_v.nan_to_num(9.0))


@gpu
def test_append_without_pages_and_without_queries():
    kp, vp, table, rows = make_pages([10, 20, 30, 40], 7, 16, heads=2, dim=64, dtype=torch.bfloat16, used=False)
    table[1, 1] = 99
    lengths = torch.tensor([10, 20, -1, table.shape[1] * 16 - 3], dtype=torch.int32, device=DEV)
    cache = B.KVCache(kp, vp, table, lengths)
    x = _queries(4, 7, 2, 64, torch.bfloat16, 4)
    flags = torch.zeros(4, dtype=torch.int32, device=DEV)
    before = kp.clone()
    assert B.kv_append(cache, B.TokenTree(2, 3), x, x, flags=flags) is None
    assert flags.tolist() == [0, 32, 32, 32]
    changed = (before.nan_to_num(9.0) != kp.nan_to_num(9.0)).flatten(3).any(-1)
    slots = {(0, rows[0][(10 + n) // 16], (10 + n) % 16) for n in range(7)}
    slots |= {(0, rows[1][(20 + n) // 16], (20 + n) % 16) for n in range(7) if (20 + n) // 16 != 1}
    assert {tuple(i) for i in changed.nonzero().tolist()} == slots


# ---------------------------------------------------------------- committing
def _outcomes(B_, N, k, seed):
    gen = torch.Generator().manual_seed(seed)
    return torch.randint(-1, k, (B_, N), generator=gen, dtype=torch.int32)


@gpu
@pytest.mark.parametrize("tree,N", [("binary5", None), ("ternary", None), ("eight", None), ("spine", None), ("roots", None), ("one", None),
                                    ("chain", 100), ("chain_table", 100), ("binary7", None)])
@pytest.mark.parametrize("dtype,dim,order", [("bf16", 128, "slots"), ("fp32", 72, "heads")])
@pytest.mark.parametrize("in_place", [False, True])
def test_commit(tree, N, dtype, dim, order, in_place):
    dt = TYPES[dtype]
    k, depth, first, N = _tree_of(tree, N)
    lengths = [0, 5, 16, 31, 100, 7, 9, 12]
    kp, vp, table, rows = make_pages(lengths, N, 5, layers=3, heads=2, dim=dim, dtype=dt, order=order, seed=1)
    counts = [N, N, N, N, N, 0, max(1, N // 2), N]
    outcome = _outcomes(len(lengths), N, k, N)
    outcome[4].clamp_(min=0)
    outcome[0].fill_(k - 1)
    accept = torch.tensor([depth - 1, depth - 1, 0, 1, 10 ** 6, 2, depth - 1, -4], dtype=torch.int32)
    len_t = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    want_k, want_v, want_len = kp.clone(), vp.clone(), []
    for b, n0 in enumerate(lengths):
        path = path_of(outcome[b].tolist(), int(accept[b]), depth, k, N, counts[b], first)
        for pool, before in ((want_k, kp), (want_v, vp)):
            for i, n in enumerate(path):
                at = lambda s: (slice(None), rows[b][s // 5], s % 5)  # noqa: E731
                pool[at(n0 + i)] = before[at(n0 + n)]
        want_len.append(n0 + len(path))
    t = B.TokenTree(k, depth, None if first is None else torch.tensor(first, dtype=torch.int32, device=DEV),
                    torch.tensor(counts, dtype=torch.int32, device=DEV))
    flags = torch.zeros(len(lengths), dtype=torch.int32, device=DEV)
    got = B.kv_commit(B.KVCache(kp, vp, table, len_t), t, outcome.to(DEV), accept.to(DEV), out=len_t if in_place else None, flags=flags)
    assert got.tolist() == want_len and not flags.any()
    if not in_place:
        assert len_t.tolist() == lengths
    assert torch.equal(kp.nan_to_num(9.0), want_k.nan_to_num(9.0)) and torch.equal(vp.nan_to_num(9.0), want_v.nan_to_num(9.0))


@gpu
@pytest.mark.parametrize("depth,page_size", [(150, 5), (70, 64), (2048, 16)])
@pytest.mark.parametrize("dtype,dim,order", [("bf16", 64, "slots"), ("fp32", 24, "heads")])
@pytest.mark.parametrize("in_place", [False, True])
def test_commit_of_long_paths(depth, page_size, dtype, dim, order, in_place):
    """Paths by the second children of a deep tree: from node 2 i to slot i, so that every slot of the first half is read, written,
    or both, over many of the kernel's steps."""
    dt, N, layers, heads = TYPES[dtype], 2 * depth - 1, 2, 2
    first = [n + 1 if n % 2 == 0 and n + 2 < N else -1 for n in range(N)]
    accept = [depth - 1, 0, 1, 7, 8, 9, 62, 63, 64, 65, depth - 1, depth - 1, depth - 2]
    lengths = [3 * b for b in range(len(accept))]
    counts = [N] * len(accept)
    counts[10] = 2 * 66          # the path ends at node 130, its 66th, where the tree is deep enough for that
    outcome = torch.ones((len(accept), N), dtype=torch.int32)
    outcome[11, 2 * 67 if 67 < depth - 1 else 2 * 60] = 0      # a first child, which is a leaf
    # pages behind one another in a mixed order, every slot with a number of its own
    need = [-(-(n + N) // page_size) for n in lengths]
    gen = torch.Generator().manual_seed(depth)
    mixed = torch.randperm(sum(need) + 2, generator=gen).tolist()
    table = torch.full((len(accept), max(need)), -1, dtype=torch.int32)
    for b, n in enumerate(need):
        table[b, :n] = torch.tensor([mixed.pop() for _ in range(n)])
    shape = (layers, sum(need) + 2, page_size, heads, dim) if order == "slots" else (layers, sum(need) + 2, heads, page_size, dim)
    pools = [torch.randn(shape, generator=gen).to(dt).to(DEV) for _ in range(2)]
    if order != "slots":
        pools = [x.transpose(2, 3) for x in pools]
    want, want_len = [x.clone() for x in pools], []
    for b, n0 in enumerate(lengths):
        path = path_of(outcome[b].tolist(), accept[b], depth, 2, N, counts[b], first)
        assert len(path) > 1 or accept[b] == 0
        slots = n0 + torch.tensor([path, list(range(len(path)))])
        at, slot = table[b].long()[slots // page_size].to(DEV), (slots % page_size).to(DEV)
        for x, before in zip(want, pools):
            x[:, at[1], slot[1]] = before[:, at[0], slot[0]]
        want_len.append(n0 + len(path))
    assert want_len[0] == lengths[0] + depth
    len_t = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    flags = torch.zeros(len(accept), dtype=torch.int32, device=DEV)
    tree = B.TokenTree(2, depth, torch.tensor(first, dtype=torch.int32, device=DEV), torch.tensor(counts, dtype=torch.int32, device=DEV))
    got = B.kv_commit(B.KVCache(pools[0], pools[1], table.to(DEV), len_t), tree, outcome.to(DEV),
                      torch.tensor(accept, dtype=torch.int32, device=DEV), out=len_t if in_place else None, flags=flags)
    assert got.tolist() == want_len and not flags.any()
    assert all(torch.equal(x, y) for x, y in zip(pools, want))


@gpu
def test_commit_without_pages():
    kp, vp, table, rows = make_pages([10, 14, 30], 7, 4, heads=2, dim=64, dtype=torch.bfloat16, seed=2)
    lengths = torch.tensor([10, 14, -2], dtype=torch.int32, device=DEV)
    table[1, (14 + 6) // 4] = -1           # the last node's
    outcome = torch.ones((3, 7), dtype=torch.int32, device=DEV)
    flags = torch.zeros(3, dtype=torch.int32, device=DEV)
    before = kp.clone()
    got = B.kv_commit(B.KVCache(kp, vp, table, lengths), B.TokenTree(2, 3), outcome, torch.full((3,), 2, dtype=torch.int32, device=DEV),
                      flags=flags)
    assert got.tolist() == [13, 17, -2] and flags.tolist() == [0, 32, 32]
    at = lambda b, s: (0, rows[b][s // 4], s % 4)  # noqa: E731
    assert torch.equal(kp[at(0, 11)], before[at(0, 12)]) and torch.equal(kp[at(0, 12)], before[at(0, 16)])
    assert torch.equal(kp[at(1, 15)], before[at(1, 16)]) and torch.equal(kp[at(1, 16)], before[at(1, 16)])


@gpu
@pytest.mark.parametrize("in_place", [False, True])
def test_commit_of_lengths_that_have_no_successor(in_place):
    """Far behind the table nothing moves; the lengths stay lengths."""
    kp, vp, table, _ = make_pages([10, 10, 10], 7, 4, heads=2, dim=64, dtype=torch.bfloat16, seed=2)
    lengths = torch.tensor([2 ** 31 - 1, 2 ** 31 - 3, 2 ** 31 - 4], dtype=torch.int32, device=DEV)
    flags = torch.zeros(3, dtype=torch.int32, device=DEV)
    before = kp.clone()
    got = B.kv_commit(B.KVCache(kp, vp, table, lengths), B.TokenTree(2, 3), torch.ones((3, 7), dtype=torch.int32, device=DEV),
                      torch.full((3,), 2, dtype=torch.int32, device=DEV), out=lengths if in_place else None, flags=flags)
    assert got.tolist() == [2 ** 31 - 1] * 3 and flags.tolist() == [32] * 3
    assert torch.equal(kp.nan_to_num(9.0), before.nan_to_num(9.0))


# ---------------------------------------------------------------- together
@gpu
@pytest.mark.parametrize("tree", ["binary", "spine"])
def test_steps_of_a_decoder(tree):
    """Three steps of append, attend, verify, walk and commit: the cache ends up with the accepted tokens' keys at their
    positions, and what a tree attends to is what a reference that keeps whole sequences attends to."""
    from paper_2411_05289_amd import workloads as W
    k, depth, first, N = _tree_of(tree)
    Bn, heads, G, dim, V, page = 6, 2, 4, 64, 600, 16
    dt = torch.bfloat16
    lengths0 = [0, 3, 15, 16, 40, 77]
    kp, vp, table, rows = make_pages([n + 3 * depth for n in lengths0], N, page, heads=heads, dim=dim, dtype=dt, seed=3, used=False)
    lengths = torch.tensor(lengths0, dtype=torch.int32, device=DEV)
    cache = B.KVCache(kp, vp, table, lengths)
    table_t = None if first is None else torch.tensor(first, dtype=torch.int32, device=DEV)
    trees = B.TokenTree(k, depth, table_t)
    parent = parents(k, N, first)
    level = levels(parent)
    inv = 10000.0 ** (-torch.arange(dim // 2, dtype=torch.float32, device=DEV) / (dim // 2))
    kept_k = [[kp[0, rows[b][s // page], s % page].clone() for s in range(n)] for b, n in enumerate(lengths0)]
    for step in range(3):
        new = _queries(Bn, N, heads * (G + 2), dim, dt, 100 + step, fused=True)
        q, nk, nv = new[:, :, :heads * G], new[:, :, heads * G:heads * (G + 1)], new[:, :, heads * (G + 1):]
        now = lengths.tolist()
        assert [len(x) for x in kept_k] == now
        turned = B.kv_append(cache, trees, nk, nv, q, inv)
        out = B.tree_attention(cache, trees, turned)
        rows_now = table.cpu().tolist()
        want, off = attention(kp[0], vp[0], rows_now, now, [N] * Bn, parent, turned, dim ** -0.5)
        assert ((out.double().cpu() - want).abs() <= off).all()
        wl = W.config(3, device=DEV, B=Bn, V=V, depth=depth, seed=step) if first is None else None
        if wl is not None:
            pb = B.Problem.from_workload(wl)
        else:
            rows_t = torch.randn((Bn, N, V), device=DEV)
            pb = B.Problem(rows_t, rows_t + 0.5 * torch.randn((Bn, N, V), device=DEV), B.LOGITS, k, depth, first_child=table_t)
        u_d = B.philox_uniform(step, 1, Bn * N, k, device=DEV).view(Bn, N, k)
        u_v = B.philox_uniform(step, 2, Bn * N, k + 1, device=DEV).view(Bn, N, k + 1)
        plan = B.StepPlan("rrs", pb, u_d, u_v)
        plan.run()
        plan.commit(cache, out=lengths)
        outcome, accept = plan.out["outcome"].tolist(), plan.out["accept_depth"].tolist()
        for b in range(Bn):
            path = path_of(outcome[b], accept[b], depth, k, N, N, first)
            assert len(path) == accept[b] + 1
            for i, n in enumerate(path):
                x = rotated(nk[b, n].double().cpu(), now[b] + level[n], inv.cpu(), False)
                s = now[b] + i
                got = kp[0, rows[b][s // page], s % page]
                assert ((got.double().cpu() - x).abs() <= x.abs() * half_step(dt) + 10 * 2.0 ** -24 * nk[b, n].abs().max().item()).all()
                kept_k[b].append(got.clone())
        assert lengths.tolist() == [len(x) for x in kept_k]
        for b in range(Bn):
            for s, x in enumerate(kept_k[b]):
                assert torch.equal(kp[0, rows[b][s // page], s % page].nan_to_num(9.0), x.nan_to_num(9.0))


@gpu
def test_marshalling_in_python_gives_the_same(monkeypatch):
    """The calls marshalled by _host.so and in Python, outputs given and made, all arguments and as few as possible."""
    k, depth, first, N = _tree_of("spine")
    results = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(B, "_native", lambda: None)
        for given in (True, False):
            lengths = [5, 700, 0]
            kp, vp, table, _ = make_pages(lengths, N, 16, heads=2, dim=64, dtype=torch.bfloat16, layers=2, order="heads", seed=15)
            len_t = torch.tensor(lengths, dtype=torch.int32, device=DEV)
            cache = B.KVCache(kp, vp, table, len_t)
            tree = B.TokenTree(k, depth, torch.tensor(first, dtype=torch.int32, device=DEV),
                               torch.tensor([9, 4, 9], dtype=torch.int32, device=DEV))
            new = _queries(3, N, 8, 64, torch.bfloat16, 16)
            inv = 1.0 / torch.arange(1, 17, dtype=torch.float32, device=DEV)
            outcome = torch.zeros((3, N), dtype=torch.int32, device=DEV)
            accept = torch.tensor([4, 1, 0], dtype=torch.int32, device=DEV)
            kw = [{}, {}, {}]
            if given:
                flags = torch.zeros(3, dtype=torch.int32, device=DEV)
                q_out, out = torch.zeros((3, N, 4, 64), dtype=torch.bfloat16, device=DEV), torch.zeros((3, N, 4, 64), dtype=torch.bfloat16, device=DEV)
                ws = B.attention_workspace(cache, tree, q_out, longest=700)
                kw = [dict(out=q_out, flags=flags), dict(out=out, flags=flags, workspace=ws, scale=0.125, longest=700),
                      dict(out=torch.zeros_like(len_t), flags=flags)]
            turned = B.kv_append(cache, tree, new[:, :, 4:6], new[:, :, 6:8], new[:, :, :4], inv, layer=1, neighbours=True, **kw[0])
            assert B.kv_append(cache, tree, new[:, :, 4:6], new[:, :, 6:8]) is None
            out = B.tree_attention(cache, tree, turned, layer=1, shared=0, **kw[1])
            after = B.kv_commit(cache, tree, outcome, accept, **kw[2])
            if given:
                assert turned is kw[0]["out"] and out is kw[1]["out"] and after is kw[2]["out"] and not flags.any()
            results.append((turned, out, after, kp.nan_to_num(9.0), vp.nan_to_num(9.0)))
    for r in results[1:]:
        for x, y in zip(r, results[0]):
            assert torch.equal(x, y)


@gpu
def test_prompt_and_tokens_agree():
    """A prompt as one tree, as two, and token by token: the same keys, and results within their rounding."""
    dim, heads, G, n, dt = 64, 2, 2, 150, torch.float32
    new = _queries(1, n, heads * (G + 2), dim, dt, 5)
    q, nk, nv = new[:, :, :heads * G], new[:, :, heads * G:heads * (G + 1)], new[:, :, heads * (G + 1):]
    inv = 10000.0 ** (-torch.arange(dim // 2, dtype=torch.float32, device=DEV) / (dim // 2))
    results = []
    for cuts in ([0, n], [0, 67, n], list(range(n + 1))):
        kp, vp, table, _ = make_pages([0], n, 16, heads=heads, dim=dim, dtype=dt, seed=6, used=False)
        lengths = torch.zeros(1, dtype=torch.int32, device=DEV)
        cache = B.KVCache(kp, vp, table, lengths)
        outs = []
        for a, z in zip(cuts, cuts[1:]):
            t = B.TokenTree(1, z - a)
            turned = B.kv_append(cache, t, nk[:, a:z], nv[:, a:z], q[:, a:z], inv)
            outs.append(B.tree_attention(cache, t, turned))
            lengths += z - a
        results.append((torch.cat(outs, 1), kp.nan_to_num(9.0)))
    for out, keys in results[1:]:
        assert torch.equal(keys, results[0][1])
        # both are within about (n + 64 + 2 (dim + 4) max|q.k| scale) half steps of the values' size
        assert (out - results[0][0]).abs().max() < 2 * (n + 64 + 2 * (dim + 4) * 40) * 2.0 ** -24 * float(nv.abs().max())


@gpu
def test_captured_and_replayed_on_another_stream():
    """A step's three calls in a graph whose lengths go on from replay to replay, against the same calls made eagerly."""
    dim, heads, G, dt = 128, 2, 4, torch.bfloat16
    k, depth, first, N = _tree_of("binary")
    lengths0 = [100, 3000, 17]

    def world():
        kp, vp, table, _ = make_pages([n + 5 * depth for n in lengths0], N, 16, heads=heads, dim=dim, dtype=dt, seed=7)
        lengths = torch.tensor(lengths0, dtype=torch.int32, device=DEV)
        new = _queries(3, N, heads * (G + 2), dim, dt, 8)
        return dict(cache=B.KVCache(kp, vp, table, lengths), q=new[:, :, :heads * G], k=new[:, :, heads * G:heads * (G + 1)],
                    v=new[:, :, heads * (G + 1):], turned=torch.zeros((3, N, heads * G, dim), dtype=dt, device=DEV),
                    out=torch.zeros((3, N, heads * G, dim), dtype=dt, device=DEV), outcome=_outcomes(3, N, k, 9).to(DEV),
                    accept=torch.tensor([2, 3, 0], dtype=torch.int32, device=DEV))

    inv = 10000.0 ** (-torch.arange(dim // 2, dtype=torch.float32, device=DEV) / (dim // 2))
    tree = B.TokenTree(k, depth)

    def step(w):
        B.kv_append(w["cache"], tree, w["k"], w["v"], w["q"], inv, out=w["turned"])
        B.tree_attention(w["cache"], tree, w["turned"], out=w["out"])
        B.kv_commit(w["cache"], tree, w["outcome"], w["accept"], out=w["cache"].lengths)

    a, b = world(), world()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            step(b)
    for replay in range(4):
        step(a)
        with torch.cuda.stream(stream):
            graph.replay()
        stream.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(a["out"], b["out"]) and torch.equal(a["cache"].lengths, b["cache"].lengths), replay
        assert torch.equal(a["cache"].k.nan_to_num(9.0), b["cache"].k.nan_to_num(9.0))
        for w in (a, b):
            w["q"].mul_(1.0009765625 if replay % 2 else 0.5)


@gpu
@pytest.mark.parametrize("axis", [0, 1, 2, (0, 1, 2)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_repeated_inputs(axis, dtype):
    """Inputs with strides of zero: the same bits as their copies give."""
    dt, axes = TYPES[dtype], (axis,) if isinstance(axis, int) else axis
    k, depth, _, N = _tree_of("binary")
    lengths = [70, 3, 900]
    results = []
    for repeated in (True, False):
        kp, vp, table, _ = make_pages(lengths, N, 16, heads=2, dim=64, dtype=dt, seed=16)
        cache = B.KVCache(kp, vp, table, torch.tensor(lengths, dtype=torch.int32, device=DEV))
        x = []
        for heads in (8, 2, 2):
            shape = [3, N, heads, 64]
            small = _queries(*[1 if a in axes else n for a, n in enumerate(shape[:3])], 64, dt, heads)
            x.append(small.expand(shape) if repeated else small.expand(shape).contiguous())
        turned = B.kv_append(cache, B.TokenTree(k, depth), x[1], x[2], x[0], 1.0 / torch.arange(1, 33, dtype=torch.float32, device=DEV))
        results.append((turned, B.tree_attention(cache, B.TokenTree(k, depth), x[0]), kp.nan_to_num(9.0), vp.nan_to_num(9.0)))
    for a, b in zip(*results):
        assert torch.equal(a, b)


@gpu
def test_two_streams_at_once():
    """Calls that overlap in time, each with its own cache and workspace: what each gives alone."""
    def world(seed):
        k, depth, _, N = _tree_of("binary5")
        lengths = [4000, 30, 900, 0]
        kp, vp, table, _ = make_pages([n + 8 * depth for n in lengths], N, 16, heads=4, dim=128, dtype=torch.bfloat16, seed=seed)
        cache = B.KVCache(kp, vp, table, torch.tensor(lengths, dtype=torch.int32, device=DEV))
        new = _queries(4, N, 24, 128, torch.bfloat16, seed)
        return cache, B.TokenTree(k, depth), new, _outcomes(4, N, k, seed).to(DEV), torch.full((4,), depth, dtype=torch.int32, device=DEV)

    def steps(w, stream):
        cache, tree, new, outcome, accept = w
        outs = []
        with torch.cuda.stream(stream):
            for _ in range(6):
                turned = B.kv_append(cache, tree, new[:, :, 16:20], new[:, :, 20:], new[:, :, :16])
                outs.append(B.tree_attention(cache, tree, turned))
                B.kv_commit(cache, tree, outcome, accept, out=cache.lengths)
            return outs + [cache.lengths, cache.k.nan_to_num(9.0), cache.v.nan_to_num(9.0)]

    alone = []
    for seed in (1, 2):
        w = world(seed)
        torch.cuda.synchronize()
        alone.append(steps(w, torch.cuda.current_stream()))
        torch.cuda.synchronize()
    worlds, streams = [world(1), world(2)], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    together = [steps(w, s) for w, s in zip(worlds, streams)]
    torch.cuda.synchronize()
    for a, b in zip(alone, together):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
