"""A long context in a small cache: keys and values in 4 bits, given positions, slots' weights, eviction.  What the calls refuse (CPU),
and what they give against 64-bit references (GPU)."""
import ctypes as C
import math

import pytest
import torch

from paper_2411_05289_amd import binding as B
from kv_long_reference import VALUES, block_of, in_four, kept_of, lse_of, values_of, weigh
from kv_reference import SPINE, TYPES, attention, half_step, levels, make_pages, parents, path_of, rotated
from test_kv_cache import _cache, _heads, _outcomes, _queries, _tree, _tree_of

gpu = pytest.mark.gpu
DEV = "cuda"


# ---------------------------------------------------------------- refusals (nothing is launched)
def _four(**kw):
    return _cache(**{**dict(dtype=B.FP4), **kw})


def _scales(**kw):
    s = B._Scales(0xD0001, 0xE0003, B.BF16)     # of any alignment
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _rotary(**kw):
    r = B._Rotary()
    r.inv_freq, r.rot = 0x60000, 64
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def _ref(x):
    return None if x is None else C.byref(x)


FOUR = object()


def _append(cache=None, scales=FOUR, tree=None, k=None, v=None, q=None, q_out=None, rotary=FOUR, k_out=None, v_out=None, layer=0, flags=None):
    scales = _scales() if scales is FOUR else scales
    rotary = _rotary() if rotary is FOUR else rotary
    return B.lib().mdsd_kv_append_at(C.byref(cache or _four()), _ref(scales), layer, C.byref(tree or _tree()), C.byref(k or _heads()),
                                     C.byref(v or _heads()), _ref(q), _ref(q_out), _ref(rotary), _ref(k_out), _ref(v_out), flags, None)


def _attend(cache=None, scales=FOUR, tree=None, q=None, out=None, scale=0.125, shared_pages=None, shared=0, longest=0, layer=0, lse=None,
            flags=None, ws=None, ws_bytes=0):
    scales = _scales() if scales is FOUR else scales
    return B.lib().mdsd_tree_attention_lse(C.byref(cache or _four()), _ref(scales), layer, C.byref(tree or _tree()), C.byref(q or _heads(4)),
                                           C.byref(out or _heads(4, p=0x70000)), scale, shared_pages, shared, longest, lse, flags, ws,
                                           ws_bytes, None)


def _commit(cache=None, scales=FOUR, tree=None, outcome=0x80000, accept_depth=0x90000, new_lengths=0xA0000):
    scales = _scales() if scales is FOUR else scales
    return B.lib().mdsd_kv4_commit(C.byref(cache or _four()), _ref(scales), C.byref(tree or _tree()), outcome, accept_depth, new_lengths,
                                   None, None)


def _weigh(cache=None, scales=FOUR, tree=None, q=None, lse=0x110000, scale=0.125, outcome=None, accept_depth=None, weights=0x120000,
           ld_weights=100, out=0x130000, ld_out=100, slots=64, layer=0, flags=None):
    scales = _scales() if scales is FOUR else scales
    return B.lib().mdsd_kv_weigh(C.byref(cache or _four()), _ref(scales), layer, C.byref(tree or _tree()), C.byref(q or _heads(4)), lse,
                                 scale, outcome, accept_depth, weights, ld_weights, out, ld_out, slots, flags, None)


def _evict(cache=None, scales=FOUR, n=1, weights=0x120000, ld_weights=100, slots=64, budget=8, first=2, recent=3, new_lengths=0xA0000,
           kept=0x140000, weights_out=0x130000, ld_out=100, flags=None, tree=None):
    scales = _scales() if scales is FOUR else scales
    return B.lib().mdsd_kv_evict(C.byref(cache or _four()), _ref(scales), n, weights, ld_weights, slots, budget, first, recent,
                                 new_lengths, kept, weights_out, ld_out, flags, None)


@pytest.mark.parametrize("call", [_append, _attend, _commit, _weigh, _evict])
@pytest.mark.parametrize("kw,code", [
    (dict(k=None), -1), (dict(v=None), -1), (dict(table=None), -1), (dict(lengths=None), -1), (dict(dtype=4), -5), (dict(dtype=B.BF16), -5),
    (dict(layers=0), -2), (dict(pages=0), -2), (dict(page_size=0), -2), (dict(heads=0), -2), (dict(table_pages=0), -2),
    (dict(dim=0), -2), (dict(dim=48), -2), (dict(dim=288), -2), (dict(ld_table=3), -2), (dict(page_size=1 << 29), -2),
    (dict(k=0x10008), -6), (dict(v=0x20002), -6), (dict(ld_slot=65), -6), (dict(ld_slot=144), -6), (dict(ld_page=-32), -6), (dict(ld_head=16), -6),
    (dict(ld_page=1 << 37), -2), (dict(ld_slot=1 << 37), -2), (dict(ld_layer=1 << 48), -6),
    (dict(table=0x30001), -6), (dict(lengths=0x40002), -6),
])
def test_bad_caches_are_refused(call, kw, code):
    assert call(cache=_four(**kw)) == code


@pytest.mark.parametrize("call", [_append, _attend, _commit, _weigh, _evict])
@pytest.mark.parametrize("kw,code", [(dict(k=None), -1), (dict(v=None), -1), (dict(dtype=B.FP4), -5), (dict(dtype=-1), -5)])
def test_bad_scales_are_refused(call, kw, code):
    assert call(scales=_scales(**kw)) == code


@pytest.mark.parametrize("call,code", [(_append, -5), (_attend, -5), (_commit, -1), (_weigh, -5), (_evict, -5)])
def test_four_bits_without_scales_are_refused(call, code):
    assert call(scales=None) == code


@pytest.mark.parametrize("call", [_append, _attend, _commit, _weigh])
@pytest.mark.parametrize("kw,code", [
    (dict(B=-1), -2), (dict(N=0), -2), (dict(N=6), -2), (dict(depth=0), -2), (dict(k=0, N=1), -3), (dict(k=9), -3),
    (dict(k=1), -2), (dict(N=4097, first_child=0xB0000), -2), (dict(first_child=0xB0002), -6), (dict(counts=0xC0003), -6),
])
def test_bad_trees_are_refused(call, kw, code):
    assert call(tree=_tree(**kw)) == code


@pytest.mark.parametrize("kw,code", [
    (dict(k=_heads(4)), -2), (dict(v=_heads(4)), -2), (dict(q=_heads(4)), -1), (dict(q_out=_heads(4)), -1), (dict(layer=2), -2), (dict(layer=-1), -2),
    (dict(rotary=_rotary(rot=66)), -2), (dict(rotary=_rotary(rot=63)), -2), (dict(rotary=_rotary(style=2)), -5), (dict(rotary=_rotary(inv_freq=None)), -1),
    (dict(rotary=_rotary(positions=0xF0000)), -2), (dict(rotary=_rotary(positions=0xF0000, axes=9)), -2),
    (dict(rotary=_rotary(positions=0xF0002, axes=1)), -6), (dict(rotary=_rotary(positions=0xF0000, axes=1, per_node=2)), -2),
    (dict(rotary=_rotary(positions=0xF0000, axes=1, ld_tree=-1)), -2), (dict(rotary=_rotary(positions=0xF0000, axes=1, ld_axis=-1)), -2),
    (dict(k_out=_heads()), -6), (dict(k_out=_heads(p=0x50080)), -6), (dict(k_out=_heads(4, p=0x90000)), -2), (dict(v_out=_heads(4, p=0x90000)), -2),
    (dict(v_out=_heads(p=0x50080)), -6), (dict(v_out=_heads(p=0x90000, ld_head=0)), -2), (dict(flags=2), -6),
    (dict(cache=_cache(), scales=None, k_out=_heads(p=0x90000)), -9), (dict(cache=_cache(), scales=None, v_out=_heads(p=0x90000)), -9),
    (dict(cache=_four(ld_slot=0)), -2), (dict(tree=_tree(B=1 << 24, N=1, k=1, depth=1)), -2),
])
def test_appends_that_are_refused(kw, code):
    assert _append(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(lse=0x110002), -6), (dict(q=_heads(3), out=_heads(3, p=0x70000)), -2), (dict(q=_heads(4), out=_heads(2, p=0x70000)), -2),
    (dict(scale=0.0), -4), (dict(shared=16), -1), (dict(shared=65, shared_pages=0xF0000), -2), (dict(ws=0x1008, ws_bytes=1 << 40), -6),
    (dict(layer=2), -2), (dict(out=_heads(4, p=0x50040)), -6), (dict(longest=-1), -2),
])
def test_attentions_that_are_refused(kw, code):
    assert _attend(**kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(lse=None), -1), (dict(out=None), -1), (dict(outcome=0x80000), -1), (dict(accept_depth=0x80000), -1), (dict(q=_heads(3)), -2),
    (dict(layer=2), -2), (dict(slots=0), -2), (dict(slots=101), -2), (dict(ld_out=63), -2), (dict(scale=0.0), -4), (dict(scale=math.nan), -4),
    (dict(weights=0x120002), -6), (dict(out=0x130001), -6), (dict(lse=0x110001), -6), (dict(out=0x120004), -6), (dict(out=0x120000 - 4 * 63), -6),
    (dict(tree=_tree(B=2), out=0x120000 + 4 * 100 - 4), -6), (dict(tree=_tree(B=2), out=0x120000, ld_out=200), -6), (dict(flags=1), -6),
    (dict(slots=1 << 30, ld_weights=1 << 30, ld_out=1 << 30, tree=_tree(B=64), out=1 << 50), -2),
])
def test_weighings_that_are_refused(kw, code):
    assert _weigh(**kw) == code


@pytest.mark.parametrize("four,B_,slots,kv_heads,heads,tree", [
    (True, 2, 1 << 30, 2, 4, {}), (False, 1 << 14, 1 << 17, 2, 4, {}),                     # few rows: stretches of 256 slots
    (True, 1 << 8, 1 << 20, 64, 64, {}), (False, 1 << 7, 1 << 20, 64, 64, {}),             # of many heads: of 32, of 16
    (True, 1 << 9, 1 << 20, 2, 256, dict(N=31, depth=5)), (False, 1 << 9, 1 << 20, 2, 256, dict(N=31, depth=5)),   # many rows: of 64
    (True, 1 << 9, 1 << 20, 8, 64, dict(N=31, depth=5)),                                   # by eight waves
])
def test_weighings_of_too_many_workgroups_are_refused(four, B_, slots, kv_heads, heads, tree):
    """2^23, whichever kernel it is."""
    kw = dict(cache=_four(heads=kv_heads), scales=_scales()) if four else dict(cache=_cache(heads=kv_heads), scales=None)
    q = _heads(heads, ld_tree=31 * heads * 64)
    assert _weigh(tree=_tree(B=B_, **tree), q=q, slots=slots, weights=None, ld_out=slots, out=1 << 50, **kw) == -2


@pytest.mark.parametrize("kw,code", [
    (dict(weights=None), -1), (dict(new_lengths=None), -1), (dict(kept=None), -1), (dict(n=-1), -2), (dict(slots=0), -2), (dict(budget=0), -2),
    (dict(first=-1), -2), (dict(recent=-1), -2), (dict(first=6), -2), (dict(budget=(1 << 30) + 1), -2), (dict(ld_weights=63), -2), (dict(ld_out=63), -2),
    (dict(weights=0x120002), -6), (dict(kept=0x140002), -6), (dict(weights_out=0x130002), -6), (dict(new_lengths=0xA0002), -6),
    (dict(new_lengths=0x40004, n=2), -6), (dict(weights_out=0x120004), -6), (dict(cache=_four(ld_head=0)), -2), (dict(n=1 << 23, weights_out=None, new_lengths=1 << 40), -2),
    (dict(flags=3), -6),
])
def test_evictions_that_are_refused(kw, code):
    assert _evict(**kw) == code


def test_empty_batches():
    for call in (_append, _attend, _commit, _weigh):
        assert call(cache=_four(k=None, dtype=9), tree=_tree(B=0)) == 0
    assert _evict(n=0, weights=None) == 0
    L = B.lib()
    assert L.mdsd_tree_attention_lse_workspace_bytes(C.byref(_four()), None, C.byref(_tree()), 4, 0, 0) == 0
    assert L.mdsd_tree_attention_lse_workspace_bytes(C.byref(_four()), C.byref(_scales()), C.byref(_tree()), 3, 0, 0) == 0
    long = dict(table_pages=8192, ld_table=8192)
    assert L.mdsd_tree_attention_lse_workspace_bytes(C.byref(_four(**long)), C.byref(_scales()), C.byref(_tree()), 4, 0, 0) > 0


def test_binding_refuses_what_is_not_on_the_gpu():
    k, v, ks, vs = B.pages_in_4_bits(1, 4, 16, 2, 64, device="cpu")
    cache = B.KVCache(k, v, torch.zeros((1, 4), dtype=torch.int32), torch.zeros(1, dtype=torch.int32), ks, vs)
    x, tree = torch.zeros((1, 7, 2, 64), dtype=torch.bfloat16), B.TokenTree(2, 3)
    for call in (lambda: B.kv_append(cache, tree, x, x), lambda: B.tree_attention(cache, tree, x),
                 lambda: B.kv_commit(cache, tree, torch.zeros((1, 7), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)),
                 lambda: B.kv_weigh(cache, tree, x, torch.zeros((1, 7, 2)), torch.zeros((1, 64))),
                 lambda: B.kv_evict(cache, torch.zeros((1, 64)), 8)):
        with pytest.raises(ValueError):
            call()


def test_reference_takes_the_nearest_value():
    """The encoding that the GPU's is compared with: every value stands for itself, nothing is nearer, ties are even."""
    for e in (-3, 0, 5):
        for c, w in enumerate(VALUES):
            x = [0.0] * 32
            x[0], x[1], x[7] = 6 * 2.0 ** e, w * 2.0 ** e, -w * 2.0 ** e
            codes, scale = block_of(x, torch.float32)
            assert scale == e + 127 and codes[0] == 7 + 16 * c and codes[3] >> 4 == 8 + c
    assert block_of([7.0] + [5.0, 2.5, 0.25, 0.75, 1.75, 3.5, 1.25] + [0.0] * 24, torch.float32)[0][:4] == [0x67, 0x04, 0x42, 0x26]
    assert block_of([7.01] + [0.0] * 31, torch.float32) == ([6] + [0] * 15, 128)
    assert block_of([math.inf] + [1.0] * 31, torch.float32) == ([0] * 16, 255)
    assert block_of([60000.0] + [0.0] * 31, torch.float16) == ([7] + [0] * 15, 140)


# ---------------------------------------------------------------- attention
def _pages(lengths, N, page_size, *, heads=2, dim=64, dtype=torch.bfloat16, order="slots", layers=1, shared=0, seed=0, spare=2, used=True):
    """make_pages in 4 bits: -> codes and scales of k and v, the table, its rows, and both pools as numbers.  What is not in use is NaN."""
    kp, vp, table, rows = make_pages(lengths, N, page_size, layers=layers, heads=heads, dim=dim, dtype=dtype, order="slots", shared=shared,
                                     seed=seed, device="cpu", spare=spare, used=used)
    got = []
    for pool in (kp, vp):
        # by torch, as pools are large; what it gives is checked against the loops above in test_append_in_four_bits
        codes, scales = _encode(pool.float(), dtype)
        if order == "heads":
            codes, scales = (x.transpose(2, 3).contiguous().transpose(2, 3) for x in (codes, scales))
        got += [codes, scales]
    kc, ks, vc, vs = ((x.to(DEV) if order == "slots" else x.transpose(2, 3).to(DEV).transpose(2, 3)) for x in got)
    return kc, vc, ks, vs, table.to(DEV), rows


def _encode(x, dtype):
    from kv_long_reference import EXPONENTS
    lo, hi = EXPONENTS[dtype]
    blocks = x.unflatten(-1, (-1, 32)).double()
    most = blocks.abs().amax(-1, keepdim=True)
    fine = torch.isfinite(most)
    e = torch.full_like(most, float(lo))
    for n in range(lo, hi):
        e = torch.where(most > 7 * 2.0 ** n, float(n + 1), e)
    y = blocks.abs() / 2.0 ** e
    code = (y > 0.25).int() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0) + 8 * torch.signbit(blocks).int()
    code = torch.where(fine, code, 0).flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), torch.where(fine, e + 127, 255.0).to(torch.uint8).squeeze(-1)


def _trees(tree, N, counts=None):
    k, depth, first, N = _tree_of(tree, N)
    t = B.TokenTree(k, depth, None if first is None else torch.tensor(first, dtype=torch.int32, device=DEV),
                    None if counts is None else torch.tensor(counts, dtype=torch.int32, device=DEV))
    return t, N, parents(k, N, first), first


def _attend_raw(cache, tree, q, out, lse, layer, shared, flags=None):
    """Without a workspace."""
    c, t = B._c_cache(cache), B._c_tree(tree, q.shape[0], q.shape[1])
    qh, oh = B._c_heads("q", q, cache), B._c_heads("out", out, cache)
    rc = B.lib().mdsd_tree_attention_lse(C.byref(c), B._scales_ref(cache, q), layer, C.byref(t), C.byref(qh), C.byref(oh), q.shape[3] ** -0.5,
                                         B._ptr(cache.table[0]), shared, 0, B._ptr(lse), B._ptr(flags), None, 0, B._stream())
    assert rc == 0


def _check_attention(dtype, dim, heads, G, tree, lengths, *, N=None, page_size=16, order="slots", counts=None, layers=1, shared=0, seed=0,
                     change=None, four=True, longest=0, flags=None):
    dt = TYPES[dtype]
    t, N, parent, _ = _trees(tree, N, counts)
    if four:
        kc, vc, ks, vs, table, _ = _pages(lengths, N, page_size, heads=heads, dim=dim, dtype=dt, order=order, layers=layers, shared=shared, seed=seed)
    else:
        kc, vc, table, _ = make_pages(lengths, N, page_size, layers=layers, heads=heads, dim=dim, dtype=dt, order=order, shared=shared, seed=seed)
        ks = vs = None
    len_t = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    q = _queries(len(lengths), N, heads * G, dim, dt, seed, fused=True)
    if change is not None:
        change(kc, vc, ks, vs, table, len_t, q)
    layer = layers - 1
    kv, vv = (values_of(kc[layer], ks[layer]), values_of(vc[layer], vs[layer])) if four else (kc[layer], vc[layer])
    # by the longest that sequences may be: as told; with tables that would hold long ones, shared out and not
    wider = torch.cat([table, torch.full((len(lengths), 140000 // page_size), -1, dtype=torch.int32, device=DEV)], 1)
    outs = [torch.full((len(lengths), N, heads * G, dim), 7.5, dtype=dt, device=DEV) for _ in range(3)]
    sums = [torch.full((len(lengths), N, heads * G), 7.5, device=DEV) for _ in range(3)]
    cache, wide = B.KVCache(kc, vc, table, len_t, ks, vs), B.KVCache(kc, vc, wider, len_t, ks, vs)
    B.tree_attention(cache, t, q, layer=layer, shared=shared, out=outs[0], longest=longest, flags=flags, lse=sums[0])
    B.tree_attention(wide, t, q, layer=layer, shared=shared, shared_pages=table[0], out=outs[1], flags=flags, lse=sums[1])
    _attend_raw(wide, t, q, outs[2], sums[2], layer, shared, flags)
    torch.cuda.synchronize()
    c = counts or [N] * len(lengths)
    rows = table.cpu().tolist()
    assert shared == 0 or all(r[:shared // page_size] == rows[0][:shared // page_size] for r in rows)
    want, off = attention(kv, vv, rows, len_t.tolist(), c, parent, q, dim ** -0.5)
    want_sum, off_sum = lse_of(kv, rows, len_t.tolist(), c, parent, q, dim ** -0.5)
    for got, o, w in [(x.double().cpu(), off, want) for x in outs] + [(x.double().cpu(), off_sum, want_sum) for x in sums]:
        for b in range(len(lengths)):
            m = max(0, min(N, c[b])) if len_t[b] >= 0 else 0
            assert (got[b, m:] == 7.5).all(), ("rows behind the last", b)
            x, y, room = w[b, :m], got[b, :m], o[b, :m]
            fine = torch.isfinite(x)
            assert torch.equal(torch.isnan(x), torch.isnan(y)) and torch.equal(x[~fine & ~torch.isnan(x)], y[~fine & ~torch.isnan(x)])
            wrong = (x - y).abs() > room
            assert not (wrong & fine).any(), (b, wrong.nonzero()[:4].tolist(), float(((x - y).abs() / room)[fine].max()))
    return outs[0], sums[0]


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 160, 192, 256])
def test_attention_types_and_dims(dtype, dim):
    _check_attention(dtype, dim, 2, 4, "binary", [0, 1, 63, 64, 65, 200], seed=dim)


@gpu
@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("fp16", 64), ("fp32", 96), ("bf16", 192)])
@pytest.mark.parametrize("tree,N,G", [("one", None, 1), ("one", None, 4), ("one", None, 20), ("spine", None, 3), ("roots", None, 4), ("binary5", None, 4),
                                      ("ternary", None, 5), ("chain", 150, 2), ("chain_table", 70, 1)])
def test_attention_trees(dtype, dim, tree, N, G):
    _check_attention(dtype, dim, 2, G, tree, [0, 7, 130], N=N, page_size=24, order="heads", layers=2, seed=1)


@gpu
@pytest.mark.parametrize("page_size", [1, 16, 48, 257])
@pytest.mark.parametrize("order", ["slots", "heads"])
def test_attention_pages(page_size, order):
    _check_attention("bf16", 128, 3, 2, "binary", [300, 5, 77], page_size=page_size, order=order, seed=2)


@gpu
@pytest.mark.parametrize("dtype,dim,heads,G,tree,page_size,lengths", [
    ("bf16", 128, 8, 4, "one", 16, [(37 * b) % 300 for b in range(70)]), ("fp16", 64, 16, 1, "spine", 5, [(91 * b) % 140 for b in range(33)]),
    ("bf16", 128, 8, 4, "binary5", 16, [(53 * b) % 200 for b in range(70)]), ("fp32", 96, 12, 2, "binary", 1, [(29 * b) % 90 for b in range(40)]),
    ("bf16", 192, 3, 3, "chain", 16, [0, 1, 700, 65])])
def test_attention_of_all_heads_of_a_unit_at_a_time(dtype, dim, heads, G, tree, page_size, lengths):
    """Heads that lie side by side, of numbers of units that no XCD's share divides."""
    _check_attention(dtype, dim, heads, G, tree, lengths, N=70 if tree == "chain" else None, page_size=page_size, seed=11)


@gpu
def test_attention_into_its_queries_place():
    """Results where the queries stand: by each kernel, shared out and not."""
    for tree, dim, heads, G, lengths in (("binary", 128, 2, 4, [300, 5, 77]), ("binary", 96, 4, 1, [20, 0, 9]), ("one", 128, 2, 4, [6000, 40, 0]),
                                         ("binary5", 128, 2, 4, [4000, 5, 77]), ("binary7", 64, 8, 2, [700, 0, 31])):
        t, N, _, _ = _trees(tree, None)
        kc, vc, ks, vs, table, _ = _pages(lengths, N, 16, heads=heads, dim=dim, seed=12)
        cache = B.KVCache(kc, vc, table, torch.tensor(lengths, dtype=torch.int32, device=DEV), ks, vs)
        q = _queries(3, N, heads * G, dim, torch.bfloat16, 12)
        want = B.tree_attention(cache, t, q)
        assert B.tree_attention(cache, t, q, out=q) is q and torch.equal(q, want)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_of_fewer_nodes(dtype):
    _check_attention(dtype, 64, 2, 3, "binary", [100, 3, 0, 40, 9], counts=[15, 1, 7, 0, -3], seed=3)
    _check_attention(dtype, 64, 2, 3, "chain", [100, 3, 0, 40], N=300, counts=[300, 1, 77, 0], seed=3)


@gpu
@pytest.mark.parametrize("dtype,dim,tree,N,G", [("bf16", 128, "one", None, 4), ("fp16", 128, "binary5", None, 4), ("fp32", 128, "spine", None, 2),
                                                ("bf16", 256, "binary", None, 3), ("bf16", 64, "ternary", None, 2)])
def test_attention_long_sequences(dtype, dim, tree, N, G):
    _check_attention(dtype, dim, 2, G, tree, [6000, 1, 2500], N=N, seed=4, order="heads", longest=6000)


@gpu
@pytest.mark.parametrize("dtype,G,tree,shared", [("bf16", 4, "one", 1040), ("fp32", 2, "spine", 1040), ("fp16", 4, "binary", 4112)])
def test_attention_shared_prefix(dtype, G, tree, shared):
    _check_attention(dtype, 64, 2, G, tree, [shared + n for n in (0, 3, 40, 64, 9, 21)], shared=shared, seed=5)


@gpu
@pytest.mark.parametrize("dtype,dim,order,G,tree,shared", [
    *((dtype, dim, order, 4, "one", 1040) for dtype in ("bf16", "fp16", "fp32") for dim, order in ((96, "heads"), (128, "slots"), (160, "heads"), (256, "slots"))),
    ("fp16", 128, "heads", 4, "binary", 4112), ("bf16", 192, "slots", 4, "binary5", 6160)])
def test_attention_shared_prefix_of_longer_heads(dtype, dim, order, G, tree, shared):
    """Prefixes that are met once, by all rows together: the workspace has room for them."""
    def change(kc, vc, ks, vs, table, lengths, q):
        cache, t = B.KVCache(kc, vc, table, lengths, ks, vs), _trees(tree, None)[0]
        assert B.attention_workspace(cache, t, q, shared=shared).numel() > B.attention_workspace(cache, t, q).numel()
    _check_attention(dtype, dim, 2, G, tree, [shared + n for n in (0, 3, 40, 64, 9, 21)], shared=shared, order=order, change=change, seed=21)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim", [128, 160, 192, 256])
@pytest.mark.parametrize("tree,N,G", [("binary5", None, 4), ("binary", None, 4), ("chain", 90, 3)])
def test_attention_of_many_rows_of_longer_heads(dtype, dim, tree, N, G):
    """By 128 rows a workgroup and by 64, shared out and not: sequences that are too long for 16 rows a workgroup."""
    _check_attention(dtype, dim, 2, G, tree, [6000, 1, 700], N=N, order="heads" if dim % 64 else "slots", seed=22)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim", [96, 128, 160, 256])
@pytest.mark.parametrize("tree,N,G", [("one", None, 2), ("spine", None, 3), ("binary", None, 4), ("binary5", None, 4), ("chain", 90, 3)])
def test_attention_of_blocks_that_are_no_numbers_in_longer_heads(dtype, dim, tree, N, G):
    def change(kc, vc, ks, vs, table, lengths, q):
        n, nodes = int(lengths[0]), q.shape[1]
        vs[0, int(table[0, (n + nodes - 1) // 16]), (n + nodes - 1) % 16, 0, dim // 32 - 1] = 255
        vs[0, int(table[0, 0]), 7, 1, 0] = 255
        vs[0, int(table[1, 0]), 3, 1, 1] = 255
        ks[0, int(table[2, 0]), 2, 1, dim // 32 - 1] = 255
        ks[0, int(table[3, (70 + nodes - 1) // 16]), (70 + nodes - 1) % 16, 0, 0] = 255
        table[1, 2] = -1
    _check_attention(dtype, dim, 2, G, tree, [20, 1000, 9, 70], N=N, change=change, seed=23)


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("tree,N,G", [("one", None, 2), ("binary5", None, 4), ("chain", 90, 3)])
def test_attention_of_blocks_that_are_no_numbers(dtype, tree, N, G):
    """A NaN block of a value reaches the rows that see it, in its own elements, and no other; of a key all that see it; slots
    that nobody sees hold nothing but NaN anyway."""
    def change(kc, vc, ks, vs, table, lengths, q):
        n = int(lengths[0])
        # the first sequence's last node: seen by itself alone; the second one's slot 3: by all
        nodes = q.shape[1]
        p = int(table[0, (n + nodes - 1) // 16])
        vs[0, p, (n + nodes - 1) % 16, 0, 1] = 255
        vs[0, int(table[1, 0]), 3, 1, 0] = 255
        ks[0, int(table[2, 0]), 2, 1, 1] = 255
    out, lse = _check_attention(dtype, 64, 2, G, tree, [20, 100, 9, 70], N=N, change=change, seed=6)
    bad = torch.isnan(out)
    assert bad[0, -1, :G, 32:].all() and not bad[0, :, :, :32].any() and not bad[0, :, G:].any() and not bad[0, :-1].any()
    assert bad[1, :, G:, :32].all() and not bad[1, :, :G].any() and not bad[1, :, :, 32:].any() and not torch.isnan(lse[1]).any()
    assert bad[2, :, G:].all() and not bad[2, :, :G].any() and torch.isnan(lse[2, :, G:]).all() and not bad[3].any()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tree,N,G", [("binary", None, 2), ("binary5", None, 4), ("one", None, 3)])
def test_attention_without_pages(dtype, tree, N, G):
    flags = torch.zeros(4, dtype=torch.int32, device=DEV)

    def change(kc, vc, ks, vs, table, lengths, q):
        table[0, 1] = 9999
        table[1, 0] = -5
        lengths[2] = -1
    _check_attention(dtype, 64, 2, G, tree, [60, 3, 20, 50], N=N, change=change, seed=7, flags=flags)
    assert flags.tolist() == [32, 32, 32, 0]


@gpu
def test_attention_of_a_row_that_no_key_is_left_for():
    def change(kc, vc, ks, vs, table, lengths, q):
        table[0].fill_(-1)
    out, lse = _check_attention("bf16", 64, 2, 2, "binary", [20, 30], change=change, seed=8)
    assert (out[0] == 0).all() and (lse[0] == -math.inf).all()


@gpu
@pytest.mark.parametrize("dtype,dim,G,tree,N,lengths,shared", [
    ("bf16", 128, 4, "one", None, [5000, 3], 0), ("fp32", 80, 3, "binary", None, [70, 0, 9], 0), ("fp16", 64, 4, "binary5", None, [3000, 40], 0),
    ("bf16", 64, 2, "chain", 200, [33, 0], 0), ("bf16", 64, 4, "one", None, [1040, 1050, 1044, 1060, 1041, 1049], 1040),
    ("fp16", 256, 3, "binary5", None, [100, 600], 0)])
def test_sums_of_caches_of_other_types(dtype, dim, G, tree, N, lengths, shared):
    """The rows' sums over caches of 16 and 32 bits, by every kernel."""
    _check_attention(dtype, dim, 2, G, tree, lengths, N=N, shared=shared, four=False, seed=9)


@gpu
@pytest.mark.parametrize("dtype,dim,G,tree,N,lengths,shared", [
    ("bf16", 128, 4, "one", None, [5000, 3], 0), ("fp32", 80, 3, "binary", None, [70, 0, 9], 0), ("fp16", 64, 4, "binary5", None, [3000, 40], 0),
    ("bf16", 64, 4, "one", None, [1040, 1050, 1044, 1060, 1041, 1049], 1040), ("fp16", 256, 3, "binary5", None, [100, 600], 0)])
def test_results_are_the_same_with_and_without_sums(dtype, dim, G, tree, N, lengths, shared):
    t, N, _, _ = _trees(tree, N)
    kp, vp, table, _ = make_pages(lengths, N, 16, layers=1, heads=2, dim=dim, dtype=TYPES[dtype], order="slots", shared=shared, seed=24)
    cache = B.KVCache(kp, vp, table, torch.tensor(lengths, dtype=torch.int32, device=DEV))
    q = _queries(len(lengths), N, 2 * G, dim, TYPES[dtype], 24)
    lse = torch.zeros((len(lengths), N, 2 * G), device=DEV)
    assert torch.equal(B.tree_attention(cache, t, q, shared=shared), B.tree_attention(cache, t, q, shared=shared, lse=lse)) and lse.all()


@gpu
def test_attention_offsets_beyond_32_bits():
    """Codes and scales far into a pool of 5 GB."""
    page, heads, dim, pages = 64, 8, 128, 160000
    kc, vc, ks, vs = B.pages_in_4_bits(1, pages, page, heads, dim)
    assert kc.numel() > 2 ** 32
    gen = torch.Generator().manual_seed(3)
    chosen = [pages - 1, pages // 2, pages - 2, 1]
    x = [torch.randn((4, page, heads, dim), generator=gen) for _ in range(2)]
    got = []
    for values, codes, scales in ((x[0], kc, ks), (x[1], vc, vs)):
        c, s = _encode(values, torch.bfloat16)
        codes[0, chosen], scales[0, chosen] = c.to(DEV), s.to(DEV)
        got.append(values_of(c, s))
    table = torch.tensor([chosen], dtype=torch.int32, device=DEV)
    lengths = torch.tensor([4 * page - 15], dtype=torch.int32, device=DEV)
    for tree, N, G in (("one", 1, 4), ("binary", 15, 8)):
        t, N, parent, _ = _trees(tree, N)
        q = _queries(1, N, heads * G, dim, torch.bfloat16, 4)
        out = B.tree_attention(B.KVCache(kc, vc, table, lengths, ks, vs), t, q)
        want, off = attention(got[0], got[1], [[0, 1, 2, 3]], [4 * page - 15], [N], parent, q, dim ** -0.5)
        assert ((out.double().cpu() - want).abs() <= off).all()
        weights = torch.zeros((1, 4 * page), device=DEV)
        lse = torch.zeros((1, N, heads * G), device=DEV)
        B.tree_attention(B.KVCache(kc, vc, table, lengths, ks, vs), t, q, lse=lse)
        B.kv_weigh(B.KVCache(kc, vc, table, lengths, ks, vs), t, q, lse, weights)
        want, off = weigh(got[0], [[0, 1, 2, 3]], [4 * page - 15], [N], parent, q, lse, dim ** -0.5, 4 * page)
        assert ((weights.double().cpu() - want).abs() <= off + 2.0 ** -24 * want).all()


# ---------------------------------------------------------------- appending
def _check_append(dtype, dim, rot, neighbours, tree, lengths, *, N=None, page_size=16, order="slots", layers=1, counts=None, four=True,
                  axes=0, per_node=False, axis_of=None, far=0, heads=2, G=3, seed=0, held=True, change=None):
    dt = TYPES[dtype]
    t, N, parent, first = _trees(tree, N, counts)
    if four:
        kc, vc, ks, vs, table, rows = _pages(lengths, N, page_size, heads=heads, dim=dim, dtype=dt, order=order, layers=layers, seed=seed, used=False)
    else:
        kc, vc, table, rows = make_pages(lengths, N, page_size, layers=layers, heads=heads, dim=dim, dtype=dt, order=order, seed=seed, used=False)
        ks = vs = None
    Bn = len(lengths)
    new = _queries(Bn, N, heads * (G + 2), dim, dt, seed, fused=True)
    if change is not None:
        change(new)
    q, nk, nv = new[:, :, :heads * G], new[:, :, heads * G:heads * (G + 1)], new[:, :, heads * (G + 1):]
    inv = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float32) / max(1, rot // 2))
    level = levels(parent)
    gen = torch.Generator().manual_seed(seed + 5)
    positions = None
    if axes:
        positions = torch.randint(-far, far + 1, (axes, Bn, N) if per_node else (axes, Bn), generator=gen, dtype=torch.int32)
    out = torch.full(q.shape, 7.5, dtype=dt, device=DEV)
    k_out = torch.full(nk.shape, 7.5, dtype=dt, device=DEV) if four and held else None
    v_out = torch.full(nk.shape, 7.5, dtype=dt, device=DEV) if four and held else None
    before = [x.clone() for x in (kc, vc, ks, vs) if x is not None]
    flags = torch.zeros(Bn, dtype=torch.int32, device=DEV)
    cache = B.KVCache(kc, vc, table, torch.tensor(lengths, dtype=torch.int32, device=DEV), ks, vs)
    layer = layers - 1
    got = B.kv_append(cache, t, nk, nv, q, inv.to(DEV) if rot else None, layer=layer, neighbours=neighbours, out=out, flags=flags,
                      positions=None if positions is None else positions.to(DEV), axis_of=None if axis_of is None else axis_of.to(DEV),
                      k_out=k_out, v_out=v_out)
    assert got is out and not flags.any()
    c = counts or [N] * Bn
    wrote = torch.zeros(kc.shape[:3], dtype=torch.bool)
    for b in range(Bn):
        for n in range(N):
            if n >= c[b]:
                assert (out[b, n] == 7.5).all() and (k_out is None or (k_out[b, n] == 7.5).all() and (v_out[b, n] == 7.5).all())
                continue
            # every pair by its own axis
            at = []
            for i in range(rot // 2):
                a = 0 if axis_of is None else int(axis_of[i])
                if positions is None:
                    at.append(lengths[b] + level[n])
                elif a >= axes:
                    at.append(0)
                else:
                    at.append(int(positions[a, b, n]) if per_node else int(positions[a, b]) + level[n])

            def turned(x):
                y = x.clone()
                for i in range(rot // 2):
                    one = rotated(x, at[i], [0.0] * i + [float(inv[i])] + [0.0] * (rot // 2 - 1 - i), neighbours)
                    i0, i1 = (2 * i, 2 * i + 1) if neighbours else (i, i + rot // 2)
                    y[..., i0], y[..., i1] = one[..., i0], one[..., i1]
                return y
            x = q[b, n].double().cpu()
            w = turned(x)
            fine = torch.isfinite(w)
            # each product and its sum is rounded in fp32, cosine and sine by 2 ulp: 5 half steps of (|x| + |y|), then one to the type
            room = w.abs() * half_step(dt) + (5 * 2.0 ** -24 * 2 * x[torch.isfinite(x)].abs().max() if rot else 0.0)
            assert ((out[b, n].double().cpu() - w).abs() <= room)[fine].all(), (b, n)
            s = lengths[b] + n
            p = (layer, rows[b][s // page_size], s % page_size)
            wrote[p] = True
            key = turned(nk[b, n].double().cpu())
            if four:
                # turned in 64 bits: no border of the sixteen values is near enough to be missed
                for codes, scales, x, o in ((kc, ks, key.float(), k_out), (vc, vs, nv[b, n].float().cpu(), v_out)):
                    want = in_four(x, dt)
                    assert torch.equal(codes[p].cpu(), want[0]) and torch.equal(scales[p].cpu(), want[1]), (b, n)
                    if o is not None:
                        assert torch.equal(o[b, n].double().cpu().nan_to_num(99.0), values_of(*want).nan_to_num(99.0))
            else:
                room = key.abs() * half_step(dt) + (5 * 2.0 ** -24 * 2 * nk[b, n].abs().max().double().cpu() if rot else 0.0)
                assert ((kc[p].double().cpu() - key).abs() <= room).all() and torch.equal(vc[p], nv[b, n])
    for x, y in zip([x for x in (kc, vc, ks, vs) if x is not None], before):
        same = (x == y) | (x != x) & (y != y)
        assert same.flatten(3).all(-1).cpu()[~wrote].all()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim,rot,neighbours", [(64, 64, False), (64, 64, True), (128, 32, False), (96, 96, False), (96, 40, True), (32, 20, False),
                                                (64, 22, False), (64, 2, True), (160, 0, False), (256, 256, False)])
def test_append_in_four_bits(dtype, dim, rot, neighbours):
    _check_append(dtype, dim, rot, neighbours, "binary", [3, 40, 0], seed=dim + rot)


@gpu
@pytest.mark.parametrize("tree,N", [("spine", None), ("roots", None), ("eight", None), ("chain", 40), ("chain_table", 40), ("one", None)])
def test_append_in_four_bits_trees(tree, N):
    _check_append("bf16", 64, 64, False, tree, [5, 18, 0], N=N, page_size=3, order="heads", layers=3)
    _check_append("fp32", 64, 64, True, tree, [5, 18, 0], N=N, counts=[1, 0, 77], held=False)


@gpu
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("axes,per_node,far", [(1, False, 1000000), (1, True, 100), (3, True, 5000), (8, False, 30), (2, True, 2 ** 31 - 1)])
def test_append_at_given_positions(four, axes, per_node, far):
    far = far if per_node or far < 2 ** 31 - 100 else far - 100
    gen = torch.Generator().manual_seed(axes)
    some = torch.randint(0, axes + 1, (16,), generator=gen, dtype=torch.uint8)   # an axis that is none among them
    for dtype, neighbours, tree, axis_of in (("bf16", False, "binary", some), ("fp32", True, "chain", None), ("fp16", False, "spine", some)):
        _check_append(dtype, 64, 32, neighbours, tree, [5, 18], N=20, four=four, axes=axes, per_node=per_node, axis_of=axis_of, far=far)


@gpu
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("neighbours", [True, False])
def test_append_of_pairs_that_turn_by_no_axis(four, dtype, neighbours):
    """They stay as they are, whatever stands in the place of their frequencies."""
    axis_of = torch.tensor([0, 1, 7, 255] * 8, dtype=torch.uint8, device=DEV)
    none = (axis_of > 1).nonzero()[:, 0]
    positions = torch.tensor([[3, 70], [-20, 1000000]], dtype=torch.int32, device=DEV)
    results = []
    for number in (1.0, 0.0, math.nan, math.inf, 3e38):
        if four:
            kc, vc, ks, vs, table, _ = _pages([5, 18], 7, 16, dim=64, dtype=TYPES[dtype], seed=20, used=False)
        else:
            kc, vc, table, _ = make_pages([5, 18], 7, 16, layers=1, heads=2, dim=64, dtype=TYPES[dtype], order="slots", seed=20, used=False)
            ks = vs = None
        x = _queries(2, 7, 2, 64, TYPES[dtype], 20)
        inv = torch.linspace(1.0, 0.01, 32, device=DEV)
        inv[none] = number
        cache = B.KVCache(kc, vc, table, torch.tensor([5, 18], dtype=torch.int32, device=DEV), ks, vs)
        out = B.kv_append(cache, B.TokenTree(2, 3), x, x, x, inv, neighbours=neighbours, positions=positions, axis_of=axis_of)
        one, two = (2 * none, 2 * none + 1) if neighbours else (none, none + 32)
        assert torch.equal(out[..., one], x[..., one]) and torch.equal(out[..., two], x[..., two])
        results.append([y.nan_to_num(9.0) if y.is_floating_point() else y for y in (out, kc, vc, ks, vs) if y is not None])
    for got in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got, results[0]))


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_append_of_borders_zeros_and_what_is_no_number(dtype):
    """Ties, zeros of both signs, the smallest and largest numbers of the type, infinities and NaN."""
    info = torch.finfo(TYPES[dtype])

    def change(new):
        x = new[:, :, 6:]    # keys and values
        gen = torch.Generator().manual_seed(2)
        grid = torch.tensor([0.0, -0.0, 0.25, -0.75, 1.25, 1.75, -2.5, 3.5, 5.0, -5.0, 6.0, 6.5, 7.0, -7.0, 0.5, -3.0])
        pick = grid[torch.randint(0, 16, x.shape, generator=gen)] * 2.0 ** torch.randint(-4, 4, (*x.shape[:-1], 1), generator=gen)
        x.copy_(pick.to(TYPES[dtype]))
        x[0, 0].zero_()
        x[0, 1, :, 0:32] = info.max
        x[0, 1, :, 32:64] = info.tiny
        x[0, 2, :, 0] = info.smallest_normal * info.eps   # the smallest there is
        x[0, 3, 0, 5] = math.inf
        x[0, 3, 1, 40] = math.nan
        x[0, 4, 2, 63] = -math.inf
        x[0, 5, :, 0] = -info.max
        x[0, 5, :, 1:].zero_()
        x[0, 6] = -0.0
    _check_append(dtype, 64, 0, False, "binary", [5, 18], change=change)
    _check_append(dtype, 64, 0, True, "chain", [5], N=9, order="heads", change=change)


@gpu
def test_append_without_pages():
    kc, vc, ks, vs, table, rows = _pages([10, 20, 30, 40], 7, 16, used=False)
    table[1, 1] = 99
    lengths = torch.tensor([10, 20, -1, table.shape[1] * 16 - 3], dtype=torch.int32, device=DEV)
    x = _queries(4, 7, 2, 64, torch.bfloat16, 4)
    flags = torch.zeros(4, dtype=torch.int32, device=DEV)
    before = ks.clone()
    held = torch.full_like(x, 7.5)
    assert B.kv_append(B.KVCache(kc, vc, table, lengths, ks, vs), B.TokenTree(2, 3), x, x, flags=flags, k_out=held) is None
    assert flags.tolist() == [0, 32, 32, 32]
    changed = (before != ks).flatten(3).any(-1)
    slots = {(0, rows[0][(10 + n) // 16], (10 + n) % 16) for n in range(7)}
    slots |= {(0, rows[1][(20 + n) // 16], (20 + n) % 16) for n in range(7) if (20 + n) // 16 != 1}
    assert {tuple(i) for i in changed.nonzero().tolist()} == slots
    want = values_of(*in_four(x, torch.bfloat16))   # a key without a page has them too, a sequence without nodes has none
    assert torch.equal(held[[0, 1, 3]].double().cpu(), want[[0, 1, 3]]) and (held[2] == 7.5).all()


@gpu
def test_append_values_in_place():
    """v_out may be v itself."""
    kc, vc, ks, vs, table, _ = _pages([10, 20], 7, 16, used=False)
    lengths = torch.tensor([10, 20], dtype=torch.int32, device=DEV)
    x, y = _queries(2, 7, 2, 64, torch.bfloat16, 4), _queries(2, 7, 2, 64, torch.bfloat16, 5)
    want = values_of(*in_four(y, torch.bfloat16))
    B.kv_append(B.KVCache(kc, vc, table, lengths, ks, vs), B.TokenTree(2, 3), x, y, v_out=y)
    assert torch.equal(y.double().cpu(), want)


# ---------------------------------------------------------------- committing
@gpu
@pytest.mark.parametrize("tree,N", [("binary5", None), ("spine", None), ("one", None), ("chain", 100), ("chain_table", 100)])
@pytest.mark.parametrize("dim,order,page_size", [(128, "slots", 5), (32, "heads", 16), (96, "heads", 5)])
@pytest.mark.parametrize("in_place", [False, True])
def test_commit(tree, N, dim, order, page_size, in_place):
    t, N, parent, first = _trees(tree, N, None)
    k, depth = t.k, t.depth
    lengths, counts = [0, 5, 16, 31, 7], [N, N, N, 0, max(1, N // 2)]
    t.counts = torch.tensor(counts, dtype=torch.int32, device=DEV)
    kc, vc, ks, vs, table, rows = _pages(lengths, N, page_size, heads=3, dim=dim, order=order, layers=3, seed=1)
    outcome = _outcomes(5, N, k, N)
    outcome[0].fill_(k - 1)
    outcome[1].clamp_(min=0)
    accept = torch.tensor([depth - 1, 10 ** 6, 1, 2, depth - 1], dtype=torch.int32)
    len_t = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    want, new = [x.clone() for x in (kc, vc, ks, vs)], []
    for b in range(5):
        path = path_of(outcome[b].tolist(), int(accept[b]), depth, k, N, counts[b], first)
        new.append(lengths[b] + len(path))
        for i, n in enumerate(path):
            (p0, s0), (p1, s1) = ((rows[b][s // page_size], s % page_size) for s in (lengths[b] + n, lengths[b] + i))
            for x in want:
                x[:, p1, s1] = x[:, p0, s0]
    flags = torch.zeros(5, dtype=torch.int32, device=DEV)
    got = B.kv_commit(B.KVCache(kc, vc, table, len_t, ks, vs), t, outcome.to(DEV), accept.to(DEV), out=len_t if in_place else None, flags=flags)
    assert got.tolist() == new and not flags.any()
    for x, y in zip((kc, vc, ks, vs), want):
        assert torch.equal(x, y)


# ---------------------------------------------------------------- weights
def _check_weigh(dtype, dim, heads, G, tree, lengths, *, N=None, page_size=16, order="slots", counts=None, four=True, path=False, seed=0,
                 weights="given", width=None, layers=2, change=None, flags=None, off_lse=None):
    dt = TYPES[dtype]
    t, N, parent, first = _trees(tree, N, counts)
    if four:
        kc, vc, ks, vs, table, _ = _pages(lengths, N, page_size, heads=heads, dim=dim, dtype=dt, order=order, layers=layers, seed=seed)
    else:
        kc, vc, table, _ = make_pages(lengths, N, page_size, layers=layers, heads=heads, dim=dim, dtype=dt, order=order, seed=seed)
        ks = vs = None
    Bn, layer = len(lengths), layers - 1
    len_t = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    q = _queries(Bn, N, heads * G, dim, dt, seed, fused=True)
    if change is not None:
        change(kc, ks, table, len_t, q)
    lengths = len_t.tolist()
    kv = values_of(kc[layer], ks[layer]) if four else kc[layer].double()
    c = counts or [N] * Bn
    rows = table.cpu().tolist()
    lse = lse_of(kv, rows, lengths, c, parent, q, dim ** -0.5)[0].float()
    lse = torch.where(torch.isnan(lse), 7.5, lse) if off_lse is None else off_lse(lse)
    width = width or max(max(lengths), 0) + N + 3
    outcome = accept = paths = None
    if path:
        outcome = _outcomes(Bn, N, t.k, seed + 3)
        outcome[0].clamp_(min=0)
        accept = torch.tensor([t.depth - 1 if b % 2 == 0 else b for b in range(Bn)], dtype=torch.int32)
        paths = [path_of(outcome[b].tolist(), int(accept[b]), t.depth, t.k, N, max(0, min(N, c[b])), first) for b in range(Bn)]
    want, off = weigh(kv, rows, lengths, c, parent, q, lse, dim ** -0.5, width, paths)
    before = torch.rand((Bn, width + 5), generator=torch.Generator().manual_seed(seed)).to(DEV)
    base = before[:, 2:2 + width].double().cpu()
    kw = dict(layer=layer, flags=flags)
    if path:
        kw.update(outcome=outcome.to(DEV), accept_depth=accept.to(DEV))
    cache = B.KVCache(kc, vc, table, len_t, ks, vs)
    given = before.clone()
    into = torch.full((Bn, width + 9), 7.5, device=DEV)
    lse = lse.to(DEV)
    if weights == "given":
        got = B.kv_weigh(cache, t, q, lse, given[:, 2:2 + width], out=into[:, 1:1 + width], **kw)
        assert torch.equal(given, before) and (into[:, :1] == 7.5).all() and (into[:, 1 + width:] == 7.5).all()
        want = want + base
    elif weights == "in place":
        got = B.kv_weigh(cache, t, q, lse, given[:, 2:2 + width], **kw)
        assert torch.equal(given[:, :2], before[:, :2]) and torch.equal(given[:, 2 + width:], before[:, 2 + width:])
        want = want + base
    else:
        got = B.kv_weigh(cache, t, q, lse, None, out=into[:, 1:1 + width], **kw)
    got = got.double().cpu()
    fine = torch.isfinite(want)
    assert bool((torch.isfinite(got) == fine).all())
    wrong = ((got - want).abs() > off + 2.0 ** -23 * want.abs()) & fine
    assert not wrong.any(), (wrong.nonzero()[:4].tolist(), got[wrong][:4], want[wrong][:4])
    return got


@gpu
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 192, 256])
def test_weights_types_and_dims(four, dtype, dim):
    _check_weigh(dtype, dim, 2, 4, "binary", [0, 1, 63, 64, 65, 300], four=four, seed=dim)


@gpu
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("path", [False, True])
@pytest.mark.parametrize("tree,N,G", [("one", None, 1), ("one", None, 20), ("spine", None, 3), ("roots", None, 4), ("binary5", None, 4), ("ternary", None, 5),
                                      ("chain", 150, 2), ("chain_table", 70, 1)])
def test_weights_trees(four, path, tree, N, G):
    _check_weigh("bf16", 64, 3, G, tree, [0, 7, 270], N=N, page_size=24, order="heads", four=four, path=path, seed=1)
    _check_weigh("fp32", 64, 1, G, tree, [30, 0, 4], N=N, counts=[1, 0, 5], four=four, path=path, weights="in place", seed=2)


@gpu
@pytest.mark.parametrize("weights", ["given", "in place", "none"])
@pytest.mark.parametrize("width", [1, 65, 511, 2000])
def test_weights_rows(weights, width):
    """Rows shorter than the sequences, and longer."""
    _check_weigh("bf16", 128, 2, 4, "binary", [600, 3, 200, -1], weights=weights, width=width, seed=3)


@gpu
@pytest.mark.parametrize("four,dtype,dim,heads,G,path", [(True, "bf16", 128, 8, 1, True), (False, "bf16", 64, 8, 2, False), (True, "fp32", 96, 2, 1, False),
                                                         (False, "fp16", 128, 3, 4, True)])
@pytest.mark.parametrize("width", [17000, 40000])
def test_weights_of_few_rows_over_many_slots(four, dtype, dim, heads, G, path, width):
    """Rows of slots that are long enough for all queries to stand in LDS."""
    _check_weigh(dtype, dim, heads, G, "spine", [0, 500, 255, 257, 90, -1], four=four, path=path, width=width, seed=13, page_size=24, order="heads")


@gpu
@pytest.mark.parametrize("four,dtype,dim,heads,G,tree,N", [(False, "bf16", 128, 12, 1, "binary", None), (True, "fp32", 128, 4, 1, "chain_table", 16),
                                                           (False, "fp16", 32, 1, 1, "chain_table", 384)])
def test_weights_of_as_many_rows_as_lds_has_room_for(four, dtype, dim, heads, G, tree, N):
    _check_weigh(dtype, dim, heads, G, tree, [0, 500, 255, 257, 90, -1], N=N, four=four, width=17000, seed=25)


@gpu
@pytest.mark.parametrize("four,dtype,dim,heads,G,tree,N", [(True, "bf16", 64, 8, 3, "chain", 40), (False, "fp16", 128, 9, 5, "binary", None),
                                                           (True, "bf16", 160, 11, 5, "binary5", None), (True, "fp32", 64, 8, 5, "binary", None)])
def test_weights_of_many_rows_of_many_heads(four, dtype, dim, heads, G, tree, N):
    """A workgroup of eight waves, with as many heads and more."""
    _check_weigh(dtype, dim, heads, G, tree, [0, 64, 200], N=N, counts=None, four=four, seed=14)


@gpu
@pytest.mark.parametrize("four", [True, False])
def test_weights_without_pages_and_without_rows(four):
    flags = torch.zeros(4, dtype=torch.int32, device=DEV)

    def change(kc, ks, table, lengths, q):
        table[0, 1] = 9999
        table[1].fill_(-1)      # no key is left: its rows' sums are minus infinity
        lengths[2] = -1
    got = _check_weigh("bf16", 64, 2, 2, "binary", [60, 3, 20, 50], four=four, change=change, flags=flags, weights="none", seed=7)
    assert flags.tolist() == [32, 32, 32, 0] and (got[1] == 0).all() and (got[0, 16:32] == 0).all()


@gpu
def test_weights_of_keys_that_are_no_numbers():
    """What no row sees is left out, whatever it holds; what a row sees shows."""
    def change(kc, ks, table, lengths, q):
        ks[1, int(table[0, 0]), 3, 1, 1] = 255
    got = _check_weigh("bf16", 64, 2, 2, "binary", [20, 30], change=change, weights="none", seed=8,
                       off_lse=lambda x: x.nan_to_num(3.0))
    assert torch.isnan(got[0, 3]) and not torch.isnan(got[0, 4:]).any() and not torch.isnan(got[1]).any()


def _check_weigh_no_numbers(four, dtype, dim, heads, G, tree, N, path, width, muted):
    """Keys that are no numbers beside slots that their rows do not see: of other branches, without a page, behind the last."""
    dt = TYPES[dtype]
    t, N, parent, first = _trees(tree, N)
    lengths = [20, 100, 45, 30]
    Bn = len(lengths)
    if four:
        kc, vc, ks, vs, table, _ = _pages(lengths, N, 16, heads=heads, dim=dim, dtype=dt, order="heads", seed=17)
    else:
        kc, vc, table, _ = make_pages(lengths, N, 16, layers=1, heads=heads, dim=dim, dtype=dt, order="heads", seed=17)
        ks = vs = None
    outcome = _outcomes(Bn, N, t.k, 18).clamp_(min=0)
    accept = torch.tensor([t.depth - 1, t.depth, 0, 1], dtype=torch.int32)
    paths = [path_of(outcome[b].tolist(), int(accept[b]), t.depth, t.k, N, N, first) for b in range(Bn)]
    nodes = paths if path else [list(range(N))] * Bn
    # the last of the first sequence's nodes, seen by itself alone; a slot that all see, beside some without a page; a node in the middle
    table[1, 1] = -1
    for b, s, h in ((0, lengths[0] + nodes[0][-1], 0), (1, 3, heads - 1), (3, lengths[3] + nodes[3][len(nodes[3]) // 2], 0)):
        at = (0, int(table[b, s // 16]), s % 16, h, 0)
        if four:
            ks[at] = 255
        else:
            kc[at] = math.nan
    len_t = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    q = _queries(Bn, N, heads * G, dim, dt, 17, fused=True)
    cache = B.KVCache(kc, vc, table, len_t, ks, vs)
    lse = torch.zeros((Bn, N, heads * G), device=DEV)
    B.tree_attention(cache, t, q, lse=lse)
    bad = torch.isnan(lse)
    assert bad[0].any() and bad[1, :, -G:].all() and not bad[1, :, :-G].any() and not bad[2].any() and bad[3].any()
    if muted:
        lse[bad] = -math.inf
    kv = values_of(kc[0], ks[0]) if four else kc[0].double()
    width = width or max(lengths) + N + 70
    want, off = weigh(kv, table.cpu().tolist(), lengths, [N] * Bn, parent, q, lse, dim ** -0.5, width, paths if path else None)
    before = torch.rand((Bn, width), generator=torch.Generator().manual_seed(19))
    want += before
    kw = dict(outcome=outcome.to(DEV), accept_depth=accept.to(DEV)) if path else {}
    got = B.kv_weigh(cache, t, q, lse, before.to(DEV), **kw).cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.isnan(want).any() != muted
    for b in range(Bn):
        end = lengths[b] + len(nodes[b])
        assert torch.equal(got[b, end:], before[b, end:]), ("behind the last slot", b)
    assert torch.equal(got[1, 16:32], before[1, 16:32])
    fine = ~torch.isnan(want)
    wrong = ((got.double() - want).abs() > off + 2.0 ** -23 * want.abs()) & fine
    assert not wrong.any(), wrong.nonzero()[:4].tolist()


# (four, dtype, dim, heads, G, tree, N): few rows, more than 64, of eight heads and more; with a width of 40000 in LDS where they fit
ROWS_OF_NO_NUMBER = [(True, "bf16", 128, 2, 2, "binary", None), (False, "fp16", 64, 3, 4, "spine", None), (True, "fp32", 96, 2, 1, "binary", None),
                     (True, "bf16", 64, 8, 4, "binary5", None), (False, "fp32", 64, 2, 3, "chain", 40), (False, "bf16", 128, 2, 5, "chain", 9)]


@gpu
@pytest.mark.parametrize("width", [None, 40000])
@pytest.mark.parametrize("path", [False, True])
@pytest.mark.parametrize("four,dtype,dim,heads,G,tree,N", ROWS_OF_NO_NUMBER)
def test_weights_of_rows_whose_sum_is_no_number(four, dtype, dim, heads, G, tree, N, path, width):
    """The attention's own sums: what such a row sees is no number either, and what it does not see is as if it were not there."""
    _check_weigh_no_numbers(four, dtype, dim, heads, G, tree, N, path, width, False)


@gpu
@pytest.mark.parametrize("width", [None, 40000])
@pytest.mark.parametrize("path", [False, True])
@pytest.mark.parametrize("four,dtype,dim,heads,G,tree,N", ROWS_OF_NO_NUMBER)
def test_weights_of_rows_that_are_left_out(four, dtype, dim, heads, G, tree, N, path, width):
    """A row of minus infinity adds nothing, also where a key that it sees is no number."""
    _check_weigh_no_numbers(four, dtype, dim, heads, G, tree, N, path, width, True)


@gpu
def test_weights_are_the_same_from_call_to_call():
    t, N, _, _ = _trees("binary5", None)
    kc, vc, ks, vs, table, _ = _pages([3000, 70, 900], N, 16, heads=4, dim=128, order="heads", seed=9)
    cache = B.KVCache(kc, vc, table, torch.tensor([3000, 70, 900], dtype=torch.int32, device=DEV), ks, vs)
    q = _queries(3, N, 16, 128, torch.bfloat16, 9)
    lse = torch.zeros((3, N, 16), device=DEV)
    B.tree_attention(cache, t, q, lse=lse)
    first = B.kv_weigh(cache, t, q, lse)
    assert first.shape == (3, table.shape[1] * 16)
    for _ in range(5):
        assert torch.equal(B.kv_weigh(cache, t, q, lse), first)
    # every row's weights add up to one
    assert torch.allclose(first.sum(1), torch.full((3,), float(N * 16), device=DEV), rtol=1e-4)


# ---------------------------------------------------------------- eviction
def _check_evict(lengths, budget, first, recent, *, four=True, dim=64, dtype="bf16", heads=2, order="slots", page_size=16, layers=2, weights=None,
                 width=None, out="own", into="own", seed=0, change=None):
    Bn = len(lengths)
    if four:
        kc, vc, ks, vs, table, _ = _pages([max(n, 0) for n in lengths], 1, page_size, heads=heads, dim=dim, order=order, layers=layers, seed=seed)
    else:
        kc, vc, table, _ = make_pages([max(n, 0) for n in lengths], 1, page_size, layers=layers, heads=heads, dim=dim, dtype=TYPES[dtype], order=order, seed=seed)
        ks = vs = None
    len_t = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    if change is not None:
        change(table, len_t)
    width = width or max(max(lengths), 1) + 3
    if weights is None:
        weights = torch.randn((Bn, width), generator=torch.Generator().manual_seed(seed + 1)).exp()
        weights[:, ::5] = 0.25      # many that are equal
        weights[:, 3::11] = 0.0
        weights[:, 14::11] = -0.0
    w = weights.to(DEV)
    pools = [x for x in (kc, vc, ks, vs) if x is not None]
    want = [x.clone() for x in pools]
    rows, capacity = table.cpu().tolist(), table.shape[1] * page_size
    flags = torch.zeros(Bn, dtype=torch.int32, device=DEV)
    want_flags, want_kept, want_w, want_len = [], [], torch.zeros((Bn, width)), []
    for b in range(Bn):
        n = min(lengths[b], capacity)
        stay = kept_of(weights[b].tolist(), n, budget, first, recent)
        want_len.append(min(n, budget))
        want_kept.append(stay + [-1] * (budget - len(stay)))
        for i, s in enumerate(stay):
            if i < width:
                want_w[b, i] = weights[b, s] if s < width else 0.0
        flag = 32 if lengths[b] < 0 or lengths[b] > capacity else 0
        for i, s in enumerate(stay):
            if i == s:
                continue
            src, dst = (rows[b][x // page_size] for x in (s, i))
            if not 0 <= src < kc.shape[1] or not 0 <= dst < kc.shape[1]:
                flag = 32
                continue
            for x, y in zip(want, pools):
                x[:, dst, i % page_size] = y[:, src, s % page_size]
        want_flags.append(flag)
    cache = B.KVCache(kc, vc, table, len_t, ks, vs)
    new = len_t if out == "lengths" else None
    w_out = {"own": torch.full((Bn, width), 7.5, device=DEV), "in place": w, "none": None}[into]
    got, kept = B.kv_evict(cache, w, budget, first=first, recent=recent, out=new, weights_out=w_out, flags=flags)
    assert got.tolist() == want_len and kept.tolist() == want_kept
    assert new is None or got is new
    if w_out is not None:
        assert torch.equal(w_out.cpu().nan_to_num(9.0), want_w.nan_to_num(9.0))
    assert flags.tolist() == want_flags
    for x, y in zip(pools, want):
        assert torch.equal(x.nan_to_num(9.0) if x.is_floating_point() else x, y.nan_to_num(9.0) if y.is_floating_point() else y)


@gpu
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("budget,first,recent", [(100, 4, 20), (1, 0, 0), (64, 0, 64), (64, 64, 0), (50, 20, 30), (99, 0, 0), (150, 3, 0), (500, 4, 4)])
def test_evict(four, budget, first, recent):
    _check_evict([300, 0, 99, 100, 101, 150, 40, -1], budget, first, recent, four=four, seed=budget)


@gpu
@pytest.mark.parametrize("four,dim,dtype,heads,order,page_size", [
    (True, 32, "bf16", 3, "heads", 16), (True, 96, "bf16", 5, "slots", 1), (True, 128, "bf16", 8, "heads", 64), (True, 256, "bf16", 1, "slots", 24),
    (True, 160, "bf16", 16, "slots", 48), (False, 8, "bf16", 1, "slots", 16), (False, 72, "fp16", 3, "heads", 5), (False, 256, "fp32", 2, "heads", 16),
    (False, 128, "bf16", 8, "slots", 16)])
@pytest.mark.parametrize("into,out", [("own", "own"), ("in place", "lengths"), ("none", "own")])
def test_evict_layouts(four, dim, dtype, heads, order, page_size, into, out):
    _check_evict([700, 130, 20], 120, 5, 16, four=four, dim=dim, dtype=dtype, heads=heads, order=order, page_size=page_size, into=into, out=out, layers=3, seed=1)


@gpu
@pytest.mark.parametrize("n,budget", [(9000, 5000), (40000, 300), (5000, 4999), (4097, 4096), (20000, 17000)])
def test_evict_long_sequences(n, budget):
    _check_evict([n, n // 2], budget, min(4, budget), min(64, budget - 4), dim=32, heads=1, layers=1, seed=2, into="in place", out="lengths")


@gpu
@pytest.mark.parametrize("four", [True, False])
@pytest.mark.parametrize("n,budget,first,recent", [(60, 18, 3, 4), (50, 7, 0, 1), (90, 40, 0, 0)])
def test_evict_little_of_many_rows(four, n, budget, first, recent):
    """Many layers and heads of which little moves: several heads are a workgroup's."""
    _check_evict([n - b % 23 for b in range(40)], budget, first, recent, four=four, dim=128, heads=8, layers=9, seed=15)


@gpu
@pytest.mark.parametrize("numbers", [0, 1, 3, 40])
def test_evict_where_all_of_a_digit_are_kept(numbers):
    """As many numbers as places beside slots that are no number, zero, or the lowest; one more, and one fewer."""
    n, budget, first, recent = 300, 50, 5, 5
    for rest in (math.nan, 0.0, -math.inf):
        for more in (-1, 0, 1):
            w = torch.full((2, n + 3), rest)
            at = torch.randperm(n - first - recent, generator=torch.Generator().manual_seed(numbers)) + first
            w[0, at[:max(0, numbers + more)]] = 2.0
            w[1, at[:40 + more]] = torch.randn(40 + more, generator=torch.Generator().manual_seed(16)).abs() + 1
            _check_evict([n, n], budget, first, recent, weights=w, width=n + 3, seed=16)


@gpu
@pytest.mark.parametrize("kind", ["equal", "nan", "infinite", "negative", "falling", "rising", "tiny"])
@pytest.mark.parametrize("into", ["own", "in place"])
def test_evict_weights_of_every_kind(kind, into):
    n, width = 3000, 3010
    gen = torch.Generator().manual_seed(4)
    w = torch.randn((2, width), generator=gen)
    w = {"equal": torch.ones((2, width)), "nan": torch.where(w > 0.5, math.nan, w), "negative": -w.abs() - 1,
         "infinite": torch.where(w > 1, math.inf, torch.where(w < -1, -math.inf, w)), "falling": -torch.arange(width).float().expand(2, -1).clone(),
         "rising": torch.arange(width).float().expand(2, -1).clone(), "tiny": w * 1e-42}[kind]
    _check_evict([n, 1500], 1000, 10, 100, weights=w, width=width, into=into, seed=5)


@gpu
def test_evict_rows_of_weights_shorter_than_sequences():
    """Slots that have no weight count as zero."""
    w = torch.full((3, 50), 0.5)
    w[:, 7:9] = -1.0
    for into in ("own", "in place"):
        _check_evict([200, 60, 30], 40, 2, 10, weights=w.clone(), width=50, into=into, seed=6)
        _check_evict([200, 60, 30], 70, 2, 10, weights=w.clone(), width=50, into=into, seed=6)


@gpu
def test_evict_without_pages():
    def change(table, lengths):
        table[0, 3] = -1
        table[1, 0] = 12345
        lengths[2] = table.shape[1] * 16 + 40
    lengths = [200, 180, 0, 20]

    def both(table, len_t):
        change(table, len_t)
        lengths[2] = int(len_t[2])
    _check_evict(lengths, 60, 2, 10, change=both, seed=7)


# ---------------------------------------------------------------- together
def _world(four, seed, lengths=(700, 90, 333), heads=2, G=4, dim=128, dtype=torch.bfloat16):
    t, N, parent, _ = _trees("binary", None)
    room = [n + 200 for n in lengths]
    if four:
        kc, vc, ks, vs, table, _ = _pages(room, N, 16, heads=heads, dim=dim, dtype=dtype, order="heads", layers=2, seed=seed)
    else:
        kc, vc, table, _ = make_pages(room, N, 16, layers=2, heads=heads, dim=dim, dtype=dtype, order="heads", seed=seed)
        ks = vs = None
    Bn = len(lengths)
    len_t = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    new = _queries(Bn, N, heads * (G + 2), dim, dtype, seed)
    return dict(cache=B.KVCache(kc, vc, table, len_t, ks, vs), tree=t, q=new[:, :, :heads * G], k=new[:, :, heads * G:heads * (G + 1)],
                v=new[:, :, heads * (G + 1):], turned=torch.zeros((Bn, N, heads * G, dim), dtype=dtype, device=DEV),
                out=torch.zeros((2, Bn, N, heads * G, dim), dtype=dtype, device=DEV), lse=torch.zeros((Bn, N, heads * G), device=DEV),
                weights=torch.zeros((Bn, max(room) + N), device=DEV), positions=len_t.clone()[None], before=len_t.clone(),
                outcome=_outcomes(Bn, N, 2, seed).clamp_(min=0).to(DEV), accept=torch.tensor([2, 3, 0], dtype=torch.int32, device=DEV)[:Bn].contiguous(),
                kept=torch.zeros((Bn, 300), dtype=torch.int32, device=DEV))


def _step(w, evict):
    inv = 10000.0 ** (-torch.arange(64, dtype=torch.float32, device=DEV) / 64)
    cache, tree = w["cache"], w["tree"]
    w["before"].copy_(cache.lengths)
    for layer in (0, 1):
        B.kv_append(cache, tree, w["k"], w["v"], w["q"], inv, layer=layer, positions=w["positions"], out=w["turned"])
        B.tree_attention(cache, tree, w["turned"], layer=layer, out=w["out"][layer], lse=w["lse"])
        B.kv_weigh(cache, tree, w["turned"], w["lse"], w["weights"], layer=layer, outcome=w["outcome"], accept_depth=w["accept"])
    B.kv_commit(cache, tree, w["outcome"], w["accept"], out=cache.lengths)
    w["positions"].add_(cache.lengths - w["before"])
    if evict:
        B.kv_evict(cache, w["weights"], 300, first=4, recent=32, out=cache.lengths, kept=w["kept"], weights_out=w["weights"])


def _state(w):
    c = w["cache"]
    pools = [x for x in (c.k, c.v, c.k_scales, c.v_scales) if x is not None]
    return [x.nan_to_num(9.0) if x.is_floating_point() else x for x in pools + [w["out"], w["lse"], w["weights"], c.lengths, w["positions"]]]


@gpu
@pytest.mark.parametrize("four", [True, False])
def test_steps_of_a_decoder_that_evicts(four):
    """Weights of a step add up to one a row and layer; an eviction leaves the attention to what it kept."""
    w = _world(four, 1)
    rows = w["accept"].cpu() + 1
    for i in range(3):
        _step(w, False)
        # (a path's row also sees its ancestors only: all of them are on the path)
        total = w["weights"].double().sum(1).cpu()
        want = (i + 1) * 2 * 8 * rows.double()
        assert torch.allclose(total, want, rtol=1e-4), (total, want)
        assert (w["weights"][torch.arange(w["weights"].shape[1], device=DEV)[None] >= w["cache"].lengths[:, None]] == 0).all()
    lengths = w["cache"].lengths.tolist()
    assert w["positions"][0].tolist() == lengths
    kept = [kept_of(w["weights"][b].tolist(), n, 300, 4, 32) for b, n in enumerate(lengths)]
    before = [x.clone() for x in (w["cache"].k, w["cache"].v)]
    _step(w, True)
    assert w["cache"].lengths.tolist() == [min(300, n + int(a)) for n, a in zip(lengths, rows)]
    assert w["positions"][0].tolist() == [n + int(a) for n, a in zip(lengths, rows)]
    for x, y in zip(before, (w["cache"].k, w["cache"].v)):
        table = w["cache"].table.long()
        assert torch.equal(x[:, table[1, 0], :4].nan_to_num(9.0), y[:, table[1, 0], :4].nan_to_num(9.0))
    got = [[s for s in w["kept"][b].tolist() if s >= 0] for b in range(3)]
    assert [len(g) for g in got] == [min(300, n + int(a)) for n, a in zip(lengths, rows)]
    assert got[1] == list(range(lengths[1] + int(rows[1]))) and got[0][:4] == [0, 1, 2, 3] and len(set(got[0]) & set(kept[0])) > 200


@gpu
@pytest.mark.parametrize("four", [True, False])
def test_captured_and_replayed_on_another_stream(four):
    """A step's calls in a graph whose lengths, positions and weights go on from replay to replay, against the same made eagerly."""
    a, b = _world(four, 2), _world(four, 2)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            _step(b, True)
    for replay in range(4):
        _step(a, True)
        with torch.cuda.stream(stream):
            graph.replay()
        stream.synchronize()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(_state(a), _state(b))), replay
        for w in (a, b):
            w["q"].mul_(1.0009765625 if replay % 2 else 0.5)


@gpu
def test_two_streams_at_once():
    def steps(w, stream):
        with torch.cuda.stream(stream):
            for i in range(4):
                _step(w, i % 2 == 1)
            return _state(w)
    alone = []
    for seed in (3, 4):
        w = _world(True, seed)
        torch.cuda.synchronize()
        alone.append(steps(w, torch.cuda.current_stream()))
        torch.cuda.synchronize()
    worlds, streams = [_world(True, 3), _world(True, 4)], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    together = [steps(w, s) for w, s in zip(worlds, streams)]
    torch.cuda.synchronize()
    for x, y in zip(alone, together):
        assert all(torch.equal(p, q) for p, q in zip(x, y))


@gpu
@pytest.mark.parametrize("four", [True, False])
def test_marshalling_in_python_gives_the_same(four, monkeypatch):
    results = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(B, "_native", lambda: None)
        w = _world(four, 5)
        _step(w, False)
        cache, tree = w["cache"], w["tree"]
        axis_of = torch.tensor([0, 1, 1, 2] * 8, dtype=torch.uint8, device=DEV)
        positions = torch.arange(3 * 3 * 15, dtype=torch.int32, device=DEV).view(3, 3, 15)
        more = dict(k_out=torch.zeros_like(w["k"]).contiguous(), v_out=torch.zeros_like(w["v"]).contiguous()) if four else {}
        got = [B.kv_append(cache, tree, w["k"], w["v"], w["q"], torch.ones(32, device=DEV), positions=positions, axis_of=axis_of, neighbours=True, **more)]
        got += [B.tree_attention(cache, tree, w["q"], lse=w["lse"], scale=0.1), *more.values()]
        got += [B.kv_weigh(cache, tree, w["q"], w["lse"], scale=0.1)]
        got += list(B.kv_evict(cache, w["weights"], 200, flags=torch.zeros(3, dtype=torch.int32, device=DEV)))
        results.append(got + _state(w))
    for x, y in zip(*results):
        assert torch.equal(x, y)


@gpu
@pytest.mark.parametrize("native", [True, False])
def test_binding_refuses_what_does_not_fit(native, monkeypatch):
    if not native:
        monkeypatch.setattr(B, "_native", lambda: None)
    w = _world(True, 6)
    cache, tree, q, lse, weights = w["cache"], w["tree"], w["q"], w["lse"], w["weights"]
    before = [x.clone() for x in _state(w)]
    ints = lambda *n: torch.zeros(n, dtype=torch.int32, device=DEV)  # noqa: E731
    bad = [
        lambda: B.kv_append(cache, tree, w["k"], w["v"].float()), lambda: B.kv_append(cache, tree, w["k"], w["v"], positions=ints(1, 2)),
        lambda: B.kv_append(cache, tree, w["k"], w["v"], positions=ints(3)), lambda: B.kv_append(cache, tree, w["k"], w["v"], axis_of=ints(4)),
        lambda: B.kv_append(cache, tree, w["k"], w["v"], inv_freq=torch.ones(8, device=DEV), positions=ints(1, 3), axis_of=torch.zeros(7, dtype=torch.uint8, device=DEV)),
        lambda: B.kv_append(cache, tree, w["k"], w["v"], k_out=w["k"].float()), lambda: B.kv_append(cache, tree, w["k"].to(torch.uint8), w["v"].to(torch.uint8)),
        lambda: B.kv_append(cache, tree, w["k"], w["v"], positions=ints(1, 3).long()),
        lambda: B.tree_attention(cache, tree, q, lse=lse[:, :, :4].contiguous()), lambda: B.tree_attention(cache, tree, q, lse=lse.double()),
        lambda: B.tree_attention(B.KVCache(cache.k, cache.v, cache.table, cache.lengths), tree, q),
        lambda: B.tree_attention(B.KVCache(cache.k, cache.v, cache.table, cache.lengths, cache.k_scales), tree, q),
        lambda: B.tree_attention(B.KVCache(cache.k, cache.v, cache.table, cache.lengths, cache.k_scales.contiguous(), cache.v_scales.contiguous()), tree, q),
        lambda: B.tree_attention(B.KVCache(cache.k, cache.v, cache.table, cache.lengths, cache.k_scales[..., :2], cache.v_scales[..., :2]), tree, q),
        lambda: B.kv_weigh(cache, tree, q, lse.double(), weights), lambda: B.kv_weigh(cache, tree, q, lse, weights.double()),
        lambda: B.kv_weigh(cache, tree, q, lse, weights[:2]), lambda: B.kv_weigh(cache, tree, q, lse, weights, out=weights[:, :9].contiguous()),
        lambda: B.kv_weigh(cache, tree, q, lse, weights.t().contiguous().t()), lambda: B.kv_weigh(cache, tree, q, lse, weights, outcome=ints(3, 14)),
        lambda: B.kv_weigh(cache, tree, q, lse, weights, layer=2 ** 32), lambda: B.kv_weigh(cache, tree, q, lse, weights[:1].expand(3, -1)),
        lambda: B.kv_evict(cache, weights, 2 ** 32 + 8), lambda: B.kv_evict(cache, weights[:2], 8), lambda: B.kv_evict(cache, weights, 8, kept=ints(3, 9)),
        lambda: B.kv_evict(cache, weights, 8, weights_out=weights[:, :9].contiguous()), lambda: B.kv_evict(cache, weights, 8, out=ints(4)),
        lambda: B.kv_evict(cache, weights, 8, first=2 ** 32), lambda: B.kv_evict(cache, weights.cpu(), 8),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            raise AssertionError("call %d" % i)
    for call in (lambda: B.kv_append(cache, tree, w["k"], w["v"], layer=2), lambda: B.kv_weigh(cache, tree, q, lse, weights, outcome=ints(3, 15)),
                 lambda: B.kv_weigh(cache, tree, q, lse, weights, scale=0.0), lambda: B.kv_evict(cache, weights, 0), lambda: B.kv_evict(cache, weights, 8, first=9),
                 lambda: B.kv_evict(cache, weights, 8, weights_out=weights[:, 1:].new_zeros(3, 2 * weights.shape[1])[:, :weights.shape[1]], out=cache.lengths[1:].new_zeros(4)[:3], recent=9),
                 lambda: B.kv_append(cache, tree, w["k"], w["v"], k_out=w["k"])):
        with pytest.raises(B.MdsdError):
            call()
    assert all(torch.equal(x, y) for x, y in zip(_state(w), before))


@gpu
@pytest.mark.parametrize("axis", [0, 1, 2, (0, 1, 2)])
def test_repeated_inputs(axis):
    """Vectors with strides of zero: the same bits as their copies give."""
    axes, results = (axis,) if isinstance(axis, int) else axis, []
    for repeated in (True, False):
        w = _world(True, 7)
        x = []
        for heads in (8, 2, 2):
            shape = [3, 15, heads, 128]
            small = _queries(*[1 if a in axes else n for a, n in enumerate(shape[:3])], 128, torch.bfloat16, heads)
            x.append(small.expand(shape) if repeated else small.expand(shape).contiguous())
        w.update(q=x[0], k=x[1], v=x[2])
        _step(w, True)
        results.append(_state(w))
    for a, b in zip(*results):
        assert torch.equal(a, b)
