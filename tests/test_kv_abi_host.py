"""Host-side argument checks of the cache and attention entry points: every
refusal before a device is touched, no GPU needed."""
import ctypes as C
import os

import pytest

from paper_2601_21758_amd import _lib as L

pytestmark = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libewsjf.so not built")

FAKE, MIS = 0x10000, 0x10004  # never dereferenced: calls fail validation first


def cache(**kw):
    d = dict(layers=2, n_pages=10, page_size=16, kv_heads=2, head_dim=64, dtype=L.BF16, n_slots=4, width=5)
    d.update({k: v for k, v in kw.items() if k in d})
    block = d["page_size"] * d["kv_heads"] * d["head_dim"]
    s = dict(data=FAKE, refs=FAKE, table=FAKE, length=FAKE, layer_stride=2 * d["n_pages"] * block,
             kv_stride=d["n_pages"] * block, page_stride=block, head_stride=d["page_size"] * d["head_dim"],
             token_stride=d["head_dim"])
    s.update({k: v for k, v in kw.items() if k in s})
    return L.Cache(*s.values(), *d.values())


def batch(**kw):
    d = dict(n_seqs=3, n_groups=0, total_q=7, max_q=4, q_heads=8, window=0, sinks=0)
    d.update(kw)
    return L.Batch(*d.values())


def ws_bytes(c):
    return L.lib().ewsjf_cache_workspace_bytes(C.addressof(c))


def test_struct_layouts():
    assert C.sizeof(L.Cache) == 4 * 8 + 5 * 8 + 8 * 4
    assert C.sizeof(L.Batch) == 32


def test_cache_sizes():
    assert ws_bytes(cache()) > 0
    for bad in (dict(layers=0), dict(n_pages=0), dict(n_pages=(1 << 24) + 1), dict(page_size=0), dict(page_size=12),
                dict(page_size=2048), dict(kv_heads=0), dict(head_dim=4), dict(head_dim=60), dict(head_dim=264),
                dict(dtype=2), dict(dtype=-1), dict(n_slots=0), dict(width=0), dict(width=1 << 30),
                dict(head_stride=64), dict(token_stride=72), dict(page_stride=2040), dict(page_stride=2047),
                dict(kv_stride=0), dict(kv_stride=4), dict(layer_stride=20480), dict(layer_stride=-8),
                dict(data=None), dict(refs=None), dict(table=None), dict(length=None), dict(data=MIS)):
        assert ws_bytes(cache(**bad)) == 0, bad
    assert L.lib().ewsjf_cache_workspace_bytes(None) == 0
    # dims of size 1 are never stepped over; pages may be the outermost dim; heads inside tokens
    assert ws_bytes(cache(kv_heads=1, head_stride=12345)) > 0
    assert ws_bytes(cache(page_size=1, token_stride=3)) > 0
    assert ws_bytes(cache(layers=1, layer_stride=0)) > 0
    assert ws_bytes(cache(head_stride=64, token_stride=128)) > 0
    assert ws_bytes(cache(page_stride=4 * 2048, layer_stride=2 * 2048, kv_stride=2048)) > 0


def test_page_calls():
    lib = L.lib()
    c = cache()
    a, n = C.addressof(c), ws_bytes(c)

    def extend(cc=a, slot=FAKE, tokens=FAKE, k=3, granted=FAKE, ws=FAKE, wsb=n):
        return lib.ewsjf_cache_extend(cc, slot, tokens, k, granted, ws, wsb, None)

    def fork(cc=a, parent=FAKE, child=FAKE, tokens=FAKE, k=3, granted=FAKE, ws=FAKE, wsb=n):
        return lib.ewsjf_cache_fork(cc, parent, child, tokens, k, granted, ws, wsb, None)

    for f in (extend, fork):
        assert f(cc=None) == L.ERR_NULL
        assert f(tokens=None) == f(granted=None) == f(ws=None) == L.ERR_NULL
        assert f(k=-1) == f(k=4097) == L.ERR_ARG
        assert f(ws=MIS) == L.ERR_ALIGN
        assert f(wsb=n - 1) == L.ERR_WORKSPACE
    assert extend(slot=None) == fork(parent=None) == fork(child=None) == L.ERR_NULL
    assert lib.ewsjf_cache_release(a, None, None, None, 1, None) == L.ERR_NULL
    assert lib.ewsjf_cache_release(a, FAKE, FAKE, None, 1, None) == L.ERR_NULL
    assert lib.ewsjf_cache_release(a, FAKE, None, None, 4097, None) == L.ERR_ARG
    assert lib.ewsjf_cache_copy(a, FAKE, None, 1, None) == L.ERR_NULL
    assert lib.ewsjf_cache_copy(a, FAKE, FAKE, 11, None) == L.ERR_ARG
    assert lib.ewsjf_cache_compact(a, FAKE, FAKE, None, FAKE, n, None) == L.ERR_NULL
    assert lib.ewsjf_cache_compact(a, FAKE, FAKE, FAKE, FAKE, n - 1, None) == L.ERR_WORKSPACE
    assert lib.ewsjf_cache_compact(a, FAKE, FAKE, FAKE, MIS, n, None) == L.ERR_ALIGN

    def append(layer=0, k=FAKE, v=FAKE, ks=128, vs=128, slot=FAKE, qs=FAKE, ns=2, total=5):
        return lib.ewsjf_cache_append(a, layer, k, v, ks, 64, vs, 64, slot, qs, ns, total, None)

    assert append(layer=2) == append(layer=-1) == append(ns=-1) == append(ns=4097) == append(total=-1) == L.ERR_ARG
    assert append(total=1 << 24) == append(ks=12) == append(vs=-8) == L.ERR_ARG
    assert append(k=None) == append(v=None) == append(slot=None) == append(qs=None) == L.ERR_NULL
    assert append(k=MIS) == append(v=MIS) == L.ERR_ALIGN


def test_attention_calls():
    lib = L.lib()
    c = cache()
    a = C.addressof(c)

    def sizes(**kw):
        b = batch(**kw)
        return lib.ewsjf_attention_plan_bytes(a, C.addressof(b)), lib.ewsjf_attention_workspace_bytes(a, C.addressof(b))

    assert min(sizes()) > 0
    for bad in (dict(n_seqs=-1), dict(n_seqs=4097), dict(n_groups=4), dict(n_groups=-1), dict(total_q=-1),
                dict(total_q=1 << 24), dict(max_q=0), dict(q_heads=0), dict(q_heads=7), dict(q_heads=130),
                dict(window=-1), dict(sinks=3), dict(window=4, sinks=-1), dict(window=4, n_groups=1)):
        assert sizes(**bad) == (0, 0), bad
    wide = cache(head_dim=96)
    assert lib.ewsjf_attention_plan_bytes(C.addressof(wide), C.addressof(batch())) == 0

    def prefix(b, slot=FAKE, qs=FAKE, gs=FAKE, sh=FAKE, plan=FAKE, nb=1 << 30):
        return lib.ewsjf_prefix_plan(a, C.addressof(b) if b else None, slot, qs, gs, sh, plan, nb, None)

    def window(b, slot=FAKE, qs=FAKE, plan=FAKE, nb=1 << 30):
        return lib.ewsjf_window_plan(a, C.addressof(b) if b else None, slot, qs, plan, nb, None)

    g, w = batch(n_groups=2), batch(window=5, sinks=1)
    assert prefix(None) == prefix(g, slot=None) == prefix(g, qs=None) == prefix(g, plan=None) == L.ERR_NULL
    assert prefix(g, gs=None) == prefix(g, sh=None) == L.ERR_NULL
    assert prefix(w) == window(g) == window(batch()) == L.ERR_ARG
    assert prefix(g, plan=MIS) == window(w, plan=MIS) == L.ERR_ALIGN
    assert prefix(g, nb=sizes(n_groups=2)[0] - 1) == window(w, nb=1) == L.ERR_WORKSPACE
    assert window(None) == window(w, slot=None) == L.ERR_NULL

    need = sizes()[1]
    b = batch()

    def attend(bb=b, layer=0, q=FAKE, qt=512, qh=64, scale=0.125, plan=FAKE, out=FAKE, lse=FAKE, ws=FAKE, nb=need):
        return lib.ewsjf_attention(a, C.addressof(bb) if bb else None, layer, q, qt, qh, scale, plan, out, lse, ws, nb,
                                   None)

    assert attend(bb=None) == attend(q=None) == attend(plan=None) == attend(out=None) == attend(ws=None) == L.ERR_NULL
    assert attend(layer=2) == attend(layer=-1) == attend(qt=100) == attend(qh=-64) == L.ERR_ARG
    for s in (0.0, -0.125, float("nan"), float("inf")):
        assert attend(scale=s) == L.ERR_ARG
    assert attend(bb=batch(q_heads=9)) == L.ERR_ARG
    assert attend(q=MIS) == attend(out=MIS) == attend(plan=MIS) == attend(ws=MIS) == L.ERR_ALIGN
    assert attend(nb=need - 1) == L.ERR_WORKSPACE
