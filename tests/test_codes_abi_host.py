"""Host-side argument checks of the 8-bit cache, its reading, the reordering and
the beams' selection: every refusal before a device is touched, no GPU needed."""
import ctypes as C
import math
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import codes_ref  # noqa: E402

from paper_2601_21758_amd import _lib as L  # noqa: E402

FAKE, MIS = 0x10000, 0x10004  # never dereferenced: calls fail validation first
needs_library = pytest.mark.skipif(not os.path.exists(L.LIB_PATH), reason="libewsjf.so not built")


def cache(**kw):
    d = dict(layers=2, n_pages=10, page_size=16, kv_heads=2, head_dim=64, dtype=L.E4M3_BF16, n_slots=4, width=5)
    d.update({k: v for k, v in kw.items() if k in d})
    block = -(-d["page_size"] * d["kv_heads"] * (d["head_dim"] + 1) // 16) * 16
    s = dict(data=FAKE, refs=FAKE, table=FAKE, length=FAKE, layer_stride=2 * d["n_pages"] * block,
             kv_stride=d["n_pages"] * block, page_stride=block, head_stride=d["page_size"] * d["head_dim"],
             token_stride=d["head_dim"])
    s.update({k: v for k, v in kw.items() if k in s})
    return L.Cache(*s.values(), *d.values())


def ws_bytes(c):
    return L.lib().ewsjf_cache_workspace_bytes(C.addressof(c))


def beams(**kw):
    d = dict(groups=3, beams=4, picks=8, vocab=1000, dtype=L.BF16, end=2, row_stride=1000)
    d.update(kw)
    return L.Beams(*d.values())


@needs_library
def test_cache_sizes():
    for dtype in (L.E4M3_BF16, L.E4M3_F16):
        assert ws_bytes(cache(dtype=dtype)) > 0
        for bad in (dict(head_dim=8), dict(head_dim=72), dict(head_dim=272), dict(page_stride=2048), dict(page_stride=2088),
                    dict(kv_stride=2080), dict(layer_stride=2080 * 10 + 8), dict(head_stride=32), dict(data=MIS)):
            assert ws_bytes(cache(dtype=dtype, **bad)) == 0, bad
    assert ws_bytes(cache(dtype=7)) == 0 and ws_bytes(cache(dtype=10)) == 0
    assert ws_bytes(cache(head_stride=64, token_stride=128)) > 0
    assert ws_bytes(cache(page_stride=2096, kv_stride=20960, layer_stride=41920)) > 0


@needs_library
def test_page_bytes():
    f = L.lib().ewsjf_cache_page_bytes
    assert f(16, 2, 64, L.E4M3_BF16) == 2 * 16 * 65
    assert f(1, 3, 16, L.E4M3_F16) == 64  # 51 bytes up to a multiple of 16
    assert f(16, 2, 64, L.BF16) == 2 * 16 * 64 * 2
    for bad in ((12, 2, 64, 8), (16, 0, 64, 8), (16, 2, 24, 8), (16, 2, 64, 3), (0, 2, 64, 8), (2048, 2, 64, 8)):
        assert f(*bad) == 0, bad


@needs_library
def test_read():
    lib, c = L.lib(), cache()

    def read(c=c, layer=0, slot=FAKE, start=FAKE, begin=None, n=2, total=7, k=FAKE, v=FAKE):
        return lib.ewsjf_cache_read(C.addressof(c) if c is not None else None, layer, slot, start, begin, n, total, k, v, None)

    assert read(c=None) == L.ERR_NULL
    for kw in (dict(layer=-1), dict(layer=2), dict(n=-1), dict(n=4097), dict(total=-1), dict(total=2 ** 31 + 1)):
        assert read(**kw) == L.ERR_ARG, kw
    for kw in (dict(slot=None), dict(start=None), dict(k=None), dict(v=None)):
        assert read(**kw) == L.ERR_NULL, kw
    assert read(k=MIS) == L.ERR_ALIGN and read(v=MIS) == L.ERR_ALIGN


@needs_library
def test_reorder():
    lib, c = L.lib(), cache()
    need = lib.ewsjf_cache_reorder_workspace_bytes(C.addressof(c), 4)
    assert need >= 4 * 5 * 4
    assert lib.ewsjf_cache_reorder_workspace_bytes(C.addressof(c), 4097) == 0
    assert lib.ewsjf_cache_reorder_workspace_bytes(C.addressof(c), -1) == 0
    assert lib.ewsjf_cache_reorder_workspace_bytes(None, 1) == 0

    def reorder(slot=FAKE, parent=FAKE, n=4, granted=FAKE, ws=FAKE, size=need):
        return lib.ewsjf_cache_reorder(C.addressof(c), slot, parent, n, granted, ws, size, None)

    assert reorder(n=-1) == L.ERR_ARG and reorder(n=4097) == L.ERR_ARG
    for kw in (dict(slot=None), dict(parent=None), dict(granted=None), dict(ws=None)):
        assert reorder(**kw) == L.ERR_NULL, kw
    assert reorder(ws=MIS) == L.ERR_ALIGN and reorder(size=need - 1) == L.ERR_WORKSPACE


@needs_library
def test_beam_select():
    lib = L.lib()
    assert lib.ewsjf_beam_workspace_bytes(C.addressof(beams())) > 0
    assert lib.ewsjf_beam_workspace_bytes(C.addressof(beams(groups=0))) > 0
    assert lib.ewsjf_beam_workspace_bytes(None) == 0
    for bad in (dict(groups=-1), dict(groups=4097), dict(beams=0), dict(beams=33), dict(groups=1025), dict(picks=0),
                dict(picks=65), dict(vocab=0), dict(vocab=(1 << 22) + 1, row_stride=1 << 23), dict(dtype=3), dict(dtype=-1),
                dict(row_stride=999), dict(row_stride=0), dict(row_stride=1 << 50)):
        assert lib.ewsjf_beam_workspace_bytes(C.addressof(beams(**bad))) == 0, bad

    def select(b=None, logits=FAKE, score=FAKE, done=None, out=(FAKE, FAKE, FAKE), ws=FAKE, size=1 << 30):
        b = beams() if b is None else b
        return lib.ewsjf_beam_select(C.addressof(b), logits, score, done, *out, ws, size, None)

    assert lib.ewsjf_beam_select(None, FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, 1 << 30, None) == L.ERR_NULL
    assert select(beams(picks=65)) == L.ERR_ARG
    assert select(beams(end=-1), done=FAKE) == L.ERR_ARG and select(beams(end=1000), done=FAKE) == L.ERR_ARG
    for kw in (dict(logits=None), dict(score=None), dict(out=(None, FAKE, FAKE)), dict(out=(FAKE, None, FAKE)),
               dict(out=(FAKE, FAKE, None)), dict(ws=None)):
        assert select(**kw) == L.ERR_NULL, kw
    assert select(logits=FAKE + 1) == L.ERR_ALIGN and select(beams(dtype=L.F32), logits=FAKE + 2) == L.ERR_ALIGN
    assert select(ws=MIS) == L.ERR_ALIGN and select(size=100) == L.ERR_WORKSPACE


def test_quantised_reference():
    """The tests' own quantiser against the format's definition, by trying every code."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((50, 16)) * np.exp2(rng.integers(-30, 15, (50, 1)))
    code, scale, value = codes_ref.quantise(x, "f16")
    top = np.abs(x).max(-1)
    s = np.exp2(scale.astype(float) - 127)
    assert np.all(top <= 448 * s) and np.all((top > 224 * s) | (scale == 10))
    every = codes_ref.values(np.arange(256, dtype=np.uint8)[None, :].repeat(50, 0), scale)
    best = np.nanmin(np.abs(x[:, :, None] - every[:, None, :]), -1)
    assert np.array_equal(np.abs(x - value), best)
    ties = np.asarray([[448.0, 17.0, 19.0, 2.0 ** -10, 3 * 2.0 ** -10, -17.0, 0.0, -0.0]])
    assert codes_ref.quantise(ties, "f16")[2].tolist() == [[448, 16, 20, 0, 2.0 ** -8, -16, 0, 0]]


def test_select_reference():
    x = np.log(np.asarray([[0.5, 0.25, 0.25], [0.9, 0.05, 0.05]]))
    p, t, s = codes_ref.select(x, np.asarray([0.0, math.log(0.5)]), 2, 4)
    assert p.tolist() == [[0, 1, 0, 0]] and t.tolist() == [[0, 0, 1, 2]]
    assert np.allclose(np.exp(s), [[0.5, 0.45, 0.25, 0.25]])
    p, t, s = codes_ref.select(x, np.asarray([-1.0, -0.5]), 2, 3, [0, 1], 7)
    assert p.tolist() == [[1, 0, 0]] and t.tolist() == [[7, 0, 1]]
