"""Plans and the caches and batches that they belong to."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import kv
    return kv


def ints(v):
    return torch.tensor(np.asarray(v, np.int32).reshape(np.shape(v)), device="cuda")


@pytest.mark.gpu
def test_a_plan_of_another_cache(K):
    """A plan's layout follows from its cache's sizes: a cache with others is refused, one with the same is not."""
    sizes = dict(layers=1, n_pages=20, page_size=16, kv_heads=2, head_dim=64, n_slots=4, width=5, dtype=torch.float16)

    def cache(**other):
        c = K.PagedCache.new(**{**sizes, **other})
        c.extend(ints([0]), ints([40]))
        return c

    c, q = cache(), torch.randn((3, 8, 64), device="cuda").half()
    for make in (lambda c: K.prefix_plan(c, ints([0]), ints([0, 3]), None, None, total_q=3, max_q=3, q_heads=8),
                 lambda c: K.window_plan(c, ints([0]), ints([0, 3]), 9, 1, total_q=3, max_q=3, q_heads=8)):
        plan = make(c)
        want = K.attention(q, c, 0, plan)
        for other in (dict(page_size=32), dict(kv_heads=4), dict(kv_heads=1), dict(width=6), dict(width=4000),
                      dict(n_slots=2), dict(n_slots=400)):
            with pytest.raises(ValueError, match="other sizes"):
                K.attention(q, cache(**other), 0, plan)
        for other in (dict(), dict(n_pages=3), dict(layers=3)):
            for x, y in zip(K.attention(q, cache(**other), 0, plan), want):
                assert torch.equal(x, y)
        table, refs, _ = c.compact()
        c.adopt(table, refs)
        for x, y in zip(K.attention(q, c, 0, plan), want):
            assert torch.equal(x, y)


def test_queries_without_sequences():
    """No sequence could answer them: refused before anything is written or left unwritten."""
    import ctypes as C
    from paper_2601_21758_amd import _lib as L
    if not os.path.exists(L.LIB_PATH):
        pytest.skip("libewsjf.so not built")
    lib, fake = L.lib(), 0x10000
    c = L.Cache(fake, fake, fake, fake, 40960, 20480, 2048, 1024, 64, 2, 10, 16, 2, 64, L.BF16, 4, 5)
    a = C.addressof(c)
    for total, window, groups in ((1, 0, 0), (7, 5, 0)):
        b = L.Batch(0, groups, total, 1, 8, window, 0)
        p = C.addressof(b)
        assert lib.ewsjf_attention_plan_bytes(a, p) == lib.ewsjf_attention_workspace_bytes(a, p) == 0
        assert lib.ewsjf_prefix_plan(a, p, fake, fake, fake, fake, fake, 1 << 30, None) == L.ERR_ARG
        assert lib.ewsjf_window_plan(a, p, fake, fake, fake, 1 << 30, None) == L.ERR_ARG
        assert lib.ewsjf_attention(a, p, 0, fake, 512, 64, 0.125, fake, fake, fake, fake, 1 << 30, None) == L.ERR_ARG
    b = L.Batch(0, 0, 0, 1, 8, 0, 0)
    assert lib.ewsjf_attention_plan_bytes(a, C.addressof(b)) > 0
