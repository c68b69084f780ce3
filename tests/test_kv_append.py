"""Appends of requests that found no room: what other slots hold, and what the
slot held before, stays; with the grants and without them."""
import copy
import ctypes as C
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import kv_ref  # noqa: E402

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import kv
    return kv


def ints(v):
    return torch.tensor(np.asarray(v, np.int32).reshape(np.shape(v)), device="cuda")


def make(K, pages, page, slots, width, heads=2, D=8, seed=0):
    c = K.PagedCache.new(2, pages, page, heads, D, slots, width, dtype=torch.float16)
    g = torch.Generator("cuda").manual_seed(seed)
    c.data.copy_(torch.randn(c.data.shape, generator=g, device="cuda"))
    return c, kv_ref.Pages(c.data.cpu().float().numpy(), c.refs.cpu().numpy(), c.table.cpu().numpy(),
                           c.length.cpu().numpy(), page)


def same(c, r):
    assert np.array_equal(c.refs.cpu().numpy(), r.refs)
    assert np.array_equal(c.length.cpu().numpy(), r.length)
    assert np.array_equal(c.table.cpu().numpy(), r.table)
    assert np.array_equal(c.data.cpu().float().numpy(), r.data)


def append(r, layer, k, v, slot, new, granted=None):
    """The definition: refused requests write nothing; without grants, nothing goes to a whole page that others hold."""
    for b, s in enumerate(slot):
        if granted is not None and not granted[b]:
            continue
        for i in range(new[b]):
            pos = r.length[s] - new[b] + i
            page = r.table[s, pos // r.ps] if pos >= 0 else -1
            whole = pos // r.ps < r.length[s] // r.ps
            if page < 0 or (granted is None and whole and r.refs[page] > 1):
                continue
            at = sum(new[:b]) + i
            r.data[layer, 0, page, :, pos % r.ps], r.data[layer, 1, page, :, pos % r.ps] = k[at], v[at]


@pytest.mark.gpu
@pytest.mark.parametrize("page,tokens,new", [(4, 16, 1), (4, 16, 3), (16, 32, 20), (8, 21, 5), (1, 9, 2), (16, 40, 70)])
@pytest.mark.parametrize("grants", [False, True])
def test_pool_runs_out_among_children(K, page, tokens, new, grants):
    """Twelve children of one parent, at its end and inside it; some find no room for their new tokens."""
    results, at = [], [tokens, tokens - tokens % page, max(page, tokens // 2 // page * page), max(1, tokens - 1)]
    t = [at[i % 4] for i in range(12)]
    for _ in range(3):
        copies = sum(x % page > 0 for x in t)
        c, r = make(K, -(-tokens // page) + copies + 5 * -(-new // page), page, 14, 30 + tokens + new, seed=tokens)
        child, n = list(range(1, 13)), [new] * 12
        c.extend(ints([0]), ints([tokens])), r.extend([0], [tokens])
        parents = [c.data[:, :, p].clone() for p in r.table[0] if p >= 0]
        assert c.fork(ints([0] * 12), ints(child), ints(t)).tolist() == r.fork([0] * 12, child, t) == [1] * 12
        granted = c.extend(ints(child), ints(n))
        want = r.extend(child, n)
        assert granted.tolist() == want and 0 < sum(want) < 12
        g = torch.Generator("cuda").manual_seed(new)
        k, v = (torch.randn((12 * new, 2, 8), generator=g, device="cuda").half() for _ in range(2))
        before = c.data.clone()
        c.append(1, k, v, ints(child), ints(np.arange(13) * new), granted=granted if grants else None)
        wrong = copy.deepcopy(r)
        host = [x.cpu().float().numpy() for x in (k, v)]
        append(r, 1, *host, child, n, want if grants else None)
        same(c, r)
        for x, p in zip(parents, r.table[0]):
            assert torch.equal(x, c.data[:, :, p])
        assert torch.equal(before[0], c.data[0])
        for s, ok, x in zip(child, want, t):  # what a refused request held
            for j in range(x if not ok and grants else 0):
                p = r.table[s, j // page]
                assert torch.equal(before[:, :, p, :, j % page], c.data[:, :, p, :, j % page])
        results.append(c.data.clone())
        # an oracle that writes wherever a page is held is told apart
        append(wrong, 1, *host, child, n, [1] * 12)
        assert not np.array_equal(wrong.data, r.data)
    assert all(torch.equal(results[0], x) for x in results[1:])


@pytest.mark.gpu
def test_forked_before_it_is_written(K):
    """A prompt's whole pages shared first and written afterwards: with the grants they are written."""
    c, r = make(K, 20, 8, 4, 8)
    granted = c.extend(ints([0]), ints([24]))
    r.extend([0], [24])
    c.fork(ints([0, 0]), ints([1, 2]), ints([24, 16])), r.fork([0, 0], [1, 2], [24, 16])
    k, v = (torch.randn((24, 2, 8), device="cuda").half() for _ in range(2))
    c.append(0, k, v, ints([0]), ints([0, 24]), granted=granted)
    append(r, 0, k.cpu().float().numpy(), v.cpu().float().numpy(), [0], [24], [1])
    same(c, r)
    assert np.array_equal(r.data[0, 0, r.table[1, 2], :, 7], k[23].cpu().float().numpy())


@pytest.mark.gpu
@pytest.mark.parametrize("spare", [0, 3, 7, 11, 40])
def test_refused_requests_have_no_slot(K, spare):
    """A step whose pool runs out in the fork or in the extend: refused requests hold, write and see nothing, the others
    what the definition says."""
    page, n, new, heads, D = 16, 8, 3, 2, 64
    c, r = make(K, 3 + spare, page, n + 1, 6, heads=heads, D=D, seed=spare)
    c.extend(ints([0]), ints([47])), r.extend([0], [47])
    child, t = list(range(1, n + 1)), [47, 40, 32, 20, 47, 46, 16, 35]
    granted = c.fork(ints([0] * n), ints(child), ints(t))
    forked = r.fork([0] * n, child, t)
    assert granted.tolist() == forked
    slot = torch.where(granted > 0, ints(child), -1)
    granted = c.extend(slot, ints([new] * n))
    held = [s if ok else -1 for s, ok in zip(child, forked)]
    want = r.extend(held, [new] * n)
    assert granted.tolist() == want
    slot, held = torch.where(granted > 0, slot, -1), [s if ok else -1 for s, ok in zip(held, want)]
    q_start = np.arange(n + 1) * new
    x = torch.randn((n * new, 4 * heads, D), device="cuda").half()
    k, v, q = x[:, :heads], x[:, heads:2 * heads], x[:, 2 * heads:]
    plan = K.prefix_plan(c, slot, ints(q_start), ints([0, n]), ints([16]), total_q=n * new, max_q=new, q_heads=2 * heads)
    c.append(0, k, v, slot, ints(q_start), granted=granted)
    host = [y.cpu().float().numpy() for y in (k, v)]
    append(r, 0, *host, held, [new] * n, want)
    same(c, r)
    out, lse = K.attention(q, c, 0, plan)
    ref = kv_ref.attention(q.cpu().double().numpy(), r.data[0].astype(np.float64), r.table, r.length, held, q_start, page,
                           D ** -0.5)
    b_out, b_lse = kv_ref.bounds(*ref, 2.0 ** -11, 50, float(np.abs(r.data).max()), D)
    fine = np.isfinite(ref[1])
    assert fine.any() == (sum(want) > 0) and np.array_equal(np.isfinite(lse.cpu().numpy()), fine)
    assert np.all(np.abs(out.cpu().double().numpy() - ref[0]) <= b_out) and not out[~torch.tensor(fine)].any()
    assert np.all(np.abs(lse.cpu().double().numpy()[fine] - ref[1][fine]) <= b_lse[fine])
    c.release(slot), r.release(held)
    same(c, r)


@pytest.mark.gpu
def test_grants_are_checked(K):
    c, _ = make(K, 10, 4, 6, 10)
    x = torch.zeros((1, 2, 8), dtype=torch.float16, device="cuda")
    with pytest.raises(TypeError):
        c.append(0, x, x, ints([0]), ints([0, 1]), granted=torch.ones(1, device="cuda"))
    with pytest.raises(ValueError):
        c.append(0, x, x, ints([0]), ints([0, 1]), granted=ints([1, 1]))


def test_refusals_on_the_host():
    from paper_2601_21758_amd import _lib as L
    if not os.path.exists(L.LIB_PATH):
        pytest.skip("libewsjf.so not built")
    fake, c = 0x10000, L.Cache(0x10000, 0x10000, 0x10000, 0x10000, 40960, 20480, 2048, 1024, 64, 2, 10, 16, 2, 64, L.BF16,
                               4, 5)

    def call(cc=c, layer=0, k=fake, v=fake, ks=128, vs=128, slot=fake, qs=fake, granted=fake, ns=2, total=5):
        return L.lib().ewsjf_cache_append_granted(C.addressof(cc) if cc else None, layer, k, v, ks, 64, vs, 64, slot, qs,
                                                  granted, ns, total, None)

    assert call(cc=None) == call(k=None) == call(v=None) == call(slot=None) == call(qs=None) == L.ERR_NULL
    assert call(layer=2) == call(ns=4097) == call(total=-1) == call(total=1 << 24) == call(ks=12) == L.ERR_ARG
    assert call(k=fake + 4) == call(v=fake + 4) == L.ERR_ALIGN
