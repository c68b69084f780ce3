"""Pages of the key/value cache: extend, fork, release, copy, compact, append,
bit for bit against host lists, over random sequences of requests."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import kv_ref  # noqa: E402

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import kv
    return kv


def ints(v):
    return torch.tensor(np.asarray(v, np.int32).reshape(np.shape(v)), device="cuda")


def make(K, pages, page, slots, width, layers=2, heads=2, D=8, dtype=torch.float16, order="head", seed=0):
    c = K.PagedCache.new(layers, pages, page, heads, D, slots, width, dtype=dtype)
    g = torch.Generator("cuda").manual_seed(seed)
    c.data.copy_(torch.randn(c.data.shape, generator=g, device="cuda"))
    if order == "token":
        c = K.PagedCache.of(c.data.transpose(3, 4).contiguous().transpose(3, 4), c.refs, c.table, c.length)
    return c, kv_ref.Pages(c.data.cpu().float().numpy(), c.refs.cpu().numpy(), c.table.cpu().numpy(),
                           c.length.cpu().numpy(), page)


def same(c, r):
    assert np.array_equal(c.refs.cpu().numpy(), r.refs)
    assert np.array_equal(c.length.cpu().numpy(), r.length)
    assert np.array_equal(c.table.cpu().numpy(), r.table)
    assert np.array_equal(c.data.cpu().float().numpy(), r.data)


@pytest.mark.parametrize("pages,page,slots,width,order", [(37, 1, 9, 20, "head"), (64, 4, 12, 9, "token"),
                                                          (200, 16, 30, 8, "head"), (9001, 2, 40, 300, "token")])
def test_random_requests(K, pages, page, slots, width, order):
    """Long runs of mixed requests, pools that run out, slots that do not exist."""
    c, r = make(K, pages, page, slots, width, order=order, seed=pages)
    rng = np.random.default_rng(pages)
    for step in range(40):
        n = int(rng.integers(1, slots + 1))
        pick = rng.permutation(np.arange(-1, slots + 1))[:n]
        kind = rng.choice(["extend", "extend", "fork", "fork", "release", "trim", "append", "compact", "copy"])
        if kind == "extend":
            t = rng.integers(-1, page * width // 3 + 2, n)
            assert c.extend(ints(pick), ints(t)).tolist() == r.extend(pick, t)
        elif kind == "fork":
            half = max(1, n // 2)
            child, others = pick[:half], pick[half:]
            if not others.size:
                continue
            parent = rng.choice(others, half)
            have = np.asarray([r.length[p] if 0 <= p < slots else 3 for p in parent])
            t = np.where(rng.random(half) < 0.4, have, (have * rng.random(half) * 1.1).astype(np.int64))
            assert c.fork(ints(parent), ints(child), ints(t)).tolist() == r.fork(parent, child, t)
        elif kind == "release":
            some = pick[:max(1, n // 4)]
            c.release(ints(some))
            r.release(some)
        elif kind == "trim":
            lens = np.asarray([r.length[s] if 0 <= s < slots else 9 for s in pick])
            b, e = rng.integers(-2, 8, n), (lens * rng.random(n) * 1.3).astype(np.int64)
            c.release(ints(pick), ints(b), ints(e))
            r.release(pick, b, e)
        elif kind == "append":
            new = rng.integers(0, 4, n)
            q_start = np.concatenate([[0], np.cumsum(new)])
            # only pages of the slot's own may be written: others would race
            own = [s for s in pick if 0 <= s < slots and all(
                r.refs[p] <= 1 for p in r.table[s] if 0 <= p < pages)]
            keep = np.isin(pick, own)
            new = np.where(keep, new, 0)
            q_start = np.concatenate([[0], np.cumsum(new)])
            k, v = (torch.randn((int(q_start[-1]), 2, 8), device="cuda").half() for _ in range(2))
            c.append(1, k, v, ints(pick), ints(q_start))
            r.append(1, k.cpu().float().numpy(), v.cpu().float().numpy(), pick, q_start)
        elif kind == "compact":
            table, refs, used = c.compact()
            want = r.compact()
            assert np.array_equal(table.cpu().numpy(), want[0]) and np.array_equal(refs.cpu().numpy(), want[1])
            assert used.item() == want[2]
            if rng.random() < 0.5:  # the old rows still read right; the new ones take over
                c.adopt(table, refs)
                r.table, r.refs = want[0], want[1]
        else:
            free = [p for p in range(pages) if r.refs[p] == 0]
            m = min(5, len(free))
            src, dst = rng.integers(-1, pages + 1, m), rng.permutation(free)[:m] if m else np.zeros(0)
            src = np.where(np.isin(src, dst), -1, src)
            c.copy(ints(src), ints(dst))
            for a, b in zip(src, dst):
                if 0 <= a < pages:
                    r.data[:, :, int(b)] = r.data[:, :, a]
        same(c, r)


def test_compact_in_place(K):
    c, r = make(K, 5000, 2, 50, 200, seed=3)
    c.extend(ints(range(50)), ints([97] * 50))
    r.extend(range(50), [97] * 50)
    c.fork(ints([1, 1, 2]), ints([3, 4, 5]), ints([0, 0, 0]))
    drop = list(range(0, 40, 2))
    c.release(ints(drop)), r.release(drop)
    c.fork(ints([1, 1, 7]), ints([0, 2, 4]), ints([97, 50, 31]))
    r.fork([1, 1, 7], [0, 2, 4], [97, 50, 31])
    same(c, r)
    used = torch.empty(1, dtype=torch.int32, device="cuda")
    c.compact(out=(c.table, c.refs, used))
    r.table, r.refs, U = r.compact()
    assert used.item() == U
    same(c, r)
    # nothing is left to move
    before = c.data.clone()
    c.compact(out=(c.table, c.refs, used))
    assert torch.equal(before, c.data)
    same(c, r)


def test_compact_empty_and_full(K):
    for fill in (0, 1):
        c, r = make(K, 33, 4, 3, 11)
        if fill:
            assert c.extend(ints([0, 1, 2]), ints([44, 44, 44])).tolist() == [1, 1, 1] == r.extend([0, 1, 2], [44] * 3)
        table, refs, used = c.compact()
        assert used.item() == 33 * fill
        assert torch.equal(table, c.table) and torch.equal(refs, c.refs)
        same(c, r)


def test_served_in_order(K):
    """The pool runs out in the middle of a call; what comes after is refused, what needs no page with it."""
    c, r = make(K, 10, 4, 6, 10)
    want = [16, 12, 16, 1, 0]
    assert c.extend(ints([3, 1, 0, 2, 4]), ints(want)).tolist() == r.extend([3, 1, 0, 2, 4], want) == [1, 1, 0, 0, 0]
    same(c, r)


def test_many_slots_and_empty_calls(K):
    n = 4096
    c, r = make(K, 20000, 2, n, 16, layers=1, heads=1)
    t = np.random.default_rng(5).integers(0, 12, n)
    assert c.extend(ints(range(n)), ints(t)).tolist() == r.extend(range(n), t)
    same(c, r)
    none = ints(np.zeros(0))
    c.extend(none, none), c.fork(none, none, none), c.release(none), c.copy(none, none)
    c.append(0, torch.zeros((0, 1, 8), dtype=torch.float16, device="cuda"),
             torch.zeros((0, 1, 8), dtype=torch.float16, device="cuda"), none, ints([0]))
    same(c, r)
    assert c.extend(ints([0]), ints([10 ** 9])).tolist() == [0]
    same(c, r)


def test_append_strides(K):
    """Keys and values as slices of a fused projection, several tokens a sequence, fewer held than given."""
    c, r = make(K, 40, 8, 5, 8, heads=3, D=16)
    c.extend(ints([0, 2, 4]), ints([20, 3, 9])), r.extend([0, 2, 4], [20, 3, 9])
    q_start = [0, 7, 12, 12]
    x = torch.randn((12, 10, 16), device="cuda").half()
    k, v = x[:, 4:7], x[:, 7:10]
    c.append(1, k, v, ints([0, 2, 4]), ints(q_start))
    r.append(1, k.cpu().float().numpy(), v.cpu().float().numpy(), [0, 2, 4], q_start)
    same(c, r)


def test_forked_rows_read_alike(K):
    """A fork, its growth and an append change nothing that the parent's row names."""
    c, r = make(K, 60, 16, 4, 10, D=64)
    c.extend(ints([0]), ints([100])), r.extend([0], [100])
    before = [c.data[:, :, p].clone() for p in r.table[0] if p >= 0]
    c.fork(ints([0, 0]), ints([1, 2]), ints([100, 90])), r.fork([0, 0], [1, 2], [100, 90])
    c.extend(ints([1, 2]), ints([5, 5])), r.extend([1, 2], [5, 5])
    k, v = (torch.randn((10, 2, 64), device="cuda").half() for _ in range(2))
    c.append(0, k, v, ints([1, 2]), ints([0, 5, 10]))
    r.append(0, k.cpu().float().numpy(), v.cpu().float().numpy(), [1, 2], [0, 5, 10])
    same(c, r)
    for x, p in zip(before, [p for p in r.table[0] if p >= 0]):
        assert torch.equal(x, c.data[:, :, p])


def test_graph_replays(K):
    """The requests of a step, captured: replays with the program's own work between them."""
    c, r = make(K, 300, 4, 20, 30)
    c.extend(ints([0]), ints([50])), r.extend([0], [50])
    parent, child, t, new = ints([0] * 8), ints(range(4, 12)), ints([50, 49, 48, 7, 3, 50, 11, 20]), ints([1] * 8)
    ws, granted = K.Workspace(), ints([0] * 8)
    ws.get(c._ws_bytes)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.release(child)
        c.fork(parent, child, t, granted=granted, ws=ws)
        c.extend(child, new, granted=granted, ws=ws)
    for i in range(4):
        graph.replay()
        torch.cuda.synchronize()
        r.release(child.tolist())
        r.fork(parent.tolist(), child.tolist(), t.tolist())
        assert granted.tolist() == r.extend(child.tolist(), new.tolist())
        same(c, r)
        torch.ones(1 << 20, device="cuda").sum().item()


def test_refusals(K):
    c, _ = make(K, 10, 4, 6, 10)
    with pytest.raises(ValueError):
        K.PagedCache.new(1, 10, 3, 2, 64, 4, 4)      # pages of three tokens
    with pytest.raises(ValueError):
        K.PagedCache.new(1, 10, 2048, 2, 64, 4, 4)
    with pytest.raises(ValueError):
        K.PagedCache.new(1, 10, 4, 2, 12, 4, 4)      # heads that 16 bytes do not divide
    with pytest.raises(ValueError):
        K.PagedCache.of(c.data[:1].expand(2, -1, -1, -1, -1, -1), c.refs, c.table, c.length)  # layers that overlap
    with pytest.raises(ValueError):
        K.PagedCache.of(c.data, c.refs[:5], c.table, c.length)
    with pytest.raises(TypeError):
        K.PagedCache.of(c.data, c.refs.long(), c.table, c.length)
    with pytest.raises(TypeError):
        c.extend(torch.zeros(2, dtype=torch.int64, device="cuda"), ints([1, 1]))
    with pytest.raises(ValueError):
        c.extend(ints([0, 1]), ints([1]))
    with pytest.raises(K.L.EwsjfError):
        c.release(ints(np.zeros(4097)))
    with pytest.raises(K.L.EwsjfError):
        c.release(ints([0]), begin=ints([0]))
    with pytest.raises(TypeError):
        c.append(0, torch.zeros((1, 2, 4), dtype=torch.float16, device="cuda"),
                 torch.zeros((1, 2, 8), dtype=torch.float16, device="cuda"), ints([0]), ints([0, 1]))
    x = torch.zeros((1, 2, 8), dtype=torch.float16, device="cuda")
    with pytest.raises(K.L.EwsjfError):
        c.append(2, x, x, ints([0]), ints([0, 1]))


@pytest.mark.parametrize("pages", [1024, 70000])
def test_needs_past_32_bits(K, pages):
    """Requests that together need 2^32 pages and more: what follows the first that does not fit is refused too."""
    width = 1 << 20
    c, _ = make(K, pages, 1, 2, width, layers=1, heads=1)
    n = K.L.MAX_CACHE_BATCH
    t = np.full(n, width)
    t[0], t[-1] = 5, 0
    s = np.zeros(n)
    s[0] = 1
    assert c.extend(ints(s), ints(t)).tolist() == [1] + [0] * (n - 1)
    assert int(c.refs.sum()) == 5 and c.length.tolist() == [0, 5]
    assert c.table[1, :5].tolist() == [0, 1, 2, 3, 4] and int((c.table >= 0).sum()) == 5


@pytest.mark.parametrize("page,order", [(1, "head"), (4, "token")])
def test_a_large_pool(K, page, order):
    """Pools that one workgroup does not rank."""
    c, r = make(K, 70001, page, 9, 20000, layers=1, heads=1, order=order)
    rng = np.random.default_rng(page)
    for step in range(6):
        pick, t = rng.permutation(8), rng.integers(0, 20000, 8)
        assert c.extend(ints(pick), ints(t)).tolist() == r.extend(pick, t)
        half = r.length[pick[0]] // 2
        c.release(ints(pick[4:])), r.release(pick[4:])
        assert c.fork(ints(pick[:1]), ints(pick[5:6]), ints([half])).tolist() == r.fork(pick[:1], pick[5:6], [half])
        same(c, r)
        out = c.compact()
        table, refs, used = r.compact()
        assert np.array_equal(out[0].cpu().numpy(), table) and np.array_equal(out[1].cpu().numpy(), refs)
        c.adopt(*out[:2])
        r.table, r.refs = table, refs
        r.data[:] = c.data.cpu().float().numpy()
        same(c, r)
