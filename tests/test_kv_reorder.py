"""Reordering of the cache's slots by parents, bit for bit against host lists."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import codes_ref  # noqa: E402
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


def make(K, pages, page, slots, width, bits=16, D=16, heads=2, seed=0):
    c = K.PagedCache.new(2, pages, page, heads, D, slots, width, torch.float16, bits=bits)
    g = torch.Generator("cuda").manual_seed(seed)
    if bits == 8:
        c.data.copy_(torch.randint(0, 256, c.data.shape, generator=g, device="cuda"))
    else:
        c.data.copy_(torch.randn(c.data.shape, generator=g, device="cuda"))
    return c, kv_ref.Pages(c.data.cpu().numpy(), c.refs.cpu().numpy(), c.table.cpu().numpy(), c.length.cpu().numpy(), page)


def same(c, r):
    assert np.array_equal(c.refs.cpu().numpy(), r.refs)
    assert np.array_equal(c.length.cpu().numpy(), r.length)
    assert np.array_equal(c.table.cpu().numpy(), r.table)
    assert np.array_equal(c.data.cpu().numpy(), r.data)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("pages,page,B,G", [(40, 4, 4, 3), (5000, 4, 8, 40), (300, 1, 5, 7), (400, 16, 16, 4), (64, 64, 3, 5)])
def test_beam_steps(K, bits, pages, page, B, G):
    """Steps of a search, in pools that are roomy or run out: beams move, multiply, end and grow by a token."""
    n = B * G
    c, r = make(K, pages, page, n + 2, max(4, pages // 4), bits)
    rng = np.random.default_rng(pages + B)
    slot = rng.permutation(n + 2)[:n]
    c.extend(ints(slot[::B]), ints([2 * page + 1] * G))
    r.extend(slot[::B], [2 * page + 1] * G)
    for step in range(12):
        parent = np.concatenate([g * B + rng.integers(0, B, B) for g in range(G)])
        if step == 0:
            parent = np.repeat(np.arange(G) * B, B)
        elif step % 3 == 0:
            parent = np.where(rng.random(n) < 0.1, -1, parent)
        elif step % 5 == 0:
            parent = np.concatenate([g * B + rng.permutation(B) for g in range(G)])
        assert c.reorder(ints(slot), ints(parent)).tolist() == codes_ref.reorder(r, slot, parent)
        same(c, r)
        tokens = np.ones(n, np.int64)
        assert c.extend(ints(slot), ints(tokens)).tolist() == r.extend(slot, tokens)
        same(c, r)


def test_roles(K):
    """Every way a slot can fare: stays, moves, is copied, is emptied, does not exist, has a parent that does not."""
    c, r = make(K, 30, 4, 8, 6)
    for s, t in ((0, 6), (1, 8), (2, 3), (3, 0), (4, 9), (5, 5)):
        c.extend(ints([s]), ints([t])), r.extend([s], [t])
    slot = [0, 1, 2, 3, 4, 9, -1, 5]
    for parent in ([0, 0, 1, 1, 3, 0, 0, 5], [4, 4, 4, 4, 4, 4, 4, 4], [-1, 8, 7, 6, 5, 0, 1, 2], [1, 0, 4, 2, 7, 3, 3, 3],
                   [-5, 2 ** 31 - 1, 2, -2 ** 31, 0, 0, 0, 0]):
        assert c.reorder(ints(slot), ints(parent)).tolist() == codes_ref.reorder(r, slot, parent)
        same(c, r)


@pytest.mark.parametrize("spare", [0, 1, 2, 5])
def test_pool_runs_out(K, spare):
    """Copies are granted in order; requests that need no page keep theirs, and what nobody names frees its pages first."""
    c, r = make(K, 4 * 2 + 1 + spare, 4, 12, 4)
    c.extend(ints([0, 1, 2, 3, 4]), ints([7, 6, 8, 5, 1])), r.extend([0, 1, 2, 3, 4], [7, 6, 8, 5, 1])
    slot = [5, 6, 0, 1, 2, 3, 4, 7, 8, 9]
    parent = [2, 2, 2, 3, 4, 4, 3, 5, 4, 2]
    assert c.reorder(ints(slot), ints(parent)).tolist() == codes_ref.reorder(r, slot, parent)
    same(c, r)


def test_pages_given_up_by_a_window(K):
    """Holes are shared as holes; a partial page that is gone is not copied."""
    c, r = make(K, 20, 4, 4, 6)
    c.extend(ints([0, 1]), ints([14, 14])), r.extend([0, 1], [14, 14])
    c.release(ints([0]), ints([0]), ints([9])), r.release([0], [0], [9])
    c.table[1, 3], r.table[1, 3] = -1, -1
    slot, parent = [0, 1, 2, 3], [0, 1, 0, 1]
    assert c.reorder(ints(slot), ints(parent)).tolist() == codes_ref.reorder(r, slot, parent)
    same(c, r)


def test_largest_call(K):
    """As many requests as a call may have, all from one parent, in a pool that several workgroups rank."""
    n = 4096
    c, r = make(K, 9000, 2, n, 3, D=8)
    c.extend(ints([7]), ints([5])), r.extend([7], [5])
    slot, parent = np.arange(n), np.full(n, 7)
    assert c.reorder(ints(slot), ints(parent)).tolist() == codes_ref.reorder(r, slot, parent)
    same(c, r)
    parent = np.roll(np.arange(n), 1)
    assert c.reorder(ints(slot), ints(parent)).tolist() == codes_ref.reorder(r, slot, parent)
    same(c, r)


def test_stream_and_graph(K):
    c, r = make(K, 300, 4, 16, 40, bits=8)
    slot = np.arange(16)
    c.extend(ints(slot), ints([9] * 16)), r.extend(slot, [9] * 16)
    from paper_2601_21758_amd import ewsjf
    ws = ewsjf.Workspace()
    parent = np.asarray([0, 0, 1, 1, 2, 3, 4, 4, 8, 8, 8, 8, 15, 14, 13, 12])
    ps, pp, granted = ints(slot), ints(parent), ints(np.zeros(16))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.reorder(ps, pp, granted=granted, ws=ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert granted.tolist() == codes_ref.reorder(r, slot, parent)
    same(c, r)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.reorder(ps, pp, granted=granted, ws=ws)
    rng = np.random.default_rng(0)
    for _ in range(4):
        parent = rng.integers(-1, 16, 16)
        pp.copy_(ints(parent))
        graph.replay()
        torch.cuda.synchronize()
        assert granted.tolist() == codes_ref.reorder(r, slot, parent)
        same(c, r)
