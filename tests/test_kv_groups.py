"""The plan's rules for shared prefixes where they count: tables so wide that a
group's shared keys are a phase of their own, in one kernel with the sequences'
own keys and in two, against the definition in 64 bits."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_kv_attention import Batch, ints, widen  # noqa: E402

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HEAVY = pytest.mark.parametrize("heavy", [False, True])


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import kv
    return kv


def plans(K, b, cache=None):
    """The batch's plan, whose shared keys are a phase of their own, and the one without groups."""
    c = cache or b.cache(K)
    args = [ints(x) for x in (b.slot, b.q_start, b.group_start, b.shared)]
    kw = dict(total_q=b.total, max_q=b.max_q, q_heads=b.Hq)
    plan, alone = K.prefix_plan(c, *args, **kw), K.prefix_plan(c, *args[:2], None, None, **kw)
    assert plan.ws_bytes > alone.ws_bytes
    return c, plan, alone


def check(K, b):
    """With groups and without, against the definition."""
    c, plan, alone = plans(K, b)
    ref = b.reference(b.D ** -0.5)
    for p in (plan, alone):
        b.compare(*K.attention(b.q, c, 0, p), ref)


def same_pages(b, members, tokens):
    """The members' rows name the first one's pages there."""
    pages = -(-tokens // b.page)
    for i in members[1:]:
        b.table[b.slot[i], :pages] = b.table[b.slot[members[0]], :pages]


@HEAVY
@pytest.mark.parametrize("dtype,D,group", [("bf16", 128, 4), ("f16", 64, 8)])
def test_shared_beyond_a_member(K, heavy, dtype, D, group):
    """More than a member has before its first query, all of 32 bits, less than nothing; groups of one."""
    b = widen(Batch(51, dtype, D, 2, group, 16, [340, 333, 364, 290, 300, 410], [2, 33, 1, 1, 4, 3],
                    shared=[(3, 320), (1, 280), (2, 288)]), heavy)
    check(K, b)  # 300 tokens lie before every query of the first group, 288 count; 288 of the last
    same_pages(b, [0, 1, 2], 300)
    b.shared[:] = [1000, 2 ** 31 - 1, -5]
    check(K, b)
    b.shared[:] = [300, 0, 17]
    check(K, b)
    b.shared[:] = [15, -2 ** 31, 2]  # nothing that counts
    check(K, b)


@HEAVY
def test_first_members_without_queries(K, heavy):
    """The shared keys are read from the first member that has queries, whatever the rows before it name."""
    b = widen(Batch(52, "bf16", 128, 2, 4, 16, [250, 300, 310, 270], [0, 1, 2, 0], shared=[(4, 240)]), heavy)
    b.table[b.slot[0]] = -1
    b.length[b.slot[3]] = 7  # shorter than what the others share
    check(K, b)
    b.table[b.slot[0]] = b.table[b.slot[1], ::-1]
    check(K, b)
    b.slot[0] = -1
    check(K, b)


@HEAVY
@pytest.mark.parametrize("page", [8, 16, 64])
def test_groups_and_sequences_outside_them(K, heavy, page):
    """Empty groups, sequences before, between and after the groups, members that each have all lengths of queries."""
    lengths = [150, 230, 260, 200, 215, 90, 333, 340, 77]
    b = Batch(53, "f16", 64, 2, 4, page, lengths, [3, 1, 40, 2, 1, 5, 129, 1, 77])
    for members, tokens in (([1, 2, 3, 4], 192), ([6, 7], 200)):
        same_pages(b, members, tokens // page * page)
    b.group_start, b.shared = np.asarray([1, 1, 5, 6, 8], np.int32), np.asarray([64, 192, 64, 200 // page * page], np.int32)
    widen(b, heavy)
    check(K, b)


@HEAVY
def test_more_queries_than_tokens_and_slots_outside(K, heavy):
    """A member that has nothing before its first query, or no slot, leaves nothing to share."""
    b = widen(Batch(54, "bf16", 64, 2, 4, 16, [100, 30, 140], [1, 40, 2], shared=[(3, 16)]), heavy)
    check(K, b)
    b = widen(Batch(55, "bf16", 64, 2, 4, 16, [100, 130, 140, 150], [1, 4, 2, 1], shared=[(4, 80)]), heavy)
    b.slot[1] = -1
    check(K, b)
    b.slot[1] = b.n_slots
    check(K, b)


@HEAVY
@pytest.mark.parametrize("out", [[0], [2], [0, 1, 5], [0, 1, 2, 3, 4]])
def test_members_without_slots_leave_the_rest_sharing(K, heavy, out):
    """Requests that found no room have no slot: they see nothing, and the others share all the same."""
    b = widen(Batch(59, "bf16", 128, 2, 4, 16, [250, 233, 264, 300, 270, 241], [1, 2, 1, 30, 1, 1],
                    shared=[(6, 224)]), heavy)
    b.slot[out] = [-1, b.n_slots, -7, 2 ** 31 - 1, -2 ** 31][:len(out)]
    check(K, b)
    _, plan, _ = plans(K, b)
    tiles = int(plan.buf[:8].view(torch.int64))  # a plan begins with the shared phase's tiles
    assert (tiles > 0) == (len(out) < 5)


@HEAVY
def test_many_members(K, heavy):
    """More rows than a tile in one group."""
    n = 150
    b = widen(Batch(56, "bf16", 128, 2, 4, 16, [201 + i % 70 for i in range(n)], [1] * n, shared=[(n, 200)]), heavy)
    check(K, b)


@HEAVY
def test_holes_in_shared_pages(K, heavy):
    b = widen(Batch(57, "f16", 64, 2, 4, 16, [210, 220, 230], [1, 1, 2], shared=[(3, 208)]), heavy)
    for s in b.slot:
        b.table[s, 4:6] = -1
    check(K, b)
    for s in b.slot:
        b.table[s, :13] = 10 ** 6  # every shared page
    check(K, b)


@HEAVY
def test_other_stream_and_graph(K, heavy):
    """On a stream of its own, and captured: replays with new queries and keys give what the eager call gives."""
    b = widen(Batch(58, "bf16", 128, 2, 4, 16, [700, 300, 290, 90], [1, 7, 2, 1], shared=[(3, 256), (1, 0)]), heavy)
    c, plan, _ = plans(K, b)
    want = K.attention(b.q, c, 0, plan)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = K.attention(b.q, c, 0, plan, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    ws, out, lse = K.Workspace(), torch.empty_like(want[0]), torch.empty_like(want[1])
    ws.get(plan.ws_bytes)
    q = b.q.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K.attention(q, c, 0, plan, out=out, lse=lse, ws=ws)
    for i in range(4):
        q.copy_(torch.randn_like(q))
        b.data.mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip((out, lse), K.attention(q, c, 0, plan)):
            assert torch.equal(x, y)
        torch.ones(1 << 20, device="cuda").sum().item()


def test_an_oracle_that_sees_too_much_is_told_apart(K):
    """The definition with one more shared page than the rows share differs by more than the bounds."""
    b = widen(Batch(51, "bf16", 128, 2, 4, 16, [340, 333, 364], [2, 33, 1], shared=[(3, 288)]))
    c, plan, _ = plans(K, b)
    out, lse = K.attention(b.q, c, 0, plan)
    b.table[b.slot[1], 18] = b.table[b.slot[0], 18]
    with pytest.raises(AssertionError):
        b.compare(out, lse, b.reference(b.D ** -0.5))
