"""Memory of calls on another stream than the current one: what a call takes
comes from that stream's memory, and what it reads is not given away while the
stream may still be at it."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

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


class Case:
    """One prompt of 3000 tokens: outputs, plan, workspace and (slots) table of a size of their own."""

    def __init__(self, K, n=3000, pages=200, slots=2):
        self.cache = K.PagedCache.new(1, pages, 16, 2, 64, slots, 200, dtype=torch.float16)
        self.n, self.slot, self.q_start = n, ints([0]), ints([0, n])
        self.cache.extend(self.slot, ints([n]))
        self.q = torch.randn((n, 8, 64), device="cuda").half()
        self.cache.append(0, self.q[:, :2], self.q[:, 2:4], self.slot, self.q_start)

    def plan(self, K, stream=None):
        return K.prefix_plan(self.cache, self.slot, self.q_start, None, None, total_q=self.n, max_q=self.n, q_heads=8,
                             stream=stream)


class Busy:
    """A stream with work of many milliseconds before whatever is asked of it."""

    def __init__(self):
        self.stream = torch.cuda.Stream()
        a = torch.randn((8192, 8192), device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(self.stream):
            for _ in range(6):
                a = a @ a * 1e-4
            self.done = torch.cuda.Event()
            self.done.record()
        self.a = a

    def later(self):
        assert not self.done.query(), "the stream's work ended before the test's"


def taken_again(tensor_bytes, ptr):
    """Whether memory of this size on the current stream is the memory at ptr; nothing is written there."""
    return torch.empty(tensor_bytes, dtype=torch.uint8, device="cuda").data_ptr() == ptr


def test_results_come_from_the_streams_memory(K):
    """Memory that the current stream gave back may still be in use there: a call on another stream takes other memory."""
    case, side = Case(K), torch.cuda.Stream()
    plan = case.plan(K)
    torch.cuda.synchronize()
    shapes = {"out": (case.n * 8 * 64 * 2, lambda: K.attention(case.q, case.cache, 0, plan, stream=side)),
              "plan": (plan.buf.numel(), lambda: case.plan(K, stream=side)),
              "table": (case.cache.table.numel() * 4, lambda: case.cache.compact(stream=side)),
              "scratch": (plan.ws_bytes, lambda: K.attention(case.q, case.cache, 0, plan, stream=side))}
    for name, (size, call) in shapes.items():
        x = torch.empty(size, dtype=torch.uint8, device="cuda")
        ptr = x.data_ptr()
        del x
        kept = call()
        free = taken_again(size, ptr)
        torch.cuda.synchronize()
        assert free, name
        del kept


def test_a_plan_is_kept_for_the_stream_that_reads_it(K):
    case = Case(K)
    plan = case.plan(K)
    torch.cuda.synchronize()
    busy = Busy()
    kept = K.attention(case.q, case.cache, 0, plan, stream=busy.stream)
    size, ptr = plan.buf.numel(), plan.buf.data_ptr()
    del plan
    again = taken_again(size, ptr)
    busy.later()
    torch.cuda.synchronize()
    assert not again
    del kept


def test_a_workspace_that_grows_is_kept_for_the_stream_that_uses_it(K):
    case, ws = Case(K), K.Workspace()
    plan = case.plan(K)
    ws.get(plan.ws_bytes)  # taken on the current stream
    torch.cuda.synchronize()
    busy = Busy()
    kept = K.attention(case.q, case.cache, 0, plan, ws=ws, stream=busy.stream)
    size, ptr = ws.buf.numel(), ws.buf.data_ptr()
    ws.get(2 * size)
    again = taken_again(size, ptr)
    busy.later()
    torch.cuda.synchronize()
    assert not again
    # and one that grew on the other stream, used on the current one
    ws = K.Workspace()
    busy = Busy()
    kept = K.attention(case.q, case.cache, 0, plan, ws=ws, stream=busy.stream)
    torch.cuda.synchronize()
    size, ptr = ws.buf.numel(), ws.buf.data_ptr()
    work = Busy()
    torch.cuda.current_stream().wait_event(work.done)
    kept = K.attention(case.q, case.cache, 0, plan, ws=ws)
    ws.get(2 * size)
    with torch.cuda.stream(busy.stream):
        again = taken_again(size, ptr)
    work.later()
    torch.cuda.synchronize()
    assert not again
    del kept


def test_a_cache_is_kept_for_the_stream_that_reads_it(K):
    case = Case(K, pages=4000, slots=20000)
    plan = case.plan(K)
    torch.cuda.synchronize()
    busy = Busy()
    kept = K.attention(case.q, case.cache, 0, plan, stream=busy.stream)
    size, ptr = case.cache.data.numel() * 2, case.cache.data.data_ptr()
    t_size, t_ptr = case.cache.table.numel() * 4, case.cache.table.data_ptr()
    table, refs = case.cache.table.clone(), case.cache.refs.clone()
    case.cache.adopt(table, refs)
    t_again = taken_again(t_size, t_ptr)
    case.cache = None
    again = taken_again(size, ptr)
    busy.later()
    torch.cuda.synchronize()
    assert not again and not t_again
    del kept


def test_other_streams_give_the_same(K):
    """The same bits on the current stream, on another, and on one after the other."""
    case, side = Case(K), torch.cuda.Stream()
    plan, ws = case.plan(K), K.Workspace()
    want = K.attention(case.q, case.cache, 0, plan)
    for i in range(4):
        side.wait_stream(torch.cuda.current_stream())
        got = K.attention(case.q, case.cache, 0, plan if i % 2 else case.plan(K, stream=side), ws=ws,
                          stream=side)
        torch.cuda.current_stream().wait_stream(side)
        for x, y in zip(got, want):
            assert torch.equal(x, y)
        for x, y in zip(K.attention(case.q, case.cache, 0, plan, ws=ws), want):
            assert torch.equal(x, y)
