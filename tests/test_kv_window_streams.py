"""Plans of windows on another stream than the current one: the cache is kept for it."""
import os
import sys

import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_a_cache_is_kept_for_the_stream_that_plans_a_window():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import kv
    from test_kv_streams import Busy, Case, taken_again
    case = Case(kv, pages=4000, slots=20000)
    torch.cuda.synchronize()
    busy = Busy()
    plan = kv.window_plan(case.cache, case.slot, case.q_start, 100, 4, total_q=case.n, max_q=case.n, q_heads=8,
                          stream=busy.stream)
    assert case.cache.used_on == busy.stream.cuda_stream
    size, ptr = case.cache.table.numel() * 4, case.cache.table.data_ptr()
    table, refs = case.cache.table.clone(), case.cache.refs.clone()
    case.cache.adopt(table, refs)
    again = taken_again(size, ptr)
    busy.later()
    torch.cuda.synchronize()
    assert not again
    del plan
