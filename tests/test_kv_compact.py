"""Contents of the pages that a compaction moves, in pools that one workgroup
ranks and in pools that many do."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_kv_cache import ints, make, same  # noqa: E402

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import kv
    return kv


@pytest.mark.parametrize("pages,page,order", [(1023, 4, "head"), (1024, 4, "token"), (1025, 2, "head"), (4097, 2, "token"),
                                              (70001, 1, "head"), (70001, 2, "token")])
@pytest.mark.parametrize("in_place", [False, True])
def test_moved_contents(K, pages, page, order, in_place):
    """Random fills, releases and forks; the reference moves its pages by itself."""
    slots, width = 9, pages // 4
    c, r = make(K, pages, page, slots, width, layers=2, heads=1, order=order, seed=pages)
    rng = np.random.default_rng(page)
    moved = 0
    for step in range(4):
        pick = rng.permutation(slots)
        t = rng.integers(0, width * page // 2, slots)
        assert c.extend(ints(pick), ints(t)).tolist() == r.extend(pick, t)
        c.release(ints(pick[4:])), r.release(pick[4:])
        half = r.length[pick[0]] // 2 | 1
        assert c.fork(ints(pick[:1]), ints(pick[5:6]), ints([half])).tolist() == r.fork(pick[:1], pick[5:6], [half])
        same(c, r)
        before = r.data.copy()
        out = c.compact(out=(c.table, c.refs, torch.empty(1, dtype=torch.int32, device="cuda")) if in_place else None)
        table, refs, used = r.compact()
        moved += int((before != r.data).any(axis=(0, 1, 3, 4, 5)).sum())
        assert np.array_equal(out[0].cpu().numpy(), table) and np.array_equal(out[1].cpu().numpy(), refs)
        assert int(out[2]) == used
        if not in_place:
            c.adopt(*out[:2])
        r.table, r.refs = table, refs
        same(c, r)
    assert moved > 100
