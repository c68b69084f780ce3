"""Softmax sums over very many keys: shared prefixes of more than 2^30 tokens."""
import math
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


@pytest.mark.parametrize("q", [1, 20])
def test_a_prefix_of_more_than_2_30_tokens(K, q):
    """2^30 tokens of weight 1 and value 0 (one page, named again and again), then 4096 shared ones of weight e^20 and
    value 1, then each member's own of weight 1 and value -1.  20 query tokens: tiles of 256 rows."""
    page, dull, D, G = 1024, 1 << 20, 64, 4
    own = q + 3
    data = torch.zeros((1, 2, 3, 1, page, D), dtype=torch.float16, device="cuda")
    data[0, 0, 1, 0, :, 0], data[0, 1, 1] = 20.0, 1.0
    data[0, 1, 2] = -1.0
    row = np.concatenate([np.zeros(dull), np.ones(4), [2, -1]])
    length = (dull + 4) * page + own
    cache = K.PagedCache.of(data, ints([2 * dull, 8, 2]), ints([row, row]), ints([length, length]))
    x = torch.zeros((2 * q, G, D), dtype=torch.float16, device="cuda")
    x[..., 0] = 1.0
    plan = K.prefix_plan(cache, ints([0, 1]), ints([0, q, 2 * q]), ints([0, 2]), ints([length - own]), total_q=2 * q,
                         max_q=q, q_heads=G)
    alone = K.prefix_plan(cache, ints([0, 1]), ints([0, q, 2 * q]), None, None, total_q=2 * q, max_q=q, q_heads=G)
    assert plan.ws_bytes > alone.ws_bytes  # the shared keys are a phase of their own
    out, lse = K.attention(x, cache, 0, plan, scale=1.0)
    seen = np.tile(np.arange(own - q + 1, own + 1), 2)[:, None]
    heavy = 4096 * math.exp(20)
    total = dull * page + heavy + seen
    want, want_lse = (heavy - seen) / total, np.log(total)
    # a binary32 sum of 2^30 terms of the light keys, at most all of them lost; a score's rounding 8 * 21 * 2^-24
    light = dull * page / heavy
    bound = light + 2.0 ** -11 + 2 * 8 * 21 * 2.0 ** -24
    assert np.all(np.abs(out.cpu().double().numpy() - want[..., None]) <= bound)
    assert np.all(np.abs(lse.cpu().double().numpy() - want_lse) <= light + 2.0 ** -18)
