"""Softmax sums over very many keys: shared prefixes of more than 2^30 tokens,
and many light keys behind a heavy one in float16."""
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


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("q", [1, 9, 300])
@pytest.mark.parametrize("n,drop", [(32768, 19.0), (5000, 17.0), (1700, 16.0), (131072, 20.0)])
@pytest.mark.parametrize("window", [False, True])
def test_many_light_keys_behind_a_heavy_one(K, D, q, n, drop, window):
    """float16: one key of score `drop` and value 0, the others of score 0 and value 1, whose weights lie 2^-23 to 2^-29
    below the first one's.  Such a weight is rounded to a multiple of 2^-24 of the 2^8 that the largest one is held as, so
    it is off by at most 2^-33; the sum of the light ones by n times that."""
    page = 16
    data = torch.zeros((1, 2, 2, 1, page, D), dtype=torch.float16, device="cuda")
    data[0, 0, 0, 0, 0, 0], data[0, 1, 0, 0, 1:], data[0, 1, 1] = drop, 1.0, 1.0
    row = np.ones(n // page + 2)
    row[0] = 0
    cache = K.PagedCache.of(data, ints([1, n // page + 1]), ints([row]), ints([n]))
    x = torch.zeros((q, 2, D), dtype=torch.float16, device="cuda")
    x[..., 0] = 1.0
    kw = dict(total_q=q, max_q=q, q_heads=2)
    w = n // 2 if window else n
    plan = K.window_plan(cache, ints([0]), ints([0, q]), w, 1, **kw) if window else \
        K.prefix_plan(cache, ints([0]), ints([0, q]), None, None, **kw)
    out, lse = K.attention(x, cache, 0, plan, scale=1.0)
    p = np.arange(n - q, n)
    light = np.minimum(p, w) * math.exp(-drop)
    want = (light / (1 + light))[:, None, None]
    score = 8 * (1 + drop) * 2.0 ** -24
    bound = n * 2.0 ** -33 + want * (2.0 ** -11 + 2 * score + 2.0 ** -16) + 2.0 ** -25
    assert np.all(bound < want / 8)
    assert np.all(np.abs(out.cpu().double().numpy() - want) <= bound)
    exact = drop + np.log1p(light)
    assert np.all(np.abs(lse.cpu().double().numpy() - exact[:, None]) <= score + 2.0 ** -20 * (1 + exact[:, None]))
