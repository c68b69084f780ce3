"""Attention over the paged cache: shared prefixes, sliding windows with sinks,
ragged batches, against the definition in 64 bits."""
import math
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import kv_ref  # noqa: E402

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import kv
    return kv


def ints(v):
    return torch.tensor(np.asarray(v, np.int32).reshape(np.shape(v)), device="cuda")


class Batch:
    """Sequences in a pool of scattered pages.  lengths and q: tokens and query tokens of each; shared: {group: (members,
    tokens)} in order, the group's pages named by every member's row."""

    def __init__(self, seed, dtype, D, kv_heads, group, page, lengths, q, shared=(), order="head", fused=False,
                 slots=None, spread=1.0, extra=3):
        rng = np.random.default_rng(seed)
        self.rng, self.D, self.page, self.dtype = rng, D, page, dtype
        self.torch_dtype = torch.bfloat16 if dtype == "bf16" else torch.float16
        n, self.Hk, self.Hq = len(lengths), kv_heads, kv_heads * group
        width = max(1, max(-(-x // page) for x in lengths)) + 1
        members, first = [], 0
        for m, t in shared:
            members.append((first, first + m, t))
            first += m
        need = sum(-(-x // page) for x in lengths)
        self.n_slots = slots or n + 2
        pages = need + extra
        at = list(rng.permutation(pages))
        self.slot = rng.permutation(self.n_slots)[:n].astype(np.int32)
        self.table = np.full((self.n_slots, width), -1, np.int32)
        self.length = np.zeros(self.n_slots, np.int32)
        for i, x in enumerate(lengths):
            s = self.slot[i]
            self.length[s] = x
            for j in range(-(-x // page)):
                self.table[s, j] = at.pop()
        for a, b, t in members:  # whole pages of the shared tokens are the first member's
            for i in range(a + 1, b):
                self.table[self.slot[i], :t // page] = self.table[self.slot[a], :t // page]
        self.group_start = np.asarray([0] + [b for _, b, _ in members], np.int32)
        self.shared = np.asarray([t for _, _, t in members], np.int32)
        self.refs = np.bincount(self.table[self.table >= 0], minlength=pages).astype(np.int32)
        self.q_start = np.concatenate([[0], np.cumsum(q)]).astype(np.int32)
        self.total, self.max_q = int(self.q_start[-1]), max(1, max(q))
        shape = (1, 2, pages, kv_heads, page, D)
        x = torch.tensor(rng.standard_normal(shape) * spread, dtype=self.torch_dtype)
        if order == "token":  # the block lies as [page_size][kv_heads][head_dim]
            x = x.transpose(3, 4).contiguous().cuda().transpose(3, 4)
            self.data = x
        else:
            self.data = x.cuda()
        wide = self.Hq + (2 * kv_heads if fused else 0)
        q_all = torch.tensor(rng.standard_normal((max(1, self.total), wide, D)), dtype=self.torch_dtype).cuda()
        self.q = q_all[:self.total, :self.Hq]
        # partial pages of a shared prefix hold the same tokens
        for a, b, t in members:
            rest, w = t % page, t // page
            for i in range(a + 1, b):
                if rest:
                    self.data[:, :, self.table[self.slot[i], w], :, :rest] = \
                        self.data[:, :, self.table[self.slot[a], w], :, :rest]

    def cache(self, K):
        return K.PagedCache.of(self.data, ints(self.refs), ints(self.table), ints(self.length))

    def reference(self, scale, window=0, sinks=0):
        d = self.data.cpu().double().numpy()[0]
        return kv_ref.attention(self.q.cpu().double().numpy(), d, self.table, self.length, self.slot, self.q_start,
                                self.page, scale, window, sinks)

    def run(self, K, scale=None, window=0, sinks=0, groups=True, max_q=None):
        c = self.cache(K)
        kw = dict(total_q=self.total, max_q=max_q or self.max_q, q_heads=self.Hq)
        if window:
            plan = K.window_plan(c, ints(self.slot), ints(self.q_start), window, sinks, **kw)
        elif groups and self.shared.size:
            plan = K.prefix_plan(c, ints(self.slot), ints(self.q_start), ints(self.group_start), ints(self.shared), **kw)
        else:
            plan = K.prefix_plan(c, ints(self.slot), ints(self.q_start), None, None, **kw)
        return K.attention(self.q, c, 0, plan, scale=scale)

    def check(self, K, scale=None, window=0, sinks=0, finite=True, **kw):
        out, lse = self.run(K, scale, window, sinks, **kw)
        ref = self.reference(self.D ** -0.5 if scale is None else scale, window, sinks)
        return self.compare(out, lse, ref)

    def compare(self, out, lse, ref):
        out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
        vmax = float(torch.nan_to_num(self.data[0, 1].float(), 0, 0, 0).abs().max())
        b_out, b_lse = kv_ref.bounds(*ref, UNIT[self.dtype], max(1, int(self.length.max())), vmax, self.D)
        r_out, r_lse = ref[0], ref[1]
        assert np.array_equal(np.isfinite(lse), np.isfinite(r_lse))
        assert np.all(lse[~np.isfinite(r_lse)] == -math.inf)
        fine = np.isfinite(r_lse)
        worst = np.max(np.abs(lse[fine] - r_lse[fine]) - b_lse[fine]) if fine.any() else -1
        assert worst <= 0, f"lse over its bound by {worst}"
        assert np.all(np.isfinite(out)) and np.all(out[~fine] == 0)
        worst = np.max(np.abs(out - r_out) - b_out) if out.size else -1
        assert worst <= 0, f"out over its bound by {worst}"


EDGE = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 257, 400]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("group", [1, 3, 4, 8])
def test_decode_lengths(K, dtype, D, group):
    """One query token a sequence, lengths around every tile's edge, an empty one among them."""
    Batch(1, dtype, D, 2, group, 16, EDGE, [1] * len(EDGE)).check(K)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D,group", [(64, 1), (64, 8), (128, 3), (128, 4)])
def test_decode_lengths_cut(K, dtype, D, group):
    """Single tokens where a row could be long: units are cut over the chip, whatever the lengths are."""
    b = Batch(37, dtype, D, 2, group, 16, EDGE + [2000], [1] * (len(EDGE) + 1))
    b.table = np.pad(b.table, ((0, 0), (0, 4000)), constant_values=-1)
    b.check(K)
    b.check(K, window=3000, sinks=3)
    b.check(K, window=150, sinks=20)


@pytest.mark.parametrize("dtype,D,page,order", [("bf16", 128, 16, "token"), ("f16", 64, 1, "head"), ("bf16", 64, 8, "head"),
                                                ("f16", 128, 64, "token"), ("bf16", 128, 256, "head"),
                                                ("f16", 64, 2, "token")])
def test_page_sizes_and_orders(K, dtype, D, page, order):
    lengths = [1, 7, 100, 130, 259]
    Batch(2, dtype, D, 3, 2, page, lengths, [1, 3, 1, 5, 2], order=order, fused=True).check(K)


@pytest.mark.parametrize("dtype,D,group", [("bf16", 128, 1), ("f16", 64, 5), ("bf16", 64, 7), ("f16", 128, 2)])
@pytest.mark.parametrize("q", ["all", "some"])
def test_prefill(K, dtype, D, group, q):
    """Whole prompts, and chunks of prompts behind earlier tokens; sequences without query tokens among them."""
    lengths = [1, 5, 64, 65, 130, 200, 0, 33]
    n = lengths if q == "all" else [1, 0, 3, 40, 65, 129, 0, 33]
    Batch(3, dtype, D, 2, group, 16, lengths, n).check(K)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 4), (16, 16), (64, 4), (63, 0), (65, 70), (100, 4),
                                          (128, 1), (1000, 4), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("q", ["one", "all"])
def test_window(K, dtype, D, window, sinks, q):
    lengths = [0, 1, 4, 5, 6, 63, 64, 65, 66, 130, 200, 300]
    Batch(4, dtype, D, 2, 4, 16, lengths, [1] * len(lengths) if q == "one" else lengths).check(
        K, window=window, sinks=sinks)


@pytest.mark.parametrize("dtype,D,group", [("bf16", 128, 4), ("f16", 64, 5), ("f16", 128, 1)])
@pytest.mark.parametrize("shared", [1, 15, 16, 64, 65, 130, 300])
def test_shared_prefix(K, dtype, D, group, shared):
    """Two groups and members without own tokens before their queries."""
    own, q = [1, 1, 3, 40, 70, 5, 1, 130], [1, 1, 3, 2, 1, 5, 1, 4]
    lengths = [shared + x for x in own[:5]] + [20 + x for x in own[5:]]
    Batch(5, dtype, D, 2, group, 16, lengths, q, shared=[(5, shared), (3, 20)]).check(K)


def test_shared_beyond_a_member(K):
    """shared reaches past a member's first query, and to a group of one, an empty group and a group with an empty member:
    the tokens that not every member has before its queries count as its own."""
    b = Batch(6, "bf16", 128, 2, 4, 16, [40, 33, 64, 90, 100], [2, 3, 1, 1, 4], shared=[(3, 32), (1, 80), (1, 96)])
    b.check(K)
    b.shared[:] = [1000, 2 ** 31 - 1, -5]
    for i in (1, 2):  # more than the rows share: the members' pages have to agree as far as it counts (30 tokens)
        b.table[b.slot[i], :2] = b.table[b.slot[0], :2]
    b.check(K)
    b = Batch(7, "f16", 64, 1, 8, 16, [0, 50, 60], [0, 1, 1], shared=[(3, 48)])
    for i in (1, 2):
        b.table[b.slot[i], :3] = np.arange(3)
    b.group_start, b.shared = np.asarray([0, 0, 3, 3], np.int32), np.asarray([48, 48, 48], np.int32)
    b.check(K)


def test_many_members_share(K):
    """More rows than a tile in one group, and the same batch without the plan's knowledge of the prefix."""
    n = 150
    lengths = [200 + 1 + i % 70 for i in range(n)]
    b = Batch(8, "bf16", 128, 2, 4, 16, lengths, [1] * n, shared=[(n, 200)])
    b.check(K)
    b.check(K, groups=False)

def widen(b, heavy=False):
    """A table so wide that shared prefixes count; heavy: that their phase takes kernels of its own."""
    keys = (256 << 20) // (4 * len(b.slot) * b.Hk * b.D) + 1
    if heavy:
        keys = max(keys, int(100e9 / (4 * b.total * b.Hq * b.D)) + 1)
    b.table = np.pad(b.table, ((0, 0), (0, -(-keys // b.page))), constant_values=-1)
    return b


@pytest.mark.parametrize("heavy", [False, True])
@pytest.mark.parametrize("dtype,D,group", [("bf16", 128, 4), ("f16", 64, 5), ("f16", 128, 1), ("bf16", 64, 16)])
@pytest.mark.parametrize("shared", [16, 47, 64, 130, 300])
@pytest.mark.parametrize("q", ["one", "few", "many"])
def test_shared_phase(K, heavy, dtype, D, group, shared, q):
    """The shared keys as a phase of their own: tiles of 32, 128 and 256 rows there and in the sequences' own keys, the
    phases in one kernel and in two."""
    n = {"one": [1] * 9, "few": [1, 1, 3, 2, 1, 7, 1, 4, 0], "many": [1, 60, 3, 200, 1, 5, 1, 40, 130]}[q]
    own = [x + (7 * i) % 90 for i, x in enumerate(n)]
    lengths = [shared + x for x in own[:5]] + [33 + x for x in own[5:]]
    widen(Batch(31, dtype, D, 2, group, 16, lengths, n, shared=[(5, shared), (4, 33)]), heavy).check(K)


@pytest.mark.parametrize("heavy", [False, True])
@pytest.mark.parametrize("page", [1, 8, 64])
def test_shared_phase_pages(K, heavy, page):
    own = [1 + (11 * i) % 70 for i in range(40)]
    b = Batch(32, "bf16", 128, 2, 4, page, [210 + x for x in own], [1] * 40, shared=[(17, 192), (23, 210)], order="token")
    widen(b, heavy).check(K)
    b.table[b.table == b.table[b.slot[20], 1]] = -1  # a page that a group shared
    b.check(K)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("heavy", [False, True])
def test_shared_phase_hidden_values(K, value, heavy):
    """Keys and values that are not finite behind each sequence's end, and in values that only the later of a sequence's
    query tokens sees."""
    n = [1, 2, 1, 40]
    lengths = [140 + x + (13 * i) % 50 for i, x in enumerate(n)]
    b = widen(Batch(33, "f16", 64, 2, 4, 16, lengths, n, shared=[(4, 140)]), heavy)
    for s, x in zip(b.slot, lengths):
        if x % 16:
            b.data[:, :, b.table[s, x // 16], :, x % 16:] = value
    b.check(K)
    s, x = b.slot[1], lengths[1]
    b.data[:, 1, b.table[s, (x - 1) // 16], :, (x - 1) % 16] = value
    out, lse = b.run(K)
    last = int(b.q_start[2]) - 1
    ref = b.reference(b.D ** -0.5)
    keep = [i for i in range(b.total) if i != last]
    assert not torch.isfinite(out[last]).any()
    b.compare(out[keep], lse[keep], [r[keep] for r in ref])


def test_shared_phase_same_bits(K):
    b = widen(Batch(34, "bf16", 128, 2, 4, 16, [3000, 1200, 1140, 1130], [1, 5, 40, 1], shared=[(4, 1100)]))
    first = b.run(K)
    for _ in range(3):
        for x, y in zip(first, b.run(K)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("scale", [1e-6, 0.5, 3.0])
def test_scale(K, scale):
    """Flat and peaked weights."""
    Batch(9, "bf16", 128, 2, 4, 16, [1, 70, 300], [1, 2, 30]).check(K, scale=scale)
    Batch(9, "f16", 64, 2, 4, 16, [1, 70, 300], [1, 2, 30]).check(K, scale=scale, window=50, sinks=3)


@pytest.mark.parametrize("window", [0, 100])
def test_large_scores(K, window):
    """Scores of a few thousand: one weight is 1, the rest 0, however the keys are cut."""
    Batch(10, "bf16", 128, 2, 4, 16, [1, 70, 700], [1, 1, 3], spread=60.0).check(K, window=window, sinks=0)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("D,dtype", [(64, "f16"), (128, "bf16")])
def test_hidden_values(K, value, D, dtype):
    """Whatever lies where no query looks (pages of nobody, the rest of a last page, tokens outside the window, tokens
    that come after a query) leaves the results as they are."""
    b = Batch(11, dtype, D, 2, 4, 16, [5, 100, 131, 200], [1, 1, 3, 1])
    seen = np.zeros((b.refs.size, 16), bool)
    for s in b.slot:
        for j in range(b.length[s]):
            seen[b.table[s, j // 16], j % 16] = True
    hide = torch.tensor(~seen, device="cuda")
    clean = b.run(K)
    b.data.permute(0, 1, 2, 4, 3, 5)[:, :, hide] = value
    for x, y in zip(clean, b.run(K)):
        assert torch.equal(x, y)
    b = Batch(12, dtype, D, 2, 4, 16, [90, 170, 260], [1, 2, 1])
    clean = b.run(K, window=40, sinks=5)
    for i, q in enumerate([1, 2, 1]):
        s = b.slot[i]
        for j in range(5, b.length[s] - q + 1 - 40):
            b.data[:, :, b.table[s, j // 16], :, j % 16] = value
    for x, y in zip(clean, b.run(K, window=40, sinks=5)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("D,dtype", [(64, "f16"), (128, "bf16")])
@pytest.mark.parametrize("window,n", [(0, 40), (0, 300), (70, 300)])
def test_values_some_rows_see(K, value, D, dtype, window, n):
    """A key and a value that are not finite reach the queries that see them and no other."""
    b = Batch(13, dtype, D, 2, 2, 16, [n], [n])
    s, bad = b.slot[0], n // 2 + 3
    far = n if not window else min(n, bad + window)
    clean = b.run(K, window=window)
    ref = b.reference(D ** -0.5, window)
    other = np.r_[0:bad, far:n]
    for plane in (0, 1):
        kept = b.data.clone()
        b.data[0, plane, b.table[s, bad // 16], 1, bad % 16, 5] = value
        out, lse = b.run(K, window=window)
        b.data.copy_(kept)
        b.compare(out[other], lse[other], [x[other] for x in ref])
        b.compare(out[:, :2], lse[:, :2], [x[:, :2] for x in ref])  # the other key head's queries
        if plane == 1:
            assert not torch.isfinite(out[bad:far, 2:, 5]).any()
            assert torch.isfinite(out[bad:far, 2:, 6:]).all()
            assert torch.equal(lse, clean[1])
        elif math.isnan(value):
            assert torch.isnan(out[bad:far, 2:]).all() and torch.isnan(lse[bad:far, 2:]).all()


def test_holes(K):
    """Entries outside the pool hide their tokens; a row with nothing visible gives 0 and -inf."""
    b = Batch(14, "bf16", 128, 2, 4, 16, [40, 100, 200, 64], [1, 2, 1, 64])
    b.table[b.slot[0], :] = -1
    b.table[b.slot[1], 2] = -7
    b.table[b.slot[2], 3:9] = 10 ** 6
    b.table[b.slot[3], 0] = -1
    b.check(K)
    b.check(K, window=50, sinks=8)
    b = Batch(15, "f16", 64, 2, 4, 16, [210, 220, 230], [1, 1, 2], shared=[(3, 208)])
    for s in b.slot:
        b.table[s, 4:6] = -1
    b.check(K)


def test_slots_outside(K):
    b = Batch(16, "bf16", 64, 2, 4, 16, [40, 100, 70], [1, 2, 1])
    b.slot[1] = -1
    b.check(K)
    b.slot[1] = b.n_slots
    b.check(K, window=30, sinks=2)


def test_queries_before_the_first_token(K):
    """More query tokens than the slot holds: the first see nothing."""
    b = Batch(17, "bf16", 128, 2, 2, 16, [3, 60], [10, 70])
    b.check(K)
    b.check(K, window=20, sinks=2)


def test_max_q_only_chooses(K):
    b = Batch(18, "f16", 128, 2, 4, 16, [300, 40, 7], [100, 1, 7])
    for most in (1, 8, 100, 2 ** 31 - 1):
        b.check(K, max_q=most)


def test_long_keys_are_split(K):
    """One sequence of thousands of tokens: the key axis is cut over the chip and joined."""
    b = Batch(19, "bf16", 128, 1, 4, 16, [9001], [1])
    b.check(K)
    b.check(K, window=8000, sinks=64)
    Batch(20, "f16", 64, 1, 40, 16, [5003, 4000], [2, 1]).check(K)


@pytest.mark.parametrize("kind", ["prefix", "window"])
def test_cut_and_join_over_a_large_batch(K, kind):
    """Rows and splits of a full chip, a ninth of the queries checked."""
    n = 96
    lengths = [1 + (i * 37) % 900 + (600 if kind == "prefix" else 0) for i in range(n)]
    b = Batch(21, "bf16", 128, 4, 4, 16, lengths, [1] * n, shared=[(n, 600)] if kind == "prefix" else ())
    out, lse = b.run(K, window=300 if kind == "window" else 0, sinks=4 if kind == "window" else 0)
    pick = list(range(0, n, 11))
    d = b.data.cpu().double().numpy()[0]
    q = b.q.cpu().double().numpy()
    ref = kv_ref.attention(q[pick], d, b.table, b.length, b.slot[pick], np.arange(len(pick) + 1), 16, b.D ** -0.5,
                           300 if kind == "window" else 0, 4 if kind == "window" else 0)
    b.compare(out[pick], lse[pick], ref)


def test_same_bits_every_time(K):
    b = Batch(22, "bf16", 128, 2, 4, 16, [3000, 1200, 40], [1, 5, 40], shared=[(2, 1100), (1, 0)])
    first = b.run(K)
    for _ in range(3):
        for x, y in zip(first, b.run(K)):
            assert torch.equal(x, y)


def test_other_stream_and_graph(K):
    """On a stream of its own, and captured: replays with new queries and new keys give what the eager call gives."""
    b = Batch(23, "bf16", 128, 2, 4, 16, [700, 300, 90], [1, 1, 1], shared=[(2, 256), (1, 0)])
    c = b.cache(K)
    args = [ints(x) for x in (b.slot, b.q_start, b.group_start, b.shared)]
    plan = K.prefix_plan(c, *args, total_q=b.total, max_q=1, q_heads=b.Hq)
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


def test_refusals(K):
    b = Batch(24, "bf16", 64, 2, 4, 16, [40, 30], [1, 1])
    c = b.cache(K)
    sl, qs = ints(b.slot), ints(b.q_start)
    kw = dict(total_q=2, max_q=1, q_heads=8)
    with pytest.raises(ValueError):
        K.window_plan(c, sl, qs, 0, 4, **kw)             # a window of nothing
    with pytest.raises(ValueError):
        K.window_plan(c, sl, qs, 8, -1, **kw)
    with pytest.raises(ValueError):
        K.window_plan(c, sl, qs, 8, 1, total_q=2, max_q=0, q_heads=8)
    with pytest.raises(ValueError):
        K.prefix_plan(c, sl, qs, None, None, total_q=2, max_q=1, q_heads=9)
    with pytest.raises(ValueError):
        K.prefix_plan(c, sl, ints([0, 1]), None, None, **kw)
    plan = K.prefix_plan(c, sl, qs, None, None, **kw)
    with pytest.raises(TypeError):
        K.attention(b.q.half(), c, 0, plan)
    with pytest.raises(TypeError):
        K.attention(b.q[:1], c, 0, plan)
    with pytest.raises(K.L.EwsjfError):
        K.attention(b.q, c, 1, plan)                     # no such layer
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(K.L.EwsjfError):
            K.attention(b.q, c, 0, plan, scale=scale)
    odd = torch.zeros((2, 8, 65), dtype=torch.bfloat16, device="cuda")[:, :, :64]
    with pytest.raises(K.L.EwsjfError):
        K.attention(odd, c, 0, plan)                     # strides that 16 bytes do not divide
    with pytest.raises(TypeError):
        K.PagedCache.of(b.data.float(), c.refs, c.table, c.length)
    with pytest.raises(ValueError):
        K.PagedCache.of(b.data[:, :, :, :, :15], c.refs, c.table, c.length)  # a page of 15 tokens


def test_empty_batches(K):
    b = Batch(25, "bf16", 64, 2, 4, 16, [40, 30], [0, 0])
    out, lse = b.run(K)
    assert out.shape == (0, 8, 64) and lse.shape == (0, 8)
    c = b.cache(K)
    plan = K.window_plan(c, ints(np.zeros(0)), ints([0]), 5, 1, total_q=0, max_q=1, q_heads=8)
    out, lse = K.attention(b.q, c, 0, plan)
    assert out.numel() == 0


def test_starts_out_of_order(K):
    """Starts that fall back or leave the batch count as the largest before them, within the batch."""
    b = widen(Batch(35, "bf16", 64, 2, 4, 16, [60 + 3 * i for i in range(12)], [2] * 12, shared=[(5, 48), (4, 32), (3, 32)]))
    rng = np.random.default_rng(36)
    c = b.cache(K)
    for _ in range(8):
        q = rng.integers(-3, b.total + 30, 13).astype(np.int32)
        g = rng.integers(-2, 15, 4).astype(np.int32)
        kw = dict(total_q=b.total, max_q=2, q_heads=b.Hq)
        got = []
        for qs, gs in ((q, g), (np.maximum.accumulate(q.clip(0, b.total)), np.maximum.accumulate(g.clip(0, 12)))):
            for plan in (K.prefix_plan(c, ints(b.slot), ints(qs), ints(gs), ints(b.shared), **kw),
                         K.window_plan(c, ints(b.slot), ints(qs), 20, 2, **kw)):
                out, lse = torch.zeros_like(b.q).contiguous(), torch.zeros(b.q.shape[:2], device="cuda")
                got.append(K.attention(b.q, c, 0, plan, out=out, lse=lse))
        for i in (0, 1):
            for x, y in zip(got[i], got[i + 2]):
                assert torch.equal(x, y)


@pytest.mark.parametrize("q", [1, 70])
def test_offsets_past_32_bits(K, q):
    """Pages whose keys lie more than 2^32 bytes, and more than 2^31 elements, behind the first one's."""
    pages, page, heads, D = 2500, 1024, 8, 128
    data = torch.empty((1, 2, pages, heads, page, D), dtype=torch.bfloat16, device="cuda")
    used = np.asarray([2499, 3, 2100])
    rng = np.random.default_rng(38)
    small = torch.tensor(rng.standard_normal((1, 2, 3, heads, page, D)), dtype=torch.bfloat16)
    for i, p in enumerate(used):
        data[:, :, p] = small[:, :, i].cuda()
    table, length = np.asarray([[0, 1, 2], [2, 0, -1]]), np.asarray([2300, 1500])
    q_start = np.asarray([0, q, q + 1])
    x = torch.tensor(rng.standard_normal((q + 1, 2 * heads, D)), dtype=torch.bfloat16)
    refs = np.zeros(pages, np.int32)
    refs[used] = [2, 1, 2]
    cache = K.PagedCache.of(data, ints(refs), ints(np.where(table < 0, -1, used[table])), ints(length))
    pick = [0, q - 1, q]
    for window, sinks in ((0, 0), (700, 5)):
        kw = dict(total_q=q + 1, max_q=q, q_heads=2 * heads)
        plan = K.window_plan(cache, ints([0, 1]), ints(q_start), window, sinks, **kw) if window else \
            K.prefix_plan(cache, ints([0, 1]), ints(q_start), None, None, **kw)
        out, lse = K.attention(x.cuda(), cache, 0, plan)
        ref = kv_ref.attention(x.double().numpy(), small.double().numpy()[0], table, length, [0, 1], q_start, page,
                               D ** -0.5, window, sinks)
        b_out, b_lse = kv_ref.bounds(*ref, UNIT["bf16"], 2300, float(small.float().abs().max()), D)
        assert np.all(np.abs(out.cpu().double().numpy() - ref[0])[pick] <= b_out[pick])
        assert np.all(np.abs(lse.cpu().double().numpy() - ref[1])[pick] <= b_lse[pick])
    # new tokens and a fork's copy there too
    k, v = (torch.randn((1, heads, D), device="cuda").bfloat16() for _ in range(2))
    cache.append(0, k, v, ints([1]), ints([0, 1]))
    assert torch.equal(data[0, 0, used[0], :, 1499 % page], k[0]) and torch.equal(data[0, 1, used[0], :, 1499 % page], v[0])
    cache.copy(ints([2499]), ints([2400]))
    assert torch.equal(data[:, :, 2400], data[:, :, 2499])


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 200, 2 ** 30])
@pytest.mark.parametrize("sinks", [0, 3])
def test_windows_longer_than_any_row(K, window, sinks):
    n = [300, 70, 33, 1]
    b = Batch(39, "f16", 64, 2, 4, 16, [300, 90, 20, 200], n)
    b.length = b.length.astype(np.int64)  # the definition's p - window, without a wrap of its own
    b.check(K, window=window, sinks=sinks)
