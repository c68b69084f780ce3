"""The 8-bit cache: what an append writes, bit for bit, what a read gives back, and
its pages forked, copied and compacted with their scales."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import codes_ref  # noqa: E402
import kv_ref  # noqa: E402

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def K():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import kv
    return kv


def ints(v):
    return torch.tensor(np.asarray(v, np.int32).reshape(np.shape(v)), device="cuda")


def make(K, kind, layers, pages, page, heads, D, slots, width, tokens_first=False, seed=0):
    """A cache whose bytes are random where nothing was written."""
    data = torch.randint(0, 256, (layers, 2, pages, K.page_bytes(page, heads, D)), dtype=torch.uint8,
                         generator=torch.Generator().manual_seed(seed)).cuda()
    return K.PagedCache.of_bytes(data, ints(np.zeros(pages)), ints(np.full((slots, width), -1)), ints(np.zeros(slots)),
                                 page, heads, D, dtype=TYPES[kind], tokens_first=tokens_first)


def bits(t):
    return t.view(torch.uint8).cpu().numpy()


def rows(kind, n, heads, D, seed):
    """Rows as a model's and rows at the format's edges, in the type's precision."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, heads, D)) * np.exp2(rng.integers(-12, 6, (n, heads, 1)))
    x[:, :, ::16] *= 5
    big, tiny = (3.3e38, 1e-39) if kind == "bf16" else (65504.0, 6e-8)
    edge = [[0.0], [448.0, 1.0], [449.0, 1.0], [450.0, 31.0], [-896.0, 17.0, 19.0], [tiny], [big, big / 3, 1.0], [np.inf, 5.0],
            [-np.inf, np.nan, 3.0], [np.nan], [np.nan, 2.0 ** -10, 0.5], [1.0, 2.0 ** -9, 3 * 2.0 ** -10, 2.0 ** -15],
            [tiny * 3, tiny, -tiny * 7], [0.0, -0.0, 1e-30 if kind == "bf16" else 0.0]]
    flat = x.reshape(-1, D)
    for i, e in enumerate(edge):
        if i < len(flat):
            flat[-1 - i] = 0
            flat[-1 - i, (i * 7) % (D - 4):][:len(e)] = e
    return torch.tensor(x).to(TYPES[kind])


def places(c, slot, q_start, granted=None):
    """Where each token belongs: {(page, place): token}."""
    table, length, refs = (t.cpu().numpy() for t in (c.table, c.length, c.refs))
    at = {}
    for b, s in enumerate(slot):
        if not 0 <= s < len(length) or (granted is not None and not granted[b]):
            continue
        for t in range(q_start[b], q_start[b + 1]):
            pos = length[s] - (q_start[b + 1] - t)
            if pos < 0 or not 0 <= table[s, pos // c.page_size] < len(refs):
                continue
            page = table[s, pos // c.page_size]
            if granted is None and pos // c.page_size < length[s] // c.page_size and refs[page] > 1:
                continue
            at[(page, pos % c.page_size)] = t
    return at


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("D,heads,page,tokens_first", [(128, 8, 16, False), (64, 2, 16, True), (64, 3, 1, False),
                                                       (16, 1, 8, False), (48, 5, 4, True), (256, 2, 64, False),
                                                       (80, 3, 32, True)])
def test_append_bits(K, kind, D, heads, page, tokens_first):
    """Codes and scales are the definition's, in their places, and nothing else is touched."""
    lens, new = [5, 40, 1, 17, 64], [5, 33, 1, 0, 7]
    c = make(K, kind, 2, 400 // page + 9, page, heads, D, 7, -(-70 // page) + 1, tokens_first, seed=D)
    slot = [3, 0, 6, 2, 5]
    assert c.extend(ints(slot), ints(lens)).tolist() == [1] * 5
    q_start = np.concatenate([[0], np.cumsum(new)])
    k, v = (rows(kind, int(q_start[-1]), heads, D, s) for s in (1, 2))
    before = c.data.clone()
    c.append(1, k.cuda(), v.cuda(), ints(slot), ints(q_start))
    at = places(c, slot, q_start)
    assert len(at) == q_start[-1]
    codes, scales = bits(c.codes), c.scales.cpu().numpy()
    old = K.PagedCache.of_bytes(before, c.refs, c.table, c.length, page, heads, D, c.dtype, tokens_first)
    want_codes, want_scales = bits(old.codes).copy(), old.scales.cpu().numpy().copy()
    for plane, x in enumerate((k, v)):
        code, scale, _ = codes_ref.quantise(x.double().numpy(), kind)
        for (p, i), t in at.items():
            want_codes[1, plane, p, :, i], want_scales[1, plane, p, :, i] = code[t], scale[t]
    nan = (codes & 127 == 127) & (want_codes & 127 == 127)
    assert np.array_equal(np.where(nan, 0, codes), np.where(nan, 0, want_codes))
    assert np.array_equal(scales, want_scales)
    rest = heads * page * (D + 1)
    assert torch.equal(c.data[..., rest:], before[..., rest:])


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_append_every_magnitude(K, kind):
    """All magnitudes of the type as the largest of a row, with every other beside it some time."""
    D, page = 128, 64
    every = torch.arange(0, 65536, dtype=torch.int32).to(torch.int16).view(TYPES[kind])
    x = every[torch.randperm(65536, generator=torch.Generator().manual_seed(1))].view(-1, 1, D)
    solo = torch.zeros((65536 // 64, 1, D), dtype=TYPES[kind])  # and each alone with its next ones
    solo[:, 0, :64] = every.view(-1, 64)
    x = torch.cat([x, solo])
    n = x.shape[0]
    c = make(K, kind, 1, -(-n // page), page, 1, D, 1, -(-n // page))
    c.extend(ints([0]), ints([n]))
    c.append(0, x.cuda(), x.cuda(), ints([0]), ints([0, n]))
    code, scale, value = codes_ref.quantise(x.double().numpy(), kind)
    k, v = c.read(0, ints([0]), ints([0, n]), total=n)
    assert torch.equal(k.view(torch.int16), v.view(torch.int16))
    got = k.double().cpu().numpy()
    assert np.array_equal(got, value, equal_nan=True)
    order = c.table[0].cpu().numpy()
    assert np.array_equal(c.scales[0, 0, order, 0].cpu().numpy().reshape(-1)[:n], scale[:, 0])


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("tokens_first", [False, True])
def test_read_every_code(K, kind, tokens_first):
    """Every code at every scale that an append may write: the value, where the type holds it."""
    D, page, heads = 256, 4, 2
    lo, hi = (10, 247) if kind == "bf16" else (95, 135)
    n = hi - lo + 1
    c = make(K, kind, 1, -(-n // page), page, heads, D, 1, -(-n // page), tokens_first)
    c.extend(ints([0]), ints([n]))
    codes = np.broadcast_to(np.arange(256, dtype=np.uint8), (n, heads, D))
    scales = np.broadcast_to(np.arange(lo, hi + 1, dtype=np.uint8)[:, None], (n, heads))
    for i in range(n):
        p = int(c.table[0, i // page])
        for x in (0, 1):
            c.codes.view(torch.uint8)[0, x, p, :, i % page] = torch.tensor(codes[i]).cuda()
            c.scales[0, x, p, :, i % page] = torch.tensor(scales[i].copy()).cuda()
    k, v = c.read(0, ints([0]), ints([0, n]), total=n)
    want = codes_ref.values(codes, scales)
    top = np.where(np.abs(want) > codes_ref.MOST[kind], np.nan, want)
    for got in (k, v):
        got = got.double().cpu().numpy()
        held = ~np.isnan(top)
        if kind == "f16":  # below the type's smallest number there is rounding, as nothing that is written has
            held &= np.abs(want) * 2.0 ** 24 == np.rint(np.abs(want) * 2.0 ** 24)
        assert np.array_equal(got[held], want[held])
        assert np.all(np.isnan(got[np.isnan(want)]))


@pytest.mark.parametrize("bits_", [8, 16])
@pytest.mark.parametrize("kind,D,heads,page", [("bf16", 128, 8, 16), ("f16", 64, 3, 1), ("f16", 48, 2, 8), ("bf16", 16, 1, 32)])
def test_read_rows(K, kind, bits_, D, heads, page):
    """Parts of slots, holes, slots that are not there, sequences without rows; rows past the last stay."""
    c = K.PagedCache.new(2, 60 + 200 // page, page, heads, D, 6, -(-90 // page) + 1, TYPES[kind], bits=bits_)
    c.extend(ints([0, 1, 2, 4]), ints([70, 1, 33, 90]))
    new = [70, 1, 33, 90]
    q = np.concatenate([[0], np.cumsum(new)])
    x = [(rows(kind, int(q[-1]), heads, D, s).nan_to_num(1.0, 2.0, -2.0)) for s in (3, 4)]
    c.append(1, x[0].cuda(), x[1].cuda(), ints([0, 1, 2, 4]), ints(q))
    held = {s: [t[q[i]:q[i + 1]].double().numpy() for t in x] for i, s in enumerate([0, 1, 2, 4])}
    if bits_ == 8:
        held = {s: [codes_ref.quantise(t, kind)[2] for t in h] for s, h in held.items()}
    if page < 30:
        c.release(ints([0]), ints([0]), ints([page * 2]))
        for t in held[0]:
            t[:page * 2] = 0
    slot, begin, count = [4, 9, 2, 0, 1, -1, 3, 4], [80, 0, 30, 1, 0, 2, 0, -3], [20, 4, 0, 69, 1, 2, 3, 5]
    start = np.concatenate([[0], np.cumsum(count)])
    total = int(start[-1]) + 4
    want = np.full((2, total, heads, D), 7.0)
    for b, s in enumerate(slot):
        for i in range(count[b]):
            pos = begin[b] + i
            ok = s in held and 0 <= pos < len(held[s][0])
            for w in (0, 1):
                want[w, start[b] + i] = held[s][w][pos] if ok else 0
    out = tuple(torch.full((total, heads, D), 7.0, dtype=TYPES[kind], device="cuda") for _ in range(2))
    got = c.read(1, ints(slot), ints(start), ints(begin), out=out)
    for w in (0, 1):
        assert got[w] is out[w]
        assert np.array_equal(got[w].double().cpu().numpy(), want[w])
    k, v = c.read(1, ints([4]), ints([0, 90]), total=90)
    assert np.array_equal(k.double().cpu().numpy(), held[4][0])


@pytest.mark.parametrize("kind,D,heads", [("bf16", 128, 8), ("f16", 64, 2)])
def test_large_batches(K, kind, D, heads):
    """Many tokens a workgroup, more of them than fit one pass of the grid; keys and values as slices of a projection."""
    page, lens = 16, [20011, 1, 0, 7000, 13]
    n = sum(lens)
    c = K.PagedCache.new(1, -(-n // page) + 5, page, heads, D, 5, -(-max(lens) // page), TYPES[kind], bits=8)
    c.extend(ints(range(5)), ints(lens))
    g = torch.Generator("cuda").manual_seed(5)
    both = torch.randn((n, 3 * heads, D), generator=g, device="cuda", dtype=TYPES[kind])
    k, v = both[:, heads:2 * heads], both[:, 2 * heads:]
    q = ints(np.concatenate([[0], np.cumsum(lens)]))
    c.append(0, k, v, ints(range(5)), q)
    for got, x in zip(c.read(0, ints(range(5)), q, total=n), (k, v)):
        want = codes_ref.quantise(x.double().cpu().numpy(), kind)[2]
        assert np.array_equal(got.double().cpu().numpy(), want)


def test_append_grants(K):
    """Refused requests write nothing; without grants no whole page of several rows is written."""
    c = make(K, "bf16", 1, 12, 4, 2, 16, 6, 8)
    c.extend(ints([0]), ints([8]))
    c.fork(ints([0, 0]), ints([1, 2]), ints([8, 6]))
    granted = c.extend(ints([1, 2]), ints([4, 1000]))
    assert granted.tolist() == [1, 0]
    x = rows("bf16", 8, 2, 16, 3).cuda()
    q = [0, 4, 8]
    before = c.data.clone()
    c.append(0, x, x, ints([1, 2]), ints(q), granted=granted)
    changed = torch.nonzero((c.data != before).flatten(3).any(-1)[0, 0]).flatten().tolist()
    assert changed == [int(c.table[1, 2])]
    before = c.data.clone()
    c.append(0, x, x, ints([1, 2]), ints(q))  # the refused one's tokens end in its own partial page, the rest is shared
    changed = torch.nonzero((c.data != before).flatten(3).any(-1)[0, 0]).flatten().tolist()
    assert changed == [int(c.table[2, 1])]


@pytest.mark.parametrize("pages,page,slots,width,heads,D", [(37, 1, 9, 20, 3, 16), (64, 4, 12, 9, 2, 64), (9001, 2, 40, 300, 1, 48)])
def test_books(K, pages, page, slots, width, heads, D):
    """Forks, copies and compactions move codes and scales as they are."""
    c = make(K, "f16", 2, pages, page, heads, D, slots, width, seed=pages)
    r = kv_ref.Pages(c.data.cpu().numpy(), c.refs.cpu().numpy(), c.table.cpu().numpy(), c.length.cpu().numpy(), page)
    rng = np.random.default_rng(pages)
    for step in range(25):
        pick = rng.permutation(np.arange(-1, slots + 1))[:int(rng.integers(2, slots + 1))]
        kind = rng.choice(["extend", "fork", "fork", "release", "compact", "copy", "reorder"])
        if kind == "extend":
            t = rng.integers(0, page * width // 3 + 2, pick.size)
            assert c.extend(ints(pick), ints(t)).tolist() == r.extend(pick, t)
        elif kind == "fork":
            half = pick.size // 2
            child, parent = pick[:half], rng.choice(pick[half:], half)
            t = np.asarray([int((r.length[p] if 0 <= p < slots else 3) * rng.random()) for p in parent])
            assert c.fork(ints(parent), ints(child), ints(t)).tolist() == r.fork(parent, child, t)
        elif kind == "release":
            c.release(ints(pick[:2]))
            r.release(pick[:2])
        elif kind == "compact":
            table, refs, used = c.compact()
            want = r.compact()
            assert np.array_equal(table.cpu().numpy(), want[0]) and np.array_equal(refs.cpu().numpy(), want[1])
            c.adopt(table, refs)
            r.table, r.refs = want[0], want[1]
        elif kind == "copy":
            free = [p for p in range(pages) if r.refs[p] == 0][:5]
            src = rng.integers(0, pages, len(free))
            src = np.where(np.isin(src, free), -1, src)
            c.copy(ints(src), ints(free))
            for a, b in zip(src, free):
                if a >= 0:
                    r.data[:, :, b] = r.data[:, :, a]
        else:
            parent = rng.integers(-1, pick.size + 1, pick.size)
            assert c.reorder(ints(pick), ints(parent)).tolist() == codes_ref.reorder(r, pick, parent)
        assert np.array_equal(c.refs.cpu().numpy(), r.refs) and np.array_equal(c.length.cpu().numpy(), r.length)
        assert np.array_equal(c.table.cpu().numpy(), r.table)
        assert np.array_equal(c.data.cpu().numpy(), r.data)


def test_unwritten_tokens_are_zeros(K):
    """Room that a new cache gives and nobody has written reads as zeros."""
    c = K.PagedCache.new(1, 4, 16, 2, 64, 1, 4, torch.float16, bits=8)
    c.extend(ints([0]), ints([50]))
    k, v = c.read(0, ints([0]), ints([0, 50]), total=50)
    assert not k.any() and not v.any()


def test_refusals(K):
    c = K.PagedCache.new(1, 4, 16, 2, 64, 2, 4, torch.float16, bits=8)
    one, two = ints([0]), ints([0, 1])
    x = torch.zeros((1, 2, 64), dtype=torch.float16, device="cuda")
    with pytest.raises(TypeError):
        c.append(0, x.bfloat16(), x.bfloat16(), one, two)
    with pytest.raises(TypeError):
        c.append(0, x.view(torch.int16), x, one, two)
    with pytest.raises(ValueError):
        c.read(0, one, two)
    with pytest.raises(ValueError):
        c.read(0, one, ints([0]), total=1)
    with pytest.raises(TypeError):
        c.read(0, one, two, out=(x, x.bfloat16()))
    with pytest.raises(ValueError):
        c.read(0, one, two, out=(x, x[:, :1].contiguous()))
    with pytest.raises(Exception):
        c.read(1, one, two, total=1)
    with pytest.raises(ValueError):
        c.reorder(one, two)
    with pytest.raises(ValueError):
        K.page_bytes(16, 2, 24)
    with pytest.raises(ValueError):
        K.PagedCache.new(1, 4, 16, 2, 64, 2, 4, torch.float16, bits=4)
    with pytest.raises(ValueError):
        K.PagedCache.new(1, 4, 16, 2, 24, 2, 4, torch.float16, bits=8)
    with pytest.raises(TypeError):
        K.PagedCache.new(1, 4, 16, 2, 64, 2, 4, torch.float32, bits=8)
    with pytest.raises(TypeError):
        K.PagedCache.of_bytes(c.data[..., :64], c.refs, c.table, c.length, 16, 2, 64)
    with pytest.raises(ValueError):
        K.PagedCache.new(1, 4, 16, 2, 64, 2, 4).codes
    with pytest.raises(ValueError):  # a plan of a 16-bit cache is not one of an 8-bit cache
        wide = K.PagedCache.new(1, 4, 16, 2, 64, 2, 4, torch.float16)
        plan = K.prefix_plan(wide, one, two, None, None, total_q=1, max_q=1, q_heads=2)
        K.attention(x, c, 0, plan)


def test_empty_calls(K):
    c = K.PagedCache.new(1, 4, 16, 2, 64, 2, 4, torch.float16, bits=8)
    none = ints(np.zeros(0))
    x = torch.zeros((0, 2, 64), dtype=torch.float16, device="cuda")
    c.append(0, x, x, none, ints([0]))
    k, v = c.read(0, none, ints([0]), total=0)
    assert k.shape == v.shape == (0, 2, 64)
    assert c.reorder(none, none).numel() == 0


def test_another_stream(K):
    """Appends and reads on a stream that is given, behind work there, while the current one is busy."""
    c = K.PagedCache.new(1, 80, 16, 4, 64, 3, 40, bits=8)
    slot, q = ints([0, 2]), ints([0, 300, 301])
    c.extend(slot, ints([300, 1]))
    side = torch.cuda.Stream()
    x = torch.zeros((301, 4, 64), dtype=torch.bfloat16, device="cuda")
    want = torch.randn(x.shape, generator=torch.Generator().manual_seed(9)).bfloat16()
    big = torch.randn((4096, 4096), device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        (big @ big).sum()
        x.copy_(want.cuda())
    c.append(0, x, x, slot, q, stream=side)
    k, v = c.read(0, slot, q, total=301, stream=side)
    big @ big
    torch.cuda.current_stream().wait_stream(side)
    values = codes_ref.quantise(want.double().numpy(), "bf16")[2]
    assert np.array_equal(k.double().cpu().numpy(), values) and np.array_equal(v.double().cpu().numpy(), values)
