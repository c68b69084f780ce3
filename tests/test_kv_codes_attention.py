"""Attention over the 8-bit cache: the 16-bit cache's tests with pages of codes,
against the definition in 64 bits on the values that the codes stand for."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import codes_ref  # noqa: E402
import test_kv_attention as base  # noqa: E402
from test_kv_attention import (K, test_cut_and_join_over_a_large_batch, test_decode_lengths,  # noqa: E402, F401
                               test_decode_lengths_cut, test_holes, test_large_scores, test_long_keys_are_split,
                               test_many_members_share, test_max_q_only_chooses, test_page_sizes_and_orders, test_prefill,
                               test_queries_before_the_first_token, test_same_bits_every_time, test_scale,
                               test_shared_beyond_a_member, test_shared_phase, test_shared_phase_pages,
                               test_shared_phase_same_bits, test_shared_prefix, test_slots_outside, test_starts_out_of_order,
                               test_window)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


class Codes(base.Batch):
    """The batch's keys and values as codes; what they stand for takes the place of the data that they were made from."""

    def cache(self, K):
        L, _, pages, heads, page, D = self.data.shape
        x = self.data.double().cpu().numpy()
        code, scale, value = codes_ref.quantise(x, self.dtype)
        first = heads > 1 and page > 1 and self.data.stride(3) < self.data.stride(4)  # [page_size][kv_heads][head_dim]
        c = K.PagedCache.of_bytes(torch.randint(0, 256, (L, 2, pages, K.page_bytes(page, heads, D)), dtype=torch.uint8).cuda(),
                                  base.ints(self.refs), base.ints(self.table), base.ints(self.length), page, heads, D,
                                  dtype=self.torch_dtype, tokens_first=first)
        c.codes.view(torch.uint8).copy_(torch.tensor(code))
        c.scales.copy_(torch.tensor(scale))
        self.data.copy_(torch.tensor(value))
        # bytes of tokens that nobody holds are anything: NaN codes, scales beyond every type
        if not getattr(self, "tidy", False):
            held = np.zeros((pages, page), bool)
            for s in range(self.n_slots):
                for t in range(self.length[s]):
                    p = self.table[s, t // page]
                    if 0 <= p < pages:
                        held[p, t % page] = True
            waste = torch.tensor(~held).cuda()
            code, scale = c.codes.view(torch.uint8).permute(2, 4, 0, 1, 3, 5), c.scales.permute(2, 4, 0, 1, 3)
            code[waste], scale[waste] = 0x7f, 0xff
        return c


@pytest.fixture(autouse=True)
def codes(monkeypatch):
    monkeypatch.setattr(base, "Batch", Codes)


@pytest.mark.parametrize("D,dtype", [(64, "f16"), (128, "bf16")])
@pytest.mark.parametrize("window,n", [(0, 40), (0, 300), (70, 300)])
@pytest.mark.parametrize("q", ["one", "all"])
def test_nan_codes_some_rows_see(K, D, dtype, window, n, q):
    """A NaN code reaches the queries that see it and no other."""
    b = Codes(11, dtype, D, 2, 4, 16, [n, n], [1, 1] if q == "one" else [n, n])
    plain = Codes(11, dtype, D, 2, 4, 16, [n, n], [1, 1] if q == "one" else [n, n])
    ref = plain.run(K, window=window)
    pos = n // 2
    page = b.table[b.slot[0], pos // 16]
    c = b.cache(K)
    c.codes.view(torch.uint8)[0, 1, page, 1, pos % 16, 5] = 0xff
    kw = dict(total_q=b.total, max_q=b.max_q, q_heads=b.Hq)
    args = (c, base.ints(b.slot), base.ints(b.q_start))
    plan = K.window_plan(*args, window, **kw) if window else K.prefix_plan(*args, None, None, **kw)
    out, lse = K.attention(b.q, c, 0, plan)
    first = n - (1 if q == "one" else n)
    p = torch.arange(first, n)
    sees = (p >= pos) & ((p < pos + window) if window else True)
    rows = torch.zeros((b.total, b.Hq, D), dtype=torch.bool)
    rows[:len(p), 4:, 5] = sees[:, None]
    assert torch.equal(torch.isnan(out.cpu()), rows)
    assert torch.equal(lse, ref[1])
    unit = base.UNIT[dtype]  # rows may be done again with weights in 32 bits
    clean = ~rows.cuda()
    assert ((out - ref[0]).float().abs()[clean] <= 4 * unit * ref[0].float().abs()[clean] + 4 * unit * 4).all()


def widen(b):
    """A table so wide that prefixes shared by few rows count."""
    keys = (256 << 20) // (2 * len(b.slot) * b.Hk * b.D) + 1
    b.table = np.pad(b.table, ((0, 0), (0, -(-keys // b.page))), constant_values=-1)
    return b


@pytest.mark.parametrize("dtype,D,group,page,order", [("bf16", 128, 3, 16, "head"), ("f16", 64, 1, 32, "token"),
                                                      ("bf16", 64, 4, 8, "head"), ("f16", 128, 2, 1, "token")])
@pytest.mark.parametrize("shared", [[(8, 2000), (8, 777), (8, 31)], [(24, 640)], [(1, 500)] * 24, [(3, 16)] * 8,
                                    [(0, 90), (24, 1100)], [(8, 0), (8, 1700), (8, 5)], [(20, 300), (1, 2), (1, 1), (2, 3)]])
def test_beams_behind_prompts(K, dtype, D, group, page, order, shared):
    """Few rows a group: the waves are dealt out to shared and own keys, also where one of them is nearly nothing."""
    own = [1 + (11 * i) % 45 for i in range(24)]
    prompt = [t for m, t in shared for _ in range(m)]
    b = widen(Codes(41, dtype, D, 2, group, page, [p + x for p, x in zip(prompt, own)], [1] * 24, shared=shared, order=order))
    b.check(K)


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 64)])
def test_few_queries_behind_prompts(K, dtype, D):
    """Up to three query tokens a sequence, sequences without any and without a slot, more rows in a group than a tile."""
    q = [1, 3, 0, 2, 1, 1, 3, 2, 1, 0, 1, 1, 2, 1, 3, 1]
    own = [max(1, x) + (7 * i) % 40 for i, x in enumerate(q)]
    prompt = [700] * 3 + [33] * 2 + [1200] * 11
    b = widen(Codes(42, dtype, D, 2, 2, 16, [p + x for p, x in zip(prompt, own)], q, shared=[(3, 700), (2, 33), (11, 1200)]))
    b.check(K)
    b.slot[7] = -1
    b.slot[12] = b.n_slots
    b.check(K)


@pytest.mark.parametrize("q", [1, 70])
def test_offsets_past_32_bits(K, q):
    """Pages, layers and scales beyond 2^32 bytes."""
    D, heads, page, pages = 128, 8, 64, 40000
    block = K.page_bytes(page, heads, D)
    data = torch.empty((1, 2, pages, block), dtype=torch.uint8, device="cuda")
    assert data.numel() > 2 ** 32
    n = 200
    width = -(-n // page)
    table = base.ints([[pages - 1, 3, pages - 2, 12345][:width]])
    c = K.PagedCache.of_bytes(data, base.ints(np.ones(pages)), table, base.ints([n]), page, heads, D)
    x = torch.randn((2, n, heads, D), generator=torch.Generator().manual_seed(1)).bfloat16()
    c.append(0, x[0].cuda(), x[1].cuda(), base.ints([0]), base.ints([0, n]))
    k, v = c.read(0, base.ints([0]), base.ints([0, n]), total=n)
    value = [codes_ref.quantise(t.double().numpy(), "bf16")[2] for t in x]
    assert np.array_equal(k.double().cpu().numpy(), value[0]) and np.array_equal(v.double().cpu().numpy(), value[1])
    qs = torch.randn((q, heads * 4, D), generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    plan = K.prefix_plan(c, base.ints([0]), base.ints([0, q]), None, None, total_q=q, max_q=q, q_heads=heads * 4)
    out, lse = K.attention(qs, c, 0, plan)
    pool = np.stack([t.transpose(1, 0, 2).reshape(heads, n, D) for t in value])
    pool = np.concatenate([pool, np.zeros((2, heads, width * page - n, D))], 2)
    pool = pool.reshape(2, heads, width, page, D).transpose(0, 2, 1, 3, 4)
    ref = base.kv_ref.attention(qs.cpu().double().numpy(), pool, np.arange(width)[None], np.asarray([n]), [0], [0, q], page, D ** -0.5)
    b_out, b_lse = base.kv_ref.bounds(*ref, 2.0 ** -8, n, float(np.abs(value[1]).max()), D)
    assert np.all(np.abs(out.double().cpu().numpy() - ref[0]) <= b_out)
    assert np.all(np.abs(lse.double().cpu().numpy() - ref[1]) <= b_lse)


def test_captured_step(K):
    """Append and attention in a graph, replayed among eager work: every replay is the eager result."""
    b = Codes(5, "bf16", 128, 2, 4, 16, [100, 33, 257], [1, 1, 1])
    c = b.cache(K)
    slot, q_start = base.ints(b.slot), base.ints(b.q_start)
    plan = K.prefix_plan(c, slot, q_start, None, None, total_q=3, max_q=1, q_heads=b.Hq)
    k, v = (torch.randn((3, 2, 128), device="cuda").bfloat16() for _ in range(2))
    from paper_2601_21758_amd import ewsjf
    ws = ewsjf.Workspace()

    def step():
        c.append(0, k, v, slot, q_start)
        return (*K.attention(b.q, c, 0, plan, ws=ws), *c.read(0, slot, q_start, total=3))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(4):
        k.copy_(torch.randn(k.shape, device="cuda"))
        v.copy_(torch.randn(v.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in got]
        for a, e in zip(kept, step()):
            assert torch.equal(a, e)
