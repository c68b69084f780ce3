"""The small server with a cache of 8 bits and with beams, against its model in 64 bits."""
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from test_serve import NEAR, logits  # noqa: E402

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# Codes are off by half a step at most, 2^-4 of a value, by 2^-4 / sqrt(3) times 0.72 on average over a binade: 2.6% of a
# key's or value's elements, independently.  A branch's scores and values are so off by 3.7% together, beside the 1% of
# 16 bits: 4.7 times as much, and the worst difference of some hundred 0.8 of a logit's spread where NEAR has 0.17.
NEAR_8 = 1.0


@pytest.mark.parametrize("prefix", [0, 37])
def test_answers_from_8_bits(prefix):
    """The answers of a cache of 8 bits."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import serve
    c = serve.Config(layers=2, q_heads=4, kv_heads=2, head_dim=64, vocab=256, dtype=torch.float16, window=24, sinks=2,
                     n_pages=64, slots=9, admit=4, answer=6, compact_every=2, bits=8)
    rng = np.random.default_rng(prefix)
    prompts = [rng.integers(0, c.vocab, n).tolist() for n in [1, 50, 17, 16, 15, 33, 2, 90, 5, 8, 64, 31, 3, 44, 12, 1]]
    server = serve.Server(serve.Model(c), rng.integers(0, c.vocab, prefix).tolist(), prompts)
    assert server.cache.bits == 8
    server.run()
    gaps = []
    for i, answer in server.answers.items():
        x = logits(server.model, server.prefix + prompts[i] + answer[:-1], prefix + len(prompts[i]) - 1).numpy()
        gaps.append((x.max(1) - x[np.arange(c.answer), answer]) / x.std(1))
    assert np.max(gaps) <= NEAR_8 and np.mean(np.concatenate(gaps)) <= NEAR_8 / 4


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("prefix,beams,end", [(0, 3, -1), (37, 4, -1), (20, 5, 7)])
def test_beams(bits, prefix, beams, end):
    """Beams through the whole path: their scores are those of their tokens in 64 bits, they differ from one another, the
    books are clean at the end."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import serve
    c = serve.Config(layers=2, q_heads=4, kv_heads=2, head_dim=64, vocab=64, dtype=torch.float16, window=24, sinks=2,
                     n_pages=160, slots=17, admit=3, answer=7, compact_every=2, bits=bits, beams=beams, end=end)
    rng = np.random.default_rng(prefix)
    prompts = [rng.integers(0, c.vocab, n).tolist() for n in [1, 50, 17, 16, 15, 33, 2, 90, 5]]
    server = serve.BeamServer(serve.Model(c), rng.integers(0, c.vocab, prefix).tolist(), prompts)
    seen = []
    while len(server.answers) < len(prompts):
        server.step()
        for r in server.running:
            seen.append(len({tuple(a) for a in r.answers}) == len(r.answers) or any(r.done))
            assert r.scores == sorted(r.scores, reverse=True)
    assert all(seen)
    assert sorted(server.answers) == list(range(len(prompts)))
    assert server.room == c.n_pages - -(-prefix // c.page_size) and sorted(server.free) == list(range(1, c.slots + 1))
    assert int(server.cache.refs.sum()) == -(-prefix // c.page_size)
    assert server.cache.length.tolist() == [prefix] + [0] * c.slots
    for i, answer in server.answers.items():
        x = logits(server.model, server.prefix + prompts[i] + answer[:-1], prefix + len(prompts[i]) - 1)
        p = torch.log_softmax(x, -1)[torch.arange(len(answer)), answer]
        if end in answer:  # nothing is added behind the end
            p = p[:answer.index(end) + 1]
            assert set(answer[answer.index(end):]) == {end}
        # a token's log probability is off by what its logit is
        assert abs(float(p.sum()) - server.scores[i]) <= len(p) * (NEAR_8 if bits == 8 else NEAR) * float(x.std())


def test_one_beam_is_greedy():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import serve
    c = serve.Config(layers=2, q_heads=4, kv_heads=2, head_dim=64, vocab=256, dtype=torch.float16, n_pages=64, slots=5,
                     admit=2, answer=6, compact_every=3)
    rng = np.random.default_rng(1)
    prompts = [rng.integers(0, c.vocab, n).tolist() for n in [1, 20, 17, 16, 40]]
    prefix = rng.integers(0, c.vocab, 21).tolist()
    model = serve.Model(c)
    assert serve.BeamServer(model, prefix, prompts).run() == serve.Server(model, prefix, prompts).run()


@pytest.mark.parametrize("bits", [8, 16])
def test_captured_search(bits):
    """Whole steps of a search in a graph, selection, reordering, room, appends, plan and attention, replayed among eager work:
    the same answers, books and outputs as eager steps of a cache of its own."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import beam, kv
    G, B, H, D, V = 5, 4, 2, 64, 700
    n = G * B
    g = torch.Generator("cuda").manual_seed(bits)
    slot, ones = torch.arange(n, dtype=torch.int32, device="cuda"), torch.ones(n, dtype=torch.int32, device="cuda")
    q_start = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    logits, q = torch.zeros((n, V), device="cuda"), torch.zeros((n, 2 * H, D), dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros((n, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))

    class Search:
        def __init__(self):
            self.cache = kv.PagedCache.new(1, 80, 4, H, D, n, 12, bits=bits)
            self.score = torch.zeros(n, device="cuda")

        def step(self):
            parent, token, score = beam.beam_select(logits, self.score, B)
            c = self.cache
            kept = c.reorder(slot, parent.flatten())
            room = c.extend(slot, ones)
            c.append(0, k, v, slot, q_start, granted=room)
            plan = kv.prefix_plan(c, slot, q_start, None, None, total_q=n, max_q=1, q_heads=2 * H)
            out, lse = kv.attention(q, c, 0, plan)
            self.score.copy_(score.flatten())
            return parent, token, kept, room, out, lse

        def books(self):
            return self.cache.refs, self.cache.table, self.cache.length, self.score

    def draw():
        for t in (logits, q, k, v):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda") * 3)

    eager, replayed = Search(), Search()
    draw()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        replayed.step()
    torch.cuda.current_stream().wait_stream(side)
    eager.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = replayed.step()
    for _ in range(9):
        draw()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((*got, *replayed.books()), (*eager.step(), *eager.books())):
            assert torch.equal(a, b)
    assert int(eager.cache.length.min()) == 10
