"""The small server against its model in 64 bits, request by request."""
import math
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# Greedy tokens of float16 and of 64 bits differ where logits are close.  A layer rounds its input, q, k and v (2^-11
# each); scores stay below about 8, so a weight is off by up to 8 * 2 * 2^-11, the branch by 22 * 2^-11 with its own
# roundings, about 1%; two layers, each adding as much again to what it was given, leave 4% of a logit's spread, and the
# worst of 256 differences four times that: 0.17.
NEAR = 0.25


def logits(m, tokens, first, windowed=True):
    """Logits after tokens[first:], in float64."""
    c = m.c
    w = [x.double().cpu() for x in m.qkv], [x.double().cpu() for x in m.out], m.embed.double().cpu(), m.head.double().cpu()
    x = w[2][torch.tensor(tokens)]
    n, G = len(tokens), c.q_heads // c.kv_heads
    i, j = torch.arange(n)[:, None], torch.arange(n)[None]
    for layer in range(c.layers):
        h = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
        q, k, v = (h @ w[0][layer]).view(n, -1, c.head_dim).split([c.q_heads, c.kv_heads, c.kv_heads], 1)
        k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
        s = torch.matmul(q.transpose(0, 1), k.permute(1, 2, 0)) / math.sqrt(c.head_dim)
        seen = j <= i
        if layer % 2 and windowed:
            seen = seen & ((j > i - c.window) | (j < c.sinks))
        o = torch.matmul(s.masked_fill(~seen, -math.inf).softmax(-1), v.transpose(0, 1))
        x = x + o.transpose(0, 1).reshape(n, c.width) @ w[1][layer]
    x = x[first:]
    return (x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)) @ w[3]


def misses(server, wrong=False):
    """Answered tokens whose logit is further from the largest than NEAR of the logits' spread.  wrong: against a model
    that does not see the prefix and has no windows."""
    bad = 0
    for i, answer in server.answers.items():
        before = ([] if wrong else server.prefix) + server.prompts[i]
        x = logits(server.model, before + answer[:-1], len(before) - 1, windowed=not wrong).numpy()
        gap = x.max(1) - x[np.arange(len(answer)), answer]
        bad += int((gap > NEAR * x.std(1)).sum())
    return bad


@pytest.mark.parametrize("prefix", [0, 37, 64])
def test_answers(prefix):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import serve
    c = serve.Config(layers=2, q_heads=4, kv_heads=2, head_dim=64, vocab=256, dtype=torch.float16, window=24, sinks=2,
                     n_pages=64, slots=9, admit=4, answer=6, compact_every=2)
    rng = np.random.default_rng(prefix)
    prompts = [rng.integers(0, c.vocab, n).tolist() for n in [1, 50, 17, 16, 15, 33, 2, 90, 5, 8, 64, 31, 3, 44, 12, 1]]
    server = serve.Server(serve.Model(c), rng.integers(0, c.vocab, prefix).tolist(), prompts)
    answers = server.run()
    assert sorted(answers) == list(range(len(prompts))) and all(len(a) == c.answer for a in answers.values())
    assert server.room == c.n_pages - -(-prefix // c.page_size) and sorted(server.free) == list(range(1, c.slots + 1))
    assert int(server.cache.refs.sum()) == -(-prefix // c.page_size)
    assert server.cache.length.tolist() == [prefix] + [0] * c.slots
    assert misses(server) == 0
    if prefix:
        assert misses(server, wrong=True) > 20  # the oracle with the mistake is told apart


def test_a_request_that_never_fits():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import serve
    c = serve.Config(layers=1, q_heads=2, kv_heads=1, head_dim=64, vocab=16, n_pages=4, slots=2, admit=2, answer=2)
    with pytest.raises(RuntimeError, match="does not fit"):
        serve.Server(serve.Model(c), [1] * 20, [[2] * 60]).run()
