"""Every step of a search by beams, with a cache of 16 or 8 bits, against the model in 64 bits: each beam's score, and that
no candidate which was left out is better than one that was picked."""
import math
import os
import sys

import numpy as np
import pytest

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import codes_ref  # noqa: E402

torch = pytest.importorskip("torch")

# The oracle rounds to float16 where the server does (a layer's input, q, k, v, the attention's output, the branch, the
# logits) and quantises as the cache does, so what is left are sums of another order (2^-22), which move few roundings, and
# the attention's weights of 16 bits: 0.00031 of the output's norm.  So the second layer's k and v are off by 0.0005 with
# their own roundings.  A code of 8 bits then moves a step, 9% of its value on average, with probability 0.0004 / 0.09: in
# the mean square 0.0004 * 0.09, 0.6% of a key's or value's elements.  A score of at most 8 is off by 0.6% of 8 / 2 = 0.024
# (k's elements are independent), so the weights by 2.4%, the second branch by less than 2.5% of itself (it averages over several
# weights), the residual, to which two branches of about the same size were added, by 1.7%, and a logit by 0.017 of the logits'
# spread; a log probability by hardly more, as the mean over all logits is right.  Three times that is 0.05.
# The errors of a sum's terms are those of different positions: their squares add.
NEAR = 0.05


def r16(x):
    return x.to(torch.float16).double()


class Oracle:
    """The model's log probabilities in 64 bits, rounded and quantised where the server's are."""

    def __init__(self, c, embed, qkv, out, head, noise=0.0):
        self.c, self.noise, self.known = c, noise, {}
        self.embed, self.head = embed.double().cpu(), head.double().cpu()
        self.qkv, self.out = ([w.double().cpu() for w in ws] for ws in (qkv, out))
        self.g = torch.Generator().manual_seed(0)

    @classmethod
    def of(cls, model, **kw):
        return cls(model.c, model.embed, model.qkv, model.out, model.head, **kw)

    def held(self, x):
        return torch.from_numpy(codes_ref.quantise(x.numpy(), "f16")[2]) if self.c.bits == 8 else x

    def logits(self, tokens, first):
        c = self.c
        x = self.embed[torch.tensor(tokens)]
        n, G = len(tokens), c.q_heads // c.kv_heads
        i, j = torch.arange(n)[:, None], torch.arange(n)[None]
        for layer in range(c.layers):
            h = r16(x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6))
            q, k, v = r16(h @ self.qkv[layer]).view(n, -1, c.head_dim).split([c.q_heads, c.kv_heads, c.kv_heads], 1)
            k, v = (self.held(t).repeat_interleave(G, 1) for t in (k, v))
            s = torch.matmul(q.transpose(0, 1), k.permute(1, 2, 0)) / math.sqrt(c.head_dim)
            seen = j <= i
            if layer % 2:
                seen = seen & ((j > i - c.window) | (j < c.sinks))
            o = torch.matmul(s.masked_fill(~seen, -math.inf).softmax(-1), v.transpose(0, 1))
            if self.noise:
                o = o + self.noise * o.norm(dim=-1, keepdim=True) * c.head_dim ** -0.5 * torch.randn(
                    o.shape, generator=self.g, dtype=o.dtype)
            x = x + r16(r16(o).transpose(0, 1).reshape(n, c.width) @ self.out[layer])
        x = x[first:]
        return r16(r16(x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)) @ self.head)

    def rows(self, prompt, answer):
        """The logits' log probabilities after the prompt and each token of the answer, and their spread."""
        key = tuple(prompt), tuple(answer)
        if key not in self.known:
            x = self.logits(prompt + answer, len(prompt) - 1)
            self.known[key] = torch.log_softmax(x, -1).numpy(), float(x.std())
        return self.known[key]

    def beam(self, prompt, answer):
        """A beam's score, its next tokens' log probabilities, whether it is at its end, the logits' spread."""
        p, spread = self.rows(prompt, answer)
        done = self.c.end in answer
        score = sum(p[i, answer[i]] for i in range(answer.index(self.c.end) + 1 if done else len(answer)))
        return score, p[-1], done, spread


def wrong_steps(oracle, prompt, before, answers, scores, mistake=None):
    """How many of a step's beams are not what they should be.  before: the beams that it continued; mistake: which the
    oracle makes."""
    c, bad = oracle.c, 0
    held = [oracle.beam(prompt, a) for a in before]
    base = [h[0] for h in held]
    if mistake == "beams":  # each goes on from its neighbour's score
        base = base[1:] + base[:1]
    if mistake == "step":  # the last token before this one is forgotten
        base = [oracle.beam(prompt, a[:-1])[0] if a else 0.0 for a in before]
    candidates = {}
    for a, b, (_, p, done, _) in zip(before, base, held):
        for t in [c.end] if done else range(c.vocab):
            candidates[tuple(a) + (t,)] = b + (0.0 if done else p[t])
    room = NEAR * max(h[3] for h in held) * math.sqrt(len(answers[0]))
    picked = [candidates.get(tuple(a)) for a in answers]
    bad += sum(p is None for p in picked)
    left = [s for a, s in candidates.items() if a not in {tuple(a) for a in answers}]
    for p, s in zip(picked, scores):
        if p is not None:
            bad += not abs(p - s) <= room
            bad += not p >= max(left) - 2 * room  # both may be off
    return bad + (len({tuple(a) for a in answers}) < len(answers))


def config(serve, bits, beams, end):
    return serve.Config(layers=2, q_heads=4, kv_heads=2, head_dim=64, vocab=64, dtype=torch.float16, window=24, sinks=2,
                        n_pages=160, slots=17, admit=3, answer=7, compact_every=2, bits=bits, beams=beams, end=end)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("prefix,beams,end", [(0, 3, -1), (37, 4, -1), (20, 5, 7)])
def test_every_step(bits, prefix, beams, end):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2601_21758_amd import serve
    c = config(serve, bits, beams, end)
    rng = np.random.default_rng(prefix)
    prompts = [rng.integers(0, c.vocab, n).tolist() for n in [1, 50, 17, 16, 15, 33, 2, 90, 5]]
    server = serve.BeamServer(serve.Model(c), rng.integers(0, c.vocab, prefix).tolist(), prompts)
    oracle = Oracle.of(server.model)
    steps, wrong, found, counted = 0, 0, {}, {"beams": 0, "step": 0}
    while len(server.answers) < len(prompts):
        before = {id(r): (r, [list(a) for a in r.answers]) for r in server.running}
        running = list(server.running)
        server.step()
        for r in running + [r for r in server.running if r not in running]:
            then = before[id(r)][1] if id(r) in before else [[]]
            args = server.prefix + prompts[r.id], then, r.answers, r.scores
            wrong += wrong_steps(oracle, *args)
            steps += 1
            if then != [[]]:
                for mistake in counted:
                    counted[mistake] += wrong_steps(oracle, *args, mistake=mistake) > 0
            found[r.id] = r.answers[0], r.scores[0]
    assert wrong == 0
    assert {i: (a, server.scores[i]) for i, a in server.answers.items()} == found
    later = steps - len(prompts)
    # the oracle with a mistake is told apart; neighbours' scores may be close to one another
    assert counted["beams"] > 0.7 * later and counted["step"] > 0.9 * later


@pytest.mark.parametrize("bits", [8, 16])
def test_the_tolerance(bits):
    """What the attention's 16-bit weights do to log probabilities, in the oracle itself, is within NEAR."""
    from paper_2601_21758_amd import serve
    c = config(serve, bits, 4, -1)
    rng = np.random.default_rng(3)
    g = torch.Generator().manual_seed(0)

    def draw(*shape, std):
        return (torch.randn(*shape, generator=g) * std).to(c.dtype)

    heads = c.q_heads + 2 * c.kv_heads
    weights = (draw(c.vocab, c.width, std=1.0), [draw(c.width, heads * c.head_dim, std=c.width ** -0.5) for _ in range(2)],
               [draw(c.width, c.width, std=8 * c.width ** -0.5) for _ in range(2)], draw(c.width, c.vocab, std=c.width ** -0.5))
    exact, noisy = Oracle(c, *weights), Oracle(c, *weights, noise=0.00031)
    worst = []
    for n in [1, 50, 17, 16, 15, 33, 2, 90, 5]:
        prompt, answer = rng.integers(0, c.vocab, n).tolist(), rng.integers(0, c.vocab, 6).tolist()
        (a, spread), (b, _) = exact.rows(prompt, answer), noisy.rows(prompt, answer)
        worst.append(np.abs(a - b).max() / spread)
    assert 0 < max(worst) <= NEAR
