"""A small server: the scheduler's admissions turned into tokens, all on one
GPU and one stream.

    python -m paper_2601_21758_amd.serve --requests 256 --prefix 2048 --answer 64

Prompts wait in the scheduler's pool behind one common prefix (a system
prompt), which is in the cache from the start, in slot 0.  Each step

  * lets the scheduler admit prompts (ewsjf_step) as long as slots and pages
    are left for what they may grow to,
  * forks the prefix for each, which shares its pages and copies only a
    partial one (ewsjf_cache_fork), and makes room for the step's tokens: a
    whole prompt for a new request, one token for a running one
    (ewsjf_cache_extend),
  * plans the batch once (ewsjf_prefix_plan, ewsjf_window_plan) and runs the
    layers, which write their keys and values (ewsjf_cache_append) and attend
    (ewsjf_attention): even layers to every token, the prefix read once for
    all requests, odd layers to the first `sinks` and the last `window`,
  * empties the slots of finished requests (ewsjf_cache_release) and, every
    `compact_every` steps, moves the used pages to the front of the pool
    (ewsjf_cache_compact).

The model is a stand-in, random weights without positions: it has the calls
and layouts of one, and the next token is the likeliest.
"""
from __future__ import annotations

import argparse
import json
import time
from dataclasses import dataclass, field

import numpy as np
import torch

from . import ewsjf, kv
from . import workloads as W
from .streaming import StreamingScheduler


@dataclass(frozen=True)
class Config:
    layers: int = 4
    q_heads: int = 32
    kv_heads: int = 8
    head_dim: int = 128
    vocab: int = 4096
    dtype: torch.dtype = torch.bfloat16
    page_size: int = 16
    window: int = 512       # of the odd layers
    sinks: int = 4
    n_pages: int = 16384
    slots: int = 128        # requests that run at once
    admit: int = 16         # requests that a step admits
    answer: int = 32        # tokens that a request is given
    compact_every: int = 32

    @property
    def width(self) -> int:
        return self.q_heads * self.head_dim


def _norm(x: torch.Tensor) -> torch.Tensor:
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)


class Model:
    """Layers of attention alone over a residual in float32."""

    def __init__(self, c: Config, seed: int = 0, device="cuda"):
        g = torch.Generator().manual_seed(seed)
        self.c = c
        heads = c.q_heads + 2 * c.kv_heads

        def draw(*shape, std):
            return (torch.randn(*shape, generator=g) * std).to(c.dtype).to(device)

        self.embed = draw(c.vocab, c.width, std=1.0)
        self.qkv = [draw(c.width, heads * c.head_dim, std=c.width ** -0.5) for _ in range(c.layers)]
        # attention averages over many values: enough that it outweighs the token itself
        self.out = [draw(c.width, c.width, std=8 * c.width ** -0.5) for _ in range(c.layers)]
        self.head = draw(c.width, c.vocab, std=c.width ** -0.5)
        self.ws = ewsjf.Workspace(device)

    def forward(self, tokens: torch.Tensor, cache: kv.PagedCache, slot: torch.Tensor, q_start: torch.Tensor,
                plans, last: torch.Tensor) -> torch.Tensor:
        """The likeliest next token after each of tokens[last]; plans: of the even layers and of the odd ones."""
        c, n = self.c, tokens.numel()
        x = self.embed[tokens].float()
        for layer in range(c.layers):
            heads = (_norm(x).to(c.dtype) @ self.qkv[layer]).view(n, -1, c.head_dim)
            q, k, v = heads.split([c.q_heads, c.kv_heads, c.kv_heads], 1)
            cache.append(layer, k, v, slot, q_start)
            o, _ = kv.attention(q, cache, layer, plans[layer % 2], ws=self.ws)
            x += o.view(n, c.width) @ self.out[layer]
        return (_norm(x[last]).to(c.dtype) @ self.head).argmax(-1)


@dataclass
class Request:
    id: int
    slot: int
    pages: int                                    # that it may come to hold
    answer: list = field(default_factory=list)    # tokens, the last one not in the cache yet


class Server:
    """prefix: the common first tokens; prompts: a list of token lists, never empty."""

    def __init__(self, model: Model, prefix, prompts, device="cuda"):
        c = self.c = model.c
        self.model, self.device = model, torch.device(device)
        self.prefix, self.prompts = list(prefix), [list(p) for p in prompts]
        longest = len(self.prefix) + max(len(p) for p in self.prompts) + c.answer
        self.cache = kv.PagedCache.new(c.layers, c.n_pages, c.page_size, c.kv_heads, c.head_dim, c.slots + 1,
                                       -(-longest // c.page_size), c.dtype, device)
        self.ws = ewsjf.Workspace(device)
        self.used = torch.zeros(1, dtype=torch.int32, device=device)
        self.free = list(range(c.slots, 0, -1))
        self.room = c.n_pages - -(-len(self.prefix) // c.page_size)
        self.running: list[Request] = []
        self.admitted: list[int] = []  # by the scheduler, without a slot yet
        self.answers: dict[int, list[int]] = {}
        self.steps = 0
        lengths = np.asarray([len(p) for p in self.prompts], np.int32)
        self.scheduler = StreamingScheduler(lengths.size, lengths.size, c.admit, ewsjf.params(), W.THETA_MID,
                                            device=device)
        self.scheduler.fill(lengths, np.zeros(lengths.size, np.float32))
        if self.prefix:
            self._run([(0, self.prefix)], shared=0)

    def _ints(self, *lists) -> list[torch.Tensor]:
        """Lists as int32 tensors on the device, in one copy."""
        flat = torch.tensor([x for one in lists for x in one], dtype=torch.int32).to(self.device)
        return list(flat.split([len(one) for one in lists]))

    def _granted(self, granted: torch.Tensor) -> None:
        if not bool(granted.all()):
            raise RuntimeError("the pool is out of pages")

    def _run(self, batch, shared: int) -> list[int]:
        """A forward pass of (slot, its new tokens): the next token of each."""
        c, cache = self.c, self.cache
        counts = [len(t) for _, t in batch]
        start = np.concatenate([[0], np.cumsum(counts)]).tolist()
        slot, count, q_start, last, groups, shared_, tokens = self._ints(
            [s for s, _ in batch], counts, start, [e - 1 for e in start[1:]], [0, len(batch)], [shared],
            [x for _, t in batch for x in t])
        self._granted(cache.extend(slot, count, ws=self.ws))
        sizes = dict(total_q=start[-1], max_q=max(counts), q_heads=c.q_heads)
        plans = (kv.prefix_plan(cache, slot, q_start, groups, shared_, **sizes),
                 kv.window_plan(cache, slot, q_start, c.window, c.sinks, **sizes))
        return self.model.forward(tokens, cache, slot, q_start, plans, last).tolist()

    def _pages(self, request: int) -> int:
        """Pages that a request may come to hold besides the shared ones."""
        own = len(self.prefix) + len(self.prompts[request]) + self.c.answer
        return -(-own // self.c.page_size) - len(self.prefix) // self.c.page_size

    def _admit(self) -> list[Request]:
        c, new = self.c, []
        if not self.admitted:
            ids, _, n = self.scheduler.step(float(self.steps))
            self.admitted = ids[0, :int(n)].tolist()
        while self.admitted and self.free and self._pages(self.admitted[0]) <= self.room:
            i = self.admitted.pop(0)
            new.append(Request(i, self.free.pop(), self._pages(i)))
            self.room -= new[-1].pages
        if new and self.prefix:
            zeros, child, tokens = self._ints([0] * len(new), [r.slot for r in new], [len(self.prefix)] * len(new))
            self._granted(self.cache.fork(zeros, child, tokens, ws=self.ws))
        return new

    def step(self) -> int:
        """One batch; the number of tokens that it answered with."""
        new = self._admit()
        old, self.running = self.running, self.running + new
        if not self.running:
            if self.admitted:
                raise RuntimeError("a request does not fit the pool")
            return 0
        batch = [(r.slot, r.answer[-1:]) for r in old] + [(r.slot, self.prompts[r.id]) for r in new]
        for r, token in zip(self.running, self._run(batch, len(self.prefix))):
            r.answer.append(token)
        done = [r for r in self.running if len(r.answer) == self.c.answer]
        if done:
            self.cache.release(*self._ints([r.slot for r in done]))
            self.running = [r for r in self.running if len(r.answer) < self.c.answer]
            for r in done:
                self.answers[r.id] = r.answer
                self.free.append(r.slot)
                self.room += r.pages
        self.steps += 1
        if self.steps % self.c.compact_every == 0:
            self.cache.compact(out=(self.cache.table, self.cache.refs, self.used), ws=self.ws)
        return len(batch)

    def run(self) -> dict[int, list[int]]:
        """Every request's answer."""
        while len(self.answers) < len(self.prompts):
            self.step()
        return self.answers


def main(argv=None) -> dict:
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--requests", type=int, default=256)
    ap.add_argument("--prefix", type=int, default=2048, help="tokens that all prompts begin with")
    ap.add_argument("--prompt", type=int, default=128, help="the longest prompt's own tokens")
    ap.add_argument("--answer", type=int, default=32, help="tokens of an answer")
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    if min(a.requests, a.prompt, a.answer, a.layers) < 1 or a.prefix < 0:
        ap.error("requests, prompt, answer and layers are at least 1, prefix at least 0")
    c = Config(layers=a.layers, answer=a.answer)
    rng = np.random.default_rng(a.seed)
    prompts = [rng.integers(0, c.vocab, n).tolist() for n in rng.integers(1, a.prompt + 1, a.requests)]
    server = Server(Model(c, a.seed), rng.integers(0, c.vocab, a.prefix).tolist(), prompts)
    torch.cuda.synchronize()
    t = time.perf_counter()
    server.run()
    torch.cuda.synchronize()
    t = time.perf_counter() - t
    tokens = a.requests * a.answer
    line = {"requests": a.requests, "prefix": a.prefix, "layers": a.layers, "steps": server.steps, "tokens": tokens,
            "seconds": round(t, 4), "tokens_per_second": round(tokens / t, 1)}
    print(json.dumps(line))
    return line


if __name__ == "__main__":
    main()
