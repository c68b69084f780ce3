"""The workloads the 8-bit cache's and the beam operators' speed is measured on.

What a server calls between two decoding steps whose cache is held in 8 bits
and whose requests are answered by beams:

  write    new tokens' keys and values, quantised as they are written into
           their pages, and read back;
  read     whole requests read out of an 8-bit cache as 16-bit keys and values;
  attend   attention of single tokens, chunks of new tokens and prompts over an
           8-bit cache;
  select   each request's next tokens from its beams' logits;
  reorder  the beams' slots after that: each takes over its parent's pages.

A quantised value is an e4m3 code times a power of two, one for each token and
key head: the smallest 2^e with |x| <= 448 2^e for all of them.

Prompt lengths follow the framework's workloads: short ones lognormal(ln 128,
0.6), long ones lognormal(ln 6000, 0.4), 80 to 20, up to 32,768 tokens.
Lengths are the quantiles of the distribution, in an order drawn from the
seed, so a case's work is known.

Where `own` is false `run` evaluates the definitions with elementary torch
operations in 32 bits, the logits' sums and the scores in 64; where it is true
it makes the framework's calls.
"""
from __future__ import annotations

import math
import statistics

import numpy as np
import torch

own = False

MAX_LEN = 32768
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}
# The largest magnitude that is quantised: 240 2^e, which the type still holds (256 2^e would not be).
MOST = {"bf16": 1.875 * 2.0 ** 127, "f16": 61440.0}
LEAST_EXP = -117  # of a scale
FLOOR = -3e38     # the running maximum of a row that has seen no key


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # Eight sequences of a small model take one new token each (latency).
        dict(name="write_8", kind="write", dtype="f16", seqs=8, mix="one", median=700, q_most=1, kv_heads=2, dim=64,
             page=16, fused=0),
        # 24 whole prompts of both length modes are written, keys and values as slices of the fused projection.
        dict(name="write_ragged", kind="write", dtype="bf16", seqs=24, mix="two", median=128, q_most=MAX_LEN,
             kv_heads=8, dim=128, page=16, fused=1),
        # Three short requests of a small model leave for another card (latency).
        dict(name="read_3", kind="read", dtype="f16", seqs=3, mix="one", median=200, q_most=1, kv_heads=3, dim=64,
             page=32, fused=0),
        # 64 requests of both length modes are read out, as a server does that frees a card.
        dict(name="read_64", kind="read", dtype="bf16", seqs=64, mix="two", median=128, q_most=1, kv_heads=8, dim=128,
             page=16, fused=0),
        # The smallest decoding step: three sequences, one key head (latency).
        dict(name="attend_3", kind="attend", dtype="f16", seqs=3, mix="one", median=1000, q_most=1, q_heads=8,
             kv_heads=1, dim=64, page=16, window=0, sinks=0, beams=1, fused=0),
        # The decoding step of 256 requests of both length modes, window 4,096.
        dict(name="attend_256", kind="attend", dtype="bf16", seqs=256, mix="two", median=128, q_most=1, q_heads=32,
             kv_heads=8, dim=128, page=16, window=4096, sinks=4, beams=1, fused=0),
        # 32 requests of eight beams each, a request's beams behind its prompt.
        dict(name="attend_beams", kind="attend", dtype="f16", seqs=32, mix="one", median=2000, q_most=1, q_heads=24,
             kv_heads=8, dim=128, page=16, window=0, sinks=0, beams=8, fused=0),
        # Chunks of 512 new tokens behind some thousand that are held, queries as a slice of the fused projection.
        dict(name="attend_chunk", kind="attend", dtype="f16", seqs=12, mix="one", median=6000, q_most=512, q_heads=20,
             kv_heads=4, dim=64, page=32, window=0, sinks=0, beams=1, fused=1),
        # One request of four beams, logits in 32 bits (latency).
        dict(name="select_4", kind="select", dtype="f32", groups=1, beams=4, picks=8, vocab=32000, masked=0.0,
             done=0, first=0),
        # 64 requests of eight beams, twice as many candidates as beams, some beams at their end.
        dict(name="select_512", kind="select", dtype="bf16", groups=64, beams=8, picks=16, vocab=131072, masked=0.0,
             done=1, first=0),
        # Two requests of four beams on a small model with a 16-bit cache (latency).
        dict(name="reorder_8", kind="reorder", dtype="f16", bits=16, groups=2, beams=4, layers=2, kv_heads=2, dim=64,
             page=16, most=150, spare=10),
        # 64 requests of eight beams: 192 beams take a copy of their parent's partial page, 8 layers in 8 bits.
        dict(name="reorder_512", kind="reorder", dtype="bf16", bits=8, groups=64, beams=8, layers=8, kv_heads=8,
             dim=128, page=16, most=2048, spare=300),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "read", "attend", "attend", "attend", "select", "select", "reorder"])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "f16"]))
    if kind == "select":
        rows = _log(rng, 1, 512)
        c["dtype"] = rng.choice(["bf16", "f16", "f32"])
        c["beams"] = rng.choice([1, 2, 3, 4, 5, 8, 8, 16])
        c["groups"] = max(1, rows // c["beams"])
        c["picks"] = min(64, c["beams"] * rng.choice([1, 2, 2, 3]))
        return dict(c, vocab=_log(rng, 200, 131072 if c["dtype"] != "f32" else 65536), done=rng.choice([0, 0, 1]),
                    masked=rng.choice([0.0, 0.0, 0.5, 0.999]), first=rng.choice([0, 0, 0, 1]))
    c["dim"], c["page"] = rng.choice([64, 128, 128]), rng.choice([8, 16, 16, 32, 64])
    c["kv_heads"] = rng.choice([1, 2, 3, 4, 8, 8])
    if kind == "reorder":
        c["layers"] = rng.randint(1, min(8, 128 // c["page"]))
        c["beams"] = rng.choice([1, 2, 3, 4, 5, 8, 16])
        return dict(c, bits=rng.choice([8, 8, 16]), groups=_log(rng, 1, 512 // c["beams"]), most=_log(rng, 20, 2048),
                    spare=_log(rng, 4, 300))
    c["fused"] = rng.choice([0, 1])
    if kind in ("write", "read"):
        return dict(c, seqs=_log(rng, 1, 64 if kind == "read" else 24), mix=rng.choice(["one", "two"]),
                    median=_log(rng, 1, 700), q_most=rng.choice([1, 1, 5, MAX_LEN]))
    c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 3, 4, 4, 5, 7, 8])
    form = rng.choice(["one", "one", "few", "beams", "chunk", "window"])
    c.update(window=0, sinks=0, beams=1, q_most=1, mix="one")
    if form == "beams":
        return dict(c, beams=rng.choice([2, 4, 5, 8]), seqs=_log(rng, 1, 32), median=_log(rng, 16, 2000))
    if form == "chunk":
        return dict(c, seqs=_log(rng, 1, 12), median=_log(rng, 16, 5000), q_most=rng.choice([33, 100, 512]))
    if form == "few":
        return dict(c, seqs=_log(rng, 1, 64), median=_log(rng, 1, 3000), q_most=rng.choice([2, 5]))
    c["seqs"], c["median"], c["mix"] = _log(rng, 1, 256), _log(rng, 1, 2000), rng.choice(["one", "two"])
    if form == "window" or c["mix"] == "two":
        c["window"], c["sinks"] = _log(rng, 32, 4096), rng.choice([0, 1, 4, 64])
    return c


def _lognormal(n, median, sigma, lo, hi):
    normal = statistics.NormalDist()
    return [int(min(hi, max(lo, round(math.exp(math.log(median) + sigma * normal.inv_cdf((i + 0.5) / n))))))
            for i in range(n)]


def _lengths(c):
    """The requests' tokens, the same multiset for every seed."""
    n = c["seqs"]
    if c["mix"] == "two":
        long = max(1, n // 5)
        return _lognormal(max(0, n - long), c["median"], 0.6, 1, 2048) + _lognormal(long, 6000, 0.4, 2048, MAX_LEN)
    return _lognormal(n, c["median"], 0.3, 1, MAX_LEN)


def _own(c):
    """A beam's own tokens behind its request's prompt."""
    return [1 + 7 * (i % 9) for i in range(c["seqs"] * c["beams"])]


def _q_lens(c, lengths):
    """New tokens of each sequence: 1 .. q_most, at most the sequence's own tokens."""
    return [min(n, 1 + i % c["q_most"] if c["q_most"] <= 8 else c["q_most"]) for i, n in enumerate(lengths)]


def _distinct(c):
    """Beams of a request that live on: the others' places go to copies of these."""
    return max(1, (5 * c["beams"] + 7) // 8)


def work(c):
    if c["kind"] == "select":
        rows = c["groups"] * c["beams"]
        return {"bytes": float(rows * c["vocab"] * SIZES[c["dtype"]] + 8 * rows + 12 * c["groups"] * c["picks"]),
                "flops": 0.0}
    if c["kind"] == "reorder":
        page = 2 * c["layers"] * c["kv_heads"] * c["page"] * (c["dim"] * c["bits"] // 8 + (c["bits"] == 8))
        copies = c["groups"] * (c["beams"] - _distinct(c))
        return {"bytes": 2.0 * page * copies + 8 * c["groups"] * c["beams"], "flops": 0.0}
    lengths = _lengths(c)
    wide, coded = 2 * c["kv_heads"] * c["dim"] * 2, 2 * c["kv_heads"] * (c["dim"] + 1)  # bytes of a token
    if c["kind"] == "write":
        return {"bytes": float(sum(_q_lens(c, lengths)) * 2 * (wide + coded)), "flops": 0.0}
    if c["kind"] == "read":
        return {"bytes": float(sum(lengths) * (wide + coded)), "flops": 0.0}
    rows, pairs = sum(lengths), 0
    if c["beams"] > 1:
        own_lens, q = _own(c), [1] * (c["seqs"] * c["beams"])
        rows += sum(own_lens)
        pairs = c["beams"] * sum(lengths) + sum(own_lens)
    else:
        q, W, S = _q_lens(c, lengths), c["window"] or MAX_LEN, c["sinks"]
        rows = 0
        for n, k in zip(lengths, q):
            p = np.arange(n - k, n, dtype=np.int64)
            first = np.maximum(0, p - W + 1)
            pairs += int(np.sum(p + 1 - first + np.minimum(S, first)))
            rows += n - int(first[0]) + min(S, int(first[0]))
    size = c["q_heads"] * c["dim"] * 2
    return {"bytes": float(rows * coded + sum(q) * (2 * size + 4 * c["q_heads"])),
            "flops": 4.0 * c["dim"] * c["q_heads"] * pairs}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _pages_of(tokens, page):
    return -(-tokens // page)


def _ints(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def _tokens(c, gen, *shape):
    # keys and values of a trained model: near normal, a few channels several times larger
    x = torch.randn((*shape, c["dim"]), generator=gen, device="cuda", dtype=DTYPES[c["dtype"]])
    x[..., :: 16] *= 3
    return x


def _block(c):
    """Bytes of a page's keys or values in 8 bits: the codes, the scales, room up to a multiple of 16."""
    return (c["kv_heads"] * c["page"] * (c["dim"] + 1) + 15) // 16 * 16


def _codes(c, data):
    """The codes [layer][keys, values][page][head][token][dim] that the bytes of a pool hold."""
    n = c["kv_heads"] * c["page"] * c["dim"]
    return data[..., :n].view(torch.float8_e4m3fn).unflatten(-1, (c["kv_heads"], c["page"], c["dim"]))


def _scales(c, data):
    """The scales' exponents + 127 [layer][keys, values][page][head][token]."""
    n = c["kv_heads"] * c["page"]
    return data[..., n * c["dim"]:n * (c["dim"] + 1)].unflatten(-1, (c["kv_heads"], c["page"]))


def _data(c, gen, pages):
    layers = c.get("layers", 1)
    if c.get("bits", 8) == 16:
        return _tokens(c, gen, layers, 2, pages, c["kv_heads"], c["page"])
    data = torch.zeros((layers, 2, pages, _block(c)), dtype=torch.uint8, device="cuda")
    for plane in data.flatten(0, 1):
        code, scale = _quantise(c, _tokens(c, gen, pages, c["kv_heads"], c["page"]))
        _codes(c, plane).copy_(code)
        _scales(c, plane).copy_(scale)
    return data


def prepare(case, seed):
    rng = np.random.Generator(np.random.PCG64(seed))
    gen = torch.Generator("cuda").manual_seed(seed)
    s = dict(case=case)
    {"select": _prepare_select, "reorder": _prepare_reorder}.get(case["kind"], _prepare_rows)(case, rng, gen, s)
    if own:
        from paper_2601_21758_amd import ewsjf, kv
        s["ws"] = ewsjf.Workspace()
        if case["kind"] != "select":
            books = (s["data"], s["refs"], s["table"], s["length"])
            s["cache"] = kv.PagedCache.of(*books) if case.get("bits", 8) == 16 else kv.PagedCache.of_bytes(
                *books, case["page"], case["kv_heads"], case["dim"], dtype=DTYPES[case["dtype"]])
        if case["kind"] == "attend":  # lengths are common to all layers of a step: one plan serves them all
            sizes = dict(total_q=s["total_q"], max_q=s["max_q"], q_heads=case["q_heads"])
            if case["window"]:
                s["plan"] = kv.window_plan(s["cache"], s["slot"], s["q_start"], case["window"], case["sinks"], **sizes)
            else:
                s["plan"] = kv.prefix_plan(s["cache"], s["slot"], s["q_start"], s["group_start"], s["shared"], **sizes)
    return s


def _prepare_rows(c, rng, gen, s):
    """Sequences whose pages lie anywhere in the pool; a request's beams have its prompt's whole pages in common."""
    ps, B = c["page"], c.get("beams", 1)
    prompt = rng.permutation(np.asarray(_lengths(c)))
    if B > 1:
        own_lens = rng.permutation(np.asarray(_own(c)))
        n, shared, q_lens = own_lens.size, prompt, np.ones(own_lens.size, np.int64)
    else:
        own_lens = np.sort(prompt)
        q_lens = np.asarray(_q_lens(c, own_lens.tolist()))
        order = rng.permutation(own_lens.size)
        own_lens, q_lens = own_lens[order], q_lens[order]
        n, shared = own_lens.size, np.zeros(own_lens.size, np.int64)
    group = np.arange(n) // B
    length = own_lens + shared[group]
    width = _pages_of(int(length.max()), ps)
    # whole pages are shared; the prompt's last, partial page is each beam's own copy, as a fork leaves it
    whole = shared // ps
    private = -(-length // ps) - whole[group]
    pages = int(private.sum() + whole.sum())
    at = rng.permutation(pages).astype(np.int32)
    table = np.full((n, width), -1, np.int32)
    heads, o = [], 0
    for w in whole:
        heads.append(at[o:o + w])
        o += w
    for i in range(n):
        w = whole[group[i]]
        table[i, :w] = heads[group[i]]
        table[i, w:w + private[i]] = at[o:o + private[i]]
        o += private[i]
    slot = rng.permutation(n)
    held, lens = np.empty_like(table), np.empty_like(length)
    held[slot], lens[slot] = table, length
    q_start = np.concatenate([[0], np.cumsum(q_lens)])
    total = int(q_start[-1])
    s.update(data=_data(c, gen, pages), refs=_ints(np.bincount(held[held >= 0], minlength=pages)), table=_ints(held),
             length=_ints(lens), slot=_ints(slot), q_start=_ints(q_start), total_q=total, max_q=int(q_lens.max()),
             scale=c["dim"] ** -0.5, group_start=None, shared=None)
    if c["kind"] == "read":
        s["start"], s["total"] = _ints(np.concatenate([[0], np.cumsum(length)])), int(length.sum())
        return
    if c["kind"] == "write":
        s["begin"] = _ints(length - q_lens)
        heads = 2 * c["kv_heads"] if c["fused"] else c["kv_heads"]
        both = [_tokens(c, gen, total, heads) for _ in range(1 if c["fused"] else 2)]
        s["k"], s["v"] = both[0].split(c["kv_heads"], 1) if c["fused"] else both
        return
    if B > 1:
        s.update(group_start=_ints(np.arange(c["seqs"] + 1) * B), shared=_ints(whole * ps))
        for g in range(c["seqs"]):  # the partial pages hold the same tokens
            rest = int(shared[g] - whole[g] * ps)
            if rest:
                member = torch.as_tensor(table[group == g, whole[g]], device="cuda", dtype=torch.long)
                for x in (_codes(c, s["data"]).view(torch.uint8), _scales(c, s["data"])):
                    x[:, :, member, :, :rest] = x[:, :, member[:1], :, :rest]
    heads = c["q_heads"] + (2 * c["kv_heads"] if c["fused"] else 0)
    q = torch.randn((total, heads, c["dim"]), generator=gen, device="cuda", dtype=DTYPES[c["dtype"]])
    s["q"] = q[:, :c["q_heads"]]


def _prepare_select(c, rng, gen, s):
    """Logits of a trained model: a broad bulk, a few tokens far above it; masked: tokens that a grammar forbids."""
    rows, V = c["groups"] * c["beams"], c["vocab"]
    x = torch.randn((rows, V), generator=gen, device="cuda") * 2.5
    likely = torch.randint(0, V, (rows, min(V, 20)), generator=gen, device="cuda")
    x.scatter_add_(1, likely, torch.rand(likely.shape, generator=gen, device="cuda") * 9 + 3)
    if c["masked"]:
        forbidden = torch.rand((c["groups"], 1, V), generator=gen, device="cuda") < c["masked"]
        x.view(c["groups"], c["beams"], V).masked_fill_(forbidden, -math.inf)
    s["logits"] = x.to(DTYPES[c["dtype"]])
    score = -rng.random(rows) * 20
    if c["first"]:  # the first step: all beams are the prompt itself, and one of them counts
        score = np.where(np.arange(rows) % c["beams"] == 0, 0.0, -math.inf)
    s["score"] = torch.tensor(score, dtype=torch.float32, device="cuda")
    s["done"] = _ints(rng.random(rows) < 0.2) if c["done"] else None
    s["end"] = V // 3


def _prepare_reorder(c, rng, gen, s):
    """A request's beams share its prompt's whole pages and have a few pages of their own, the last one partial."""
    ps, G, B = c["page"], c["groups"], c["beams"]
    prompt = rng.permutation(np.linspace(max(1, c["most"] // 2), c["most"], G).astype(np.int64)) // ps
    n, tail = G * B, 3
    length = (prompt.repeat(B) + tail - 1) * ps + 1 + np.repeat(np.arange(G) % max(1, ps - 1), B)
    width = int(prompt.max()) + tail + 1
    used = int(prompt.sum()) + n * tail
    pages = used + c["spare"]
    at = rng.permutation(pages)[:used]
    table, o = np.full((n, width), -1, np.int32), 0
    for g in range(G):
        common, o = at[o:o + prompt[g]], o + prompt[g]
        for b in range(g * B, (g + 1) * B):
            table[b, :prompt[g]] = common
            table[b, prompt[g]:prompt[g] + tail] = at[o:o + tail]
            o += tail
    slot = rng.permutation(n)
    held, lens = np.empty_like(table), np.empty_like(length)
    held[slot], lens[slot] = table, length
    live = _distinct(c)
    parent = np.concatenate([g * B + rng.permutation(B)[rng.permutation(
        np.concatenate([np.arange(live), rng.integers(0, live, B - live)]))] for g in range(G)])
    s.update(data=_data(c, gen, pages), refs=_ints(np.bincount(held[held >= 0], minlength=pages)), table=_ints(held),
             length=_ints(lens), slot=_ints(slot), parent=_ints(parent))


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    return {"write": _run_write, "read": _run_read, "attend": _run_attend, "select": _run_select,
            "reorder": _run_reorder}[s["case"]["kind"]](s)


def _run_write(s):
    """The new tokens go into their pages, and what the pages now stand for comes back."""
    c = s["case"]
    if own:
        s["cache"].append(0, s["k"], s["v"], s["slot"], s["q_start"])
        k, v = s["cache"].read(0, s["slot"], s["q_start"], s["begin"], total=s["total_q"])
    else:
        _plain_write(s)
        k, v = _plain_read(s, s["q_start"], s["begin"], s["total_q"])
    return dict(k=k, v=v, code=_codes(c, s["data"]), scale=_scales(c, s["data"]))


def _run_read(s):
    if own:
        k, v = s["cache"].read(0, s["slot"], s["start"], total=s["total"])
    else:
        k, v = _plain_read(s, s["start"], torch.zeros_like(s["slot"]), s["total"])
    return dict(k=k, v=v)


def _run_attend(s):
    if own:
        from paper_2601_21758_amd import kv
        out, lse = kv.attention(s["q"], s["cache"], 0, s["plan"], scale=s["scale"], ws=s["ws"])
    else:
        out, lse = _plain_attend(s)
    return dict(out=out, lse=lse)


def _run_select(s):
    c = s["case"]
    if own:
        from paper_2601_21758_amd import beam
        parent, token, score = beam.beam_select(s["logits"], s["score"], c["beams"], c["picks"], done=s["done"],
                                                end=s["end"], ws=s["ws"])
    else:
        parent, token, score = _plain_select(s)
    return dict(parent=parent, token=token, score=score)


def _run_reorder(s):
    c = s["case"]
    granted = s["cache"].reorder(s["slot"], s["parent"], ws=s["ws"]) if own else _plain_reorder(s)
    books = dict(refs=s["refs"], table=s["table"], length=s["length"], granted=granted)
    if c["bits"] == 16:
        return dict(books, data=s["data"])
    return dict(books, code=_codes(c, s["data"]), scale=_scales(c, s["data"]))


# ---------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------
def _quantise(c, x):
    """Codes and exponents + 127 of x [..][dim]."""
    x = x.float().clamp(-MOST[c["dtype"]], MOST[c["dtype"]])
    top = x.abs().nan_to_num(0.0).amax(-1)
    part, exp = torch.frexp(top)  # top = part 2^exp, part in [0.5, 1); 448 = 0.875 2^9
    exp = torch.where(top > 0, exp - 9 + (part > 0.875), LEAST_EXP).clamp(min=LEAST_EXP)
    return torch.ldexp(x, -exp[..., None]).to(torch.float8_e4m3fn), (exp + 127).to(torch.uint8)


def _values(code, scale):
    """What codes [..][dim] with exponents + 127 [..] stand for, in 32 bits."""
    return torch.ldexp(code.float(), scale.int()[..., None] - 127)


def _plain_write(s):
    c, ps = s["case"], s["case"]["page"]
    q_start = s["q_start"].long()
    n = torch.repeat_interleave(torch.arange(s["slot"].numel(), device="cuda"), q_start[1:] - q_start[:-1],
                                output_size=s["total_q"])
    pos = s["begin"].long()[n] + torch.arange(s["total_q"], device="cuda") - q_start[n]
    page = s["table"][s["slot"].long()[n], pos // ps].long()
    for plane, x in ((0, s["k"]), (1, s["v"])):
        code, scale = _quantise(c, x)
        _codes(c, s["data"]).view(torch.uint8)[0, plane][page, :, pos % ps] = code.view(torch.uint8)
        _scales(c, s["data"])[0, plane][page, :, pos % ps] = scale


def _plain_read(s, start, begin, total):
    c, ps, start = s["case"], s["case"]["page"], start.long()
    n = torch.repeat_interleave(torch.arange(s["slot"].numel(), device="cuda"), start[1:] - start[:-1],
                                output_size=total)
    pos = begin.long()[n] + torch.arange(total, device="cuda") - start[n]
    page = s["table"][s["slot"].long()[n], pos // ps].long()
    bytes_ = _codes(c, s["data"]).view(torch.uint8)
    return tuple(_values(bytes_[0, x][page, :, pos % ps].view(torch.float8_e4m3fn),
                         _scales(c, s["data"])[0, x][page, :, pos % ps]).to(DTYPES[c["dtype"]]) for x in (0, 1))


def _rows(s, plane, table, pos):
    """Keys or values at the positions pos of the rows of `table`, in 32 bits: [row][position][kv head][dim]."""
    c, page = s["case"], s["case"]["page"]
    at = torch.gather(table, 1, (pos // page).clamp(0, table.shape[1] - 1)).clamp(min=0).long()
    code = _codes(c, s["data"]).view(torch.uint8)[0, plane][at, :, pos % page].view(torch.float8_e4m3fn)
    return _values(code, _scales(c, s["data"])[0, plane][at, :, pos % page])


def _plain_attend(s):
    """Every sequence's visible keys beside its queries: softmax(scale q K^T) V."""
    c = s["case"]
    Hk, D, W, S, n = c["kv_heads"], c["dim"], c["window"], c["sinks"], s["slot"].numel()
    R, Q, dev = c["q_heads"] // c["kv_heads"], s["max_q"], "cuda"
    slot, q_start = s["slot"].long(), s["q_start"].long()
    q_len, length, table = q_start[1:] - q_start[:-1], s["length"][slot].long(), s["table"][slot]
    seq = torch.repeat_interleave(torch.arange(n, device=dev), q_len, output_size=s["total_q"])
    i = torch.arange(s["total_q"], device=dev) - q_start[seq]
    q = torch.zeros((n, Q, Hk, R, D), device=dev)
    q[seq, i] = s["q"].float().reshape(-1, Hk, R, D) * s["scale"]
    start = length - q_len
    if W:  # the window's span, and the sinks before it
        span = start[:, None] - W + 1 + torch.arange(W + Q - 1, device=dev)
        sink = torch.arange(S, device=dev).expand(n, S)
        pos = torch.cat([sink, span], 1)
        there = torch.cat([sink < span[:, :1], span >= 0], 1)
    else:
        pos = torch.arange(int(length.max()), device=dev).expand(n, -1)
        there = torch.ones_like(pos, dtype=torch.bool)
    p_at = start[:, None] + torch.arange(Q, device=dev)
    seen = (there & (pos < length[:, None]))[:, None] & (pos[:, None] <= p_at[..., None])
    if W:
        seen = seen & ((pos[:, None] > p_at[..., None] - W) | (pos[:, None] < S))
    k, v = (_rows(s, x, table, pos.clamp(min=0)).permute(0, 2, 1, 3).contiguous() for x in (0, 1))
    x = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(n, Hk, Q * R, D), k.transpose(-1, -2).contiguous())
    x = x.reshape(n, Hk, Q, R, -1).masked_fill_(~seen[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=FLOOR)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = torch.where(total > 0, top + total.log(), -math.inf).squeeze(-1)
    out = torch.matmul(p.reshape(n, Hk, Q * R, -1), v).reshape(n, Hk, Q, R, D) / torch.where(total > 0, total, 1.0)
    return (out.permute(0, 2, 1, 3, 4)[seq, i].reshape(-1, c["q_heads"], D).to(s["q"].dtype),
            lse.permute(0, 2, 1, 3)[seq, i].reshape(-1, c["q_heads"]))


def _plain_select(s):
    """A row's candidates by their logits (ties: the lower token), a group's by their scores (ties: the lower row)."""
    c = s["case"]
    G, B, K, V = c["groups"], c["beams"], c["picks"], c["vocab"]
    x, most = s["logits"].double(), min(c["picks"], c["vocab"])
    top = x.amax(1, keepdim=True)
    shift = torch.where(torch.isfinite(top), top, 0.0)
    total = (x - shift).exp_().sum(1)
    base = s["score"].double() - (shift[:, 0] + total.log())
    # one whole number for a candidate's place in its row: the logit's bits in the order of its values, then the token
    bits = s["logits"].float().view(torch.int32).long()
    bits = torch.where(bits < 0, -(bits & 0x7fffffff), bits)  # -0 counts as 0
    place = torch.topk((bits << 32) + (V - 1 - torch.arange(V, device="cuda")), most, dim=1).values
    token = (V - 1) - (place & 0xffffffff)
    score = base[:, None] + x.gather(1, token)
    if s["done"] is not None:  # a beam at its end goes on by the end token alone, at no cost
        done, first = (s["done"] != 0)[:, None], torch.arange(most, device="cuda") == 0
        score = torch.where(done, torch.where(first, s["score"].double()[:, None], -math.inf), score)
        token = torch.where(done & first, s["end"], token)
    score = torch.where(torch.isnan(score), -math.inf, score).view(G, B * most)
    value, at = torch.sort(score, dim=1, descending=True, stable=True)
    value, at = value[:, :K], at[:, :K]
    parent = at // most + torch.arange(G, device="cuda")[:, None] * B
    token = token.view(G, B * most).gather(1, at)
    if value.shape[1] < K:  # fewer candidates than asked for
        pad = (0, K - value.shape[1])
        value = torch.nn.functional.pad(value, pad, value=-math.inf)
        parent, token = torch.nn.functional.pad(parent, pad), torch.nn.functional.pad(token, pad)
    none = value == -math.inf
    return (torch.where(none, -1, parent).int(), torch.where(none, -1, token).int(), value.float())


def _plain_reorder(s):
    c, refs, table, length = s["case"], s["refs"], s["table"], s["length"]
    ps, slot, parent = c["page"], s["slot"].long(), s["parent"].long()
    n = slot.numel()
    me = torch.arange(n, device="cuda")
    # a parent's own row goes to itself, or else to the first that names it
    heir = torch.full((n,), n, device="cuda").scatter_reduce_(0, parent, me, "amin")
    heir = torch.where(parent == me, me, heir)
    rows, lens = table[slot], length[slot].long()
    gone = rows[heir == n]
    gone = gone[gone >= 0].long()
    refs.index_add_(0, gone, torch.full_like(gone, -1, dtype=torch.int32))
    last = (lens // ps)[parent]
    source = rows[parent].gather(1, last.clamp(max=rows.shape[1] - 1)[:, None])[:, 0].long()
    need = (heir[parent] != me) & ((lens % ps)[parent] > 0) & (source >= 0)
    free = torch.nonzero(refs == 0).flatten()
    ok = ~need | (torch.cumsum(need.long(), 0) <= free.numel())
    row = torch.where(torch.arange(rows.shape[1], device="cuda") < ((lens + ps - 1) // ps)[parent][:, None],
                      rows[parent], -1)
    copied = (need & ok).nonzero().flatten()
    taken = free[:copied.numel()]
    whole = row.clone()
    whole[need.nonzero().flatten(), last[need]] = -1
    whole = whole[ok & (heir[parent] != me)]
    whole = whole[whole >= 0].long()
    refs.index_add_(0, whole, torch.ones_like(whole, dtype=torch.int32))
    refs[taken] = 1
    row[copied, last[copied]] = taken.int()
    table[slot] = torch.where(ok[:, None], row, -1)
    length[slot] = torch.where(ok, lens[parent], 0).int()
    s["data"][:, :, taken] = s["data"][:, :, source[copied]]
    return ok.int()


# ---------------------------------------------------------------------------
# 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    """From the definitions in 64 bits; the reordering computes no numbers."""
    if case["kind"] == "reorder":
        return None
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    return {"write": _exact_write, "read": _exact_read, "attend": _exact_attend, "select": _exact_select}[case["kind"]](s)


def _stood_for(code, scale):
    """The values of a pool's codes in 64 bits, from the bits of the format: sign, four of exponent, three of mantissa."""
    b = code.view(torch.uint8).long()
    e, m = b >> 3 & 15, (b & 7).double()
    size = torch.where(e > 0, (8 + m) * torch.exp2((e - 10).double()), m * 2.0 ** -9)
    size = torch.where((b & 127) == 127, math.nan, size)
    return torch.where(b >= 128, -size, size) * torch.exp2(scale.double() - 127)[..., None]


def _request(s, x, r, n):
    """Keys or values [head][token][dim] of the first n tokens of slot r."""
    c = s["case"]
    at = s["table"][r, :_pages_of(n, c["page"])].long()
    y = _stood_for(_codes(c, s["data"])[0, x].view(torch.uint8)[at], _scales(c, s["data"])[0, x][at])
    return y.permute(1, 0, 2, 3).reshape(c["kv_heads"], -1, c["dim"])[:, :n]


def _exact_write(s):
    c, got = s["case"], []
    for x in (s["k"], s["v"]):
        y = x.double().cpu().numpy()
        y = np.clip(y, -MOST[c["dtype"]], MOST[c["dtype"]])
        top = np.max(np.abs(np.nan_to_num(y, nan=0.0)), -1, keepdims=True)
        exp = np.maximum(np.ceil(np.log2(np.maximum(top, 2.0 ** -200) / 448)), LEAST_EXP)
        # the format's numbers near a value lie 2^-3 of its power of two apart, 2^-9 at the least
        y = y / 2.0 ** exp
        step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -30))), -6) - 3)
        got.append(torch.tensor(np.rint(y / step) * step * 2.0 ** exp))
    return dict(k=got[0], v=got[1], code=None, scale=None)


def _exact_read(s):
    lens = s["length"].tolist()
    k, v = (torch.cat([_request(s, x, r, lens[r]).transpose(0, 1) for r in s["slot"].tolist()]) for x in (0, 1))
    return dict(k=k, v=v)


def _exact_attend(s):
    c = s["case"]
    Hk, D, R = c["kv_heads"], c["dim"], c["q_heads"] // c["kv_heads"]
    starts, slots, lengths = (s[x].tolist() for x in ("q_start", "slot", "length"))
    out = torch.zeros((s["total_q"], c["q_heads"], D), dtype=torch.float64, device="cuda")
    lse = torch.full((s["total_q"], c["q_heads"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, r in enumerate(slots):
        n, a, e = lengths[r], starts[b], starts[b + 1]
        keys, values = (_request(s, x, r, n) for x in (0, 1))
        for at in range(a, e, 256):
            stop = min(e, at + 256)
            p = torch.arange(n - e + at, n - e + stop, device="cuda")
            lo = max(0, int(p[0]) - c["window"] + 1) if c["window"] else 0
            j = torch.cat([torch.arange(min(lo, c["sinks"]), device="cuda"),
                           torch.arange(lo, int(p[-1]) + 1, device="cuda")])
            seen = j <= p[:, None]
            if c["window"]:
                seen = seen & ((j > p[:, None] - c["window"]) | (j < c["sinks"]))
            q = s["q"][at:stop].double().reshape(-1, Hk, R, D).permute(1, 2, 0, 3)
            x = torch.matmul(q, keys[:, None, j].transpose(-1, -2)) * s["scale"]
            z = torch.logsumexp(x.masked_fill(~seen, -math.inf), -1)
            w = torch.where(seen, torch.exp(x - z[..., None]), 0.0)
            out[at:stop] = torch.matmul(w, values[:, None, j]).permute(2, 0, 1, 3).reshape(stop - at, -1, D)
            lse[at:stop] = z.permute(2, 0, 1).reshape(stop - at, -1)
    return dict(out=out, lse=lse)


def _exact_select(s):
    c = s["case"]
    G, B, K, V = c["groups"], c["beams"], c["picks"], c["vocab"]
    score = torch.full((G, K), -math.inf, dtype=torch.float64, device="cuda")
    for g in range(G):
        rows = slice(g * B, (g + 1) * B)
        x = s["logits"][rows].double()
        z = s["score"][rows].double()[:, None] + x - torch.logsumexp(x, 1, keepdim=True)
        if s["done"] is not None:
            ends = torch.full_like(z, -math.inf)
            ends[:, s["end"]] = s["score"][rows].double()
            z = torch.where((s["done"][rows] != 0)[:, None], ends, z)
        z = torch.where(torch.isnan(z), -math.inf, z).flatten()
        score[g, :min(K, B * V)] = torch.topk(z, min(K, B * V)).values
    return dict(parent=None, token=None, score=score)
