"""The workloads the cache and attention operators' speed is measured on.

Three operators that a server calls with the requests the scheduler admitted:

  pages   the paged key/value cache's bookkeeping: slots released, forked from
          a parent (a prompt's pages shared, its partial page copied),
          extended by new tokens, the new tokens' keys and values written; and
          the pool compacted (used pages moved to the front);
  prefix  attention of a batch whose sequences share a long prefix;
  window  attention with a sliding window and a few first tokens (sinks) that
          stay visible.

Prompt lengths follow the framework's workloads: short ones lognormal(ln 128,
0.6), long ones lognormal(ln 6000, 0.4), 80 to 20, up to 32,768 tokens; batch
sizes are its admissions per step (64 to 512); 40 heads of 128 are those of
the model its evaluation names.  Lengths are the quantiles of the
distribution, in an order drawn from the seed, so a case's work is known.

Where `own` is false `run` evaluates the definitions with elementary torch
operations in 32 bits; where it is true it makes the framework's calls.
"""
from __future__ import annotations

import math
import statistics

import numpy as np
import torch

own = False

MAX_LEN = 32768
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
FLOOR = -3e38  # the running maximum of a row that has seen no key


# ---------------------------------------------------------------------------
# Cases
# ---------------------------------------------------------------------------
def listed():
    return [
        # Parallel samples of one short prompt on a small model: eight forks, one new token each (latency).
        dict(name="fork_8", kind="fork", dtype="f16", layers=2, kv_heads=2, dim=64, page=16, parents=1, children=8,
             most=100, new=1, spare=40),
        # A large step's admissions forked from eight system prompts, half of them at the prompt's end, one new token.
        dict(name="fork_512", kind="fork", dtype="bf16", layers=8, kv_heads=8, dim=128, page=16, parents=8,
             children=512, most=2048, new=1, spare=1500),
        # An odd number of small pages, more than half of them in use: the everyday clean-up of a small pool.
        dict(name="compact_1k", kind="compact", dtype="f16", layers=2, kv_heads=3, dim=64, page=16, pages=1021,
             used=0.6, slots=37),
        # A large pool after many requests have left: 40 percent in use, a thousand pages of 512 KiB move.
        dict(name="compact_4k", kind="compact", dtype="bf16", layers=8, kv_heads=8, dim=128, page=16, pages=4096,
             used=0.4, slots=256),
        # Four sequences behind a short common prompt, small heads: a single user's parallel samples (latency).
        dict(name="prefix_4", kind="prefix", dtype="f16", groups=1, members=4, q_most=1, q_heads=8, kv_heads=2, dim=64,
             page=16, shared_least=300, shared_most=300, own=24, fused=0),
        # 64 admissions behind one system prompt, every head with its own keys (40 heads of 128).
        dict(name="prefix_64_mha", kind="prefix", dtype="bf16", groups=1, members=64, q_most=1, q_heads=40,
             kv_heads=40, dim=128, page=16, shared_least=2048, shared_most=2048, own=128, fused=0),
        # Three services of 21 requests each, up to five draft tokens a request, five query heads to a key head,
        # queries as a slice of the fused projection.
        dict(name="prefix_groups", kind="prefix", dtype="f16", groups=3, members=21, q_most=5, q_heads=15, kv_heads=3,
             dim=64, page=32, shared_least=500, shared_most=4001, own=128, fused=1),
        # 512 admissions that answer questions on one long document.
        dict(name="prefix_512_long", kind="prefix", dtype="bf16", groups=1, members=512, q_most=1, q_heads=32,
             kv_heads=8, dim=128, page=16, shared_least=16123, shared_most=16123, own=128, fused=0),
        # Three sequences, one key head, a short window: the smallest decoding step (latency).
        dict(name="window_3", kind="window", dtype="f16", seqs=3, mix="one", median=1000, q_most=1, q_heads=8,
             kv_heads=1, dim=64, page=16, window=128, sinks=4, fused=0),
        # The decoding step of 256 requests of both length modes, window 4,096.
        dict(name="window_256", kind="window", dtype="bf16", seqs=256, mix="two", median=128, q_most=1, q_heads=32,
             kv_heads=8, dim=128, page=16, window=4096, sinks=4, fused=0),
        # 24 whole prompts of both length modes prefilled in one ragged batch.
        dict(name="window_ragged", kind="window", dtype="f16", seqs=24, mix="two", median=128, q_most=MAX_LEN,
             q_heads=20, kv_heads=4, dim=64, page=32, window=1024, sinks=16, fused=1),
        # One long prompt, 40 heads of 128, window 4,096: the largest product.
        dict(name="window_16k", kind="window", dtype="bf16", seqs=1, mix="one", median=16384, q_most=MAX_LEN,
             q_heads=40, kv_heads=40, dim=128, page=16, window=4096, sinks=4, fused=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["fork", "compact", "prefix", "prefix", "window", "window"])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "f16"]), dim=rng.choice([64, 128, 128]),
             page=rng.choice([8, 16, 16, 32, 64]))
    if kind in ("fork", "compact"):
        c["layers"], c["kv_heads"] = rng.randint(1, min(8, 128 // c["page"])), rng.randint(1, 8)
        if kind == "fork":
            c["parents"] = rng.randint(1, 8)
            return dict(c, children=_log(rng, c["parents"], 512), most=_log(rng, 20, 2048), new=rng.choice([1, 1, 4, 17]),
                        spare=_log(rng, 8, 1500))
        return dict(c, pages=max(64, min(4096, _log(rng, 64, 4096) * 16 // c["page"])), used=rng.choice([0.1, 0.4, 0.6, 0.9]),
                    slots=_log(rng, 2, 256))
    c["kv_heads"] = rng.choice([1, 2, 3, 4, 8, 8])
    c["q_heads"] = c["kv_heads"] * rng.choice([1, 2, 4, 4, 5, 7, 8])
    c["fused"] = rng.choice([0, 1])
    if kind == "prefix":
        c["groups"] = rng.choice([1, 1, 2, 3])
        most = _log(rng, 16, 16000 // c["groups"])
        return dict(c, members=max(1, _log(rng, 1, 400 // c["groups"])), q_most=rng.choice([1, 1, 1, 2, 5]),
                    shared_least=max(1, most // rng.choice([1, 2, 8])), shared_most=most, own=_log(rng, 4, 300))
    c["window"], c["sinks"] = _log(rng, 32, 4096), rng.choice([0, 1, 4, 4, 64])
    if rng.random() < 0.5:  # decoding
        return dict(c, seqs=_log(rng, 1, 256), mix=rng.choice(["one", "two"]), median=_log(rng, 16, 6000),
                    q_most=rng.choice([1, 1, 1, 2, 5]))
    c["window"] = min(c["window"], 1024)
    return dict(c, seqs=_log(rng, 1, 24), mix="one", median=_log(rng, 16, 700), q_most=rng.choice([100, 512, MAX_LEN]))


def _lognormal(n, median, sigma, lo, hi):
    normal = statistics.NormalDist()
    return [int(min(hi, max(lo, round(math.exp(math.log(median) + sigma * normal.inv_cdf((i + 0.5) / n))))))
            for i in range(n)]


def _lengths(c):
    """The case's lengths, the same multiset for every seed: window sequences' tokens, prefix sequences' own tokens."""
    if c["kind"] == "prefix":
        return _lognormal(c["groups"] * c["members"], c["own"], 0.6, 1, 2048)
    n = c["seqs"]
    if c["mix"] == "two":
        long = max(1, n // 5)
        return _lognormal(n - long, c["median"], 0.6, 1, 2048) + _lognormal(long, 6000, 0.4, 2048, MAX_LEN)
    return _lognormal(n, c["median"], 0.3, 1, MAX_LEN)


def _shared(c):
    g = c["groups"]
    return [c["shared_most"] if g == 1 else
            round(c["shared_least"] + (c["shared_most"] - c["shared_least"]) * i / (g - 1)) for i in range(g)]


def _q_lens(c, lengths):
    """Query tokens of each sequence, shortest sequence first: 1 .. q_most, at most the sequence's own tokens."""
    return [min(n, 1 + i % c["q_most"] if c["q_most"] <= 8 else c["q_most"]) for i, n in enumerate(lengths)]


def work(c):
    planes = 2 * c.get("layers", 1)
    if c["kind"] == "fork":
        page = planes * c["kv_heads"] * c["page"] * c["dim"] * 2
        # nearly every child has a partial page, as far as the pool reaches; tables and counts are small
        done = min(c["children"], c["spare"])
        return {"bytes": 2.0 * page * done + 8.0 * c["kv_heads"] * c["dim"] * done * c["new"], "flops": 0.0}
    if c["kind"] == "compact":
        page = planes * c["kv_heads"] * c["page"] * c["dim"] * 2
        return {"bytes": 2.0 * page * c["pages"] * c["used"] * (1 - c["used"]) + 8 * c["pages"], "flops": 0.0}
    lengths = _lengths(c)
    q = _q_lens(c, lengths)
    rows, pairs = sum(lengths), 0
    if c["kind"] == "prefix":
        shared = _shared(c)
        rows += sum(shared)
        # every group has members of all own lengths; the mean prefix stands for each
        pairs = sum(k * sum(shared) / c["groups"] + k * n - k * (k - 1) / 2 for n, k in zip(lengths, q))
    else:
        W, S, rows = c["window"], c["sinks"], 0
        for n, k in zip(lengths, q):
            p = np.arange(n - k, n, dtype=np.int64)
            first = np.maximum(0, p - W + 1)
            pairs += int(np.sum(p + 1 - first + np.minimum(S, first)))
            rows += n - int(first[0]) + min(S, int(first[0]))
    size = c["q_heads"] * c["dim"] * 2
    return {"bytes": float(2 * rows * c["kv_heads"] * c["dim"] * 2 + sum(q) * (2 * size + 4 * c["q_heads"])),
            "flops": 4.0 * c["dim"] * c["q_heads"] * pairs}


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _pages_of(tokens, page):
    return -(-tokens // page)


def _ints(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def _data(c, gen, pages):
    # keys and values of a trained model: near normal, a few channels several times larger
    shape = (c.get("layers", 1), 2, pages, c["kv_heads"], c["page"], c["dim"])
    x = torch.randn(shape, generator=gen, device="cuda", dtype=DTYPES[c["dtype"]])
    x[:, 0, ..., :: 16] *= 3
    return x


def prepare(case, seed):
    rng = np.random.Generator(np.random.PCG64(seed))
    gen = torch.Generator("cuda").manual_seed(seed)
    s = dict(case=case)
    {"fork": _prepare_fork, "compact": _prepare_compact}.get(case["kind"], _prepare_attention)(case, rng, gen, s)
    if own:
        from paper_2601_21758_amd import kv
        s["cache"] = kv.PagedCache.of(s["data"], s["refs"], s["table"], s["length"])
        s["ws"] = kv.Workspace()
        if case["kind"] == "prefix":  # lengths are common to all layers of a step: one plan serves them all
            s["plan"] = kv.prefix_plan(s["cache"], s["slot"], s["q_start"], s["group_start"], s["shared"],
                                       total_q=s["total_q"], max_q=s["max_q"], q_heads=case["q_heads"])
        elif case["kind"] == "window":
            s["plan"] = kv.window_plan(s["cache"], s["slot"], s["q_start"], case["window"], case["sinks"],
                                       total_q=s["total_q"], max_q=s["max_q"], q_heads=case["q_heads"])
    return s


def _prepare_fork(c, rng, gen, s):
    """Parents with their pages somewhere in the pool, children empty; the pool has `spare` pages beyond the parents'."""
    ps, P, n = c["page"], c["parents"], c["children"]
    top = rng.permutation(np.linspace(max(1, c["most"] // 2), c["most"], P).astype(np.int64))
    width = _pages_of(c["most"] + c["new"], ps) + 1
    used = sum(_pages_of(int(t), ps) for t in top)
    pages = used + c["spare"]
    at = rng.permutation(pages)[:used]
    table = np.full((P + n, width), -1, np.int32)
    o = 0
    for i, t in enumerate(top):
        k = _pages_of(int(t), ps)
        table[i, :k] = at[o:o + k]
        o += k
    refs = np.zeros(pages, np.int32)
    refs[at] = 1
    parent = np.sort(rng.integers(0, P, n))
    tokens = np.where(rng.random(n) < 0.5, top[parent], np.maximum(1, (top[parent] * rng.random(n)).astype(np.int64)))
    s.update(data=_data(c, gen, pages), refs=_ints(refs), table=_ints(table),
             length=_ints(np.concatenate([top, np.zeros(n, np.int64)])), parent=_ints(parent),
             child=_ints(P + rng.permutation(n)), tokens=_ints(tokens), new=_ints(np.full(n, c["new"])),
             q_start=_ints(np.arange(n + 1) * c["new"]))
    shape = (n * c["new"], c["kv_heads"], c["dim"])
    s["k"], s["v"] = (torch.randn(shape, generator=gen, device="cuda", dtype=DTYPES[c["dtype"]]) for _ in range(2))


def _prepare_compact(c, rng, gen, s):
    """Used pages anywhere in the pool, one in ten in two rows; every used page is in a row."""
    n, used = c["pages"], max(1, int(c["pages"] * c["used"]))
    at = rng.permutation(n)[:used]
    twice = rng.choice(at, used // 10, replace=False)
    every = np.concatenate([at, twice])
    row = rng.permutation(every.size) % c["slots"]
    width = int(np.bincount(row, minlength=c["slots"]).max()) + 1
    table = np.full((c["slots"], width), -1, np.int32)
    fill = np.zeros(c["slots"], np.int64)
    for p, r in zip(every, row):
        table[r, fill[r]] = p
        fill[r] += 1
    s.update(data=_data(c, gen, n), refs=_ints(np.bincount(every, minlength=n)), table=_ints(table),
             length=_ints(fill * c["page"]), out_table=torch.empty_like(_ints(table)),
             out_refs=torch.empty(n, dtype=torch.int32, device="cuda"),
             used=torch.empty(1, dtype=torch.int32, device="cuda"))


def _prepare_attention(c, rng, gen, s):
    """Sequences whose pages lie anywhere in the pool; a group's shared pages are in every member's row."""
    ps, own_lens = c["page"], _lengths(c)
    q_lens = _q_lens(c, own_lens)
    n = len(own_lens)
    order = rng.permutation(n)
    own_lens, q_lens = np.asarray(own_lens)[order], np.asarray(q_lens)[order]
    group = np.repeat(np.arange(c["groups"]), c["members"]) if c["kind"] == "prefix" else np.zeros(n, np.int64)
    shared = np.asarray(_shared(c) if c["kind"] == "prefix" else [0])
    length = own_lens + shared[group]
    width = _pages_of(int(length.max()), ps)
    # whole pages are shared; the prefix's last, partial page is each member's own copy, as a fork leaves it
    whole = shared // ps
    private = -(-length // ps) - whole[group]
    pages = int(private.sum() + whole.sum())
    at = rng.permutation(pages).astype(np.int32)
    table = np.full((n, width), -1, np.int32)
    heads, o = [], 0
    for g in range(whole.size):
        heads.append(at[o:o + whole[g]])
        o += whole[g]
    for i in range(n):
        w = whole[group[i]]
        table[i, :w] = heads[group[i]]
        table[i, w:w + private[i]] = at[o:o + private[i]]
        o += private[i]
    slot = rng.permutation(n)
    held = np.empty_like(table)
    held[slot] = table
    lens = np.empty_like(length)
    lens[slot] = length
    q_start = np.concatenate([[0], np.cumsum(q_lens)])
    total = int(q_start[-1])
    s.update(data=_data(c, gen, pages), refs=_ints(np.bincount(held[held >= 0], minlength=pages)), table=_ints(held),
             length=_ints(lens), slot=_ints(slot), q_start=_ints(q_start), total_q=total, max_q=int(q_lens.max()),
             scale=c["dim"] ** -0.5)
    if c["kind"] == "prefix":
        s.update(group_start=_ints(np.arange(c["groups"] + 1) * c["members"]), shared=_ints(whole * ps))
        # the partial pages hold the same tokens
        d = s["data"]
        for g in range(whole.size):
            rest = int(shared[g] - whole[g] * ps)
            if rest:
                member = torch.as_tensor(table[group == g, whole[g]], device="cuda", dtype=torch.long)
                d[:, :, member, :, :rest] = d[:, :, member[:1], :, :rest]
    wide = c["q_heads"] + (2 * c["kv_heads"] if c["fused"] else 0)
    q = torch.randn((total, wide, c["dim"]), generator=gen, device="cuda", dtype=DTYPES[c["dtype"]])
    s["q"] = q[:, :c["q_heads"]]


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    return {"fork": _run_fork, "compact": _run_compact, "prefix": _run_prefix, "window": _run_window}[s["case"]["kind"]](s)


def _run_fork(s):
    """The slots' last requests leave, new ones are forked into them and take their first tokens."""
    if own:
        cache = s["cache"]
        cache.release(s["child"], ws=s["ws"])
        forked = cache.fork(s["parent"], s["child"], s["tokens"], ws=s["ws"])
        extended = cache.extend(s["child"], s["new"], ws=s["ws"])
        cache.append(0, s["k"], s["v"], s["child"], s["q_start"])
    else:
        _plain_release(s, s["child"])
        forked = _plain_fork(s, s["parent"], s["child"], s["tokens"])
        extended = _plain_extend(s, s["child"], s["new"])
        _plain_append(s, s["child"], s["case"]["new"])
    return dict(data=s["data"], refs=s["refs"], table=s["table"], length=s["length"], forked=forked, extended=extended)


def _run_compact(s):
    if own:
        table, refs, used = s["cache"].compact(out=(s["out_table"], s["out_refs"], s["used"]), ws=s["ws"])
    else:
        table, refs, used = _plain_compact(s)
    return dict(data=s["data"], table=table, refs=refs, used=used)


def _run_prefix(s):
    if own:
        from paper_2601_21758_amd import kv
        out, lse = kv.attention(s["q"], s["cache"], 0, s["plan"], scale=s["scale"], ws=s["ws"])
    else:
        out, lse = _plain_prefix(s)
    return dict(out=out, lse=lse)


def _run_window(s):
    if own:
        from paper_2601_21758_amd import kv
        out, lse = kv.attention(s["q"], s["cache"], 0, s["plan"], scale=s["scale"], ws=s["ws"])
    else:
        out, lse = _plain_window(s)
    return dict(out=out, lse=lse)


# ---------------------------------------------------------------------------
# The plain forms
# ---------------------------------------------------------------------------
def _plain_release(s, slot):
    slot = slot.long()
    rows = s["table"][slot]
    pages = rows[rows >= 0].long()
    s["refs"].index_add_(0, pages, torch.full_like(pages, -1, dtype=torch.int32))
    s["table"][slot] = -1
    s["length"][slot] = 0


def _plain_fork(s, parent, child, tokens):
    page, table, length, refs = s["case"]["page"], s["table"], s["length"], s["refs"]
    parent, child, tokens = parent.long(), child.long(), tokens.long()
    full, part = tokens // page, tokens % page > 0
    fine = (length[child] == 0) & (tokens <= length[parent])
    free = torch.nonzero(refs == 0).flatten()
    total = torch.cumsum((part & fine).long(), 0)
    ok = fine & (total <= free.numel())
    rows = table[parent]
    row = torch.where(torch.arange(table.shape[1], device="cuda") < full[:, None], rows, -1)
    copied = (ok & part).nonzero().flatten()
    src, dst = rows[copied, full[copied]].long(), free[:copied.numel()]
    row[copied, full[copied]] = dst.int()
    shared = row.clone()
    shared[copied, full[copied]] = -1
    shared = shared[ok]
    shared = shared[shared >= 0].long()
    refs.index_add_(0, shared, torch.ones_like(shared, dtype=torch.int32))
    refs[dst] = 1
    table[child[ok]] = row[ok]
    length[child[ok]] = tokens[ok].int()
    s["data"][:, :, dst] = s["data"][:, :, src]
    return ok.int()


def _plain_extend(s, slot, tokens):
    page, table, length, refs = s["case"]["page"], s["table"], s["length"], s["refs"]
    slot, tokens = slot.long(), tokens.long()
    have = length[slot].long()
    first = (have + page - 1) // page
    need = (have + tokens + page - 1) // page - first
    fine = have + tokens <= table.shape[1] * page
    need = need * fine
    free = torch.nonzero(refs == 0).flatten()
    total = torch.cumsum(need, 0)
    ok = fine & (total <= free.numel())
    need = need * ok
    i = torch.repeat_interleave(torch.arange(slot.numel(), device="cuda"), need)
    taken = free[:i.numel()]
    j = torch.arange(i.numel(), device="cuda") - (torch.cumsum(need, 0) - need)[i]
    table[slot[i], first[i] + j] = taken.int()
    refs[taken] = 1
    length[slot] = (have + tokens * ok).int()
    return ok.int()


def _plain_append(s, slot, new):
    page = s["case"]["page"]
    slot = slot.long().repeat_interleave(new)
    pos = s["length"][slot].long() - new + torch.arange(slot.numel(), device="cuda") % new
    at = s["table"][slot, pos.clamp(min=0) // page].long()
    put = ((pos >= 0) & (at >= 0)).nonzero().flatten()
    for plane, x in ((0, s["k"]), (1, s["v"])):
        s["data"][0, plane][at[put], :, pos[put] % page] = x[put]


def _plain_compact(s):
    refs, n = s["refs"], s["refs"].numel()
    inuse = refs > 0
    used = inuse.sum()
    page = torch.arange(n, device="cuda")
    holes = torch.nonzero(~inuse & (page < used)).flatten()
    movers = torch.nonzero(inuse & (page >= used)).flatten().flip(0)
    s["data"][:, :, holes] = s["data"][:, :, movers]
    to = page.clone()
    to[movers] = holes
    table = s["table"]
    s["out_table"].copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].int(), -1))
    new = torch.where(inuse & (page < used), refs, 0)
    new[holes] = refs[movers]
    s["out_refs"].copy_(new)
    s["used"].copy_(used)
    return s["out_table"], s["out_refs"], s["used"]


def _rows(s, plane, table, pos):
    """Keys or values at the positions pos of the rows of `table`, in 32 bits: [row][position][kv head][dim]."""
    page = s["case"]["page"]
    at = torch.gather(table, 1, (pos // page).clamp(0, table.shape[1] - 1)).clamp(min=0).long()
    return s["data"][0, plane][at, :, pos % page].float()


def _softmax(scores, seen):
    """exp(score - maximum) where seen, its sum and ln of the sum; a row that sees nothing has 0, 0 and -inf."""
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True).clamp(min=FLOOR)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lse = torch.where(total > 0, top + total.log(), -math.inf)
    return p, total, lse.squeeze(-1)


def _plain_prefix(s):
    c = s["case"]
    G, M, Hk, D = c["groups"], c["members"], c["kv_heads"], c["dim"]
    R, dev, n, dtype = c["q_heads"] // Hk, "cuda", G * M, s["q"].dtype
    slot, q_start = s["slot"].long(), s["q_start"].long()
    q_len, length, shared = q_start[1:] - q_start[:-1], s["length"][slot].long(), s["shared"].long()
    table = s["table"][slot]
    Q, P = s["max_q"], max(1, int(shared.max()))
    O = max(1, int((length - shared.repeat_interleave(M)).max()))
    seq = torch.repeat_interleave(torch.arange(n, device=dev), q_len)
    i = torch.arange(s["total_q"], device=dev) - q_start[seq]
    q = torch.zeros((n, Q, Hk, R, D), device=dev)
    q[seq, i] = s["q"].float().reshape(-1, Hk, R, D) * s["scale"]
    # the shared part: one product for a group and key head
    pos = torch.arange(P, device=dev).expand(G, P)
    first = table[torch.arange(G, device=dev) * M]
    kp, vp = (_rows(s, x, first, pos).permute(0, 2, 1, 3).contiguous() for x in (0, 1))
    rows = q.reshape(G, M * Q, Hk, R, D).permute(0, 2, 1, 3, 4).reshape(G, Hk, M * Q * R, D)
    sp = torch.matmul(rows, kp.transpose(-1, -2))
    # each sequence's own part
    own_pos = shared.repeat_interleave(M)[:, None] + torch.arange(O, device=dev)
    ko, vo = (_rows(s, x, table, own_pos).permute(0, 2, 1, 3).contiguous() for x in (0, 1))
    so = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(n, Hk, Q * R, D), ko.transpose(-1, -2))
    sp = sp.reshape(G, Hk, M, Q * R, P).permute(0, 2, 1, 3, 4).reshape(n, Hk, Q, R, P)
    at = (length - q_len)[:, None] + torch.arange(Q, device=dev)
    seen_own = (own_pos[:, None] <= at[..., None])[:, None, :, None].expand(n, Hk, Q, R, O)
    seen_shared = ((pos < shared[:, None]).repeat_interleave(M, 0)[:, None] & (pos[:1, None] <= at[..., None]))
    seen = torch.cat([seen_shared[:, None, :, None].expand(n, Hk, Q, R, P), seen_own], -1)
    p, total, lse = _softmax(torch.cat([sp, so.reshape(n, Hk, Q, R, O)], -1), seen)
    pp = p[..., :P].reshape(G, M, Hk, Q * R, P).permute(0, 2, 1, 3, 4).reshape(G, Hk, M * Q * R, P)
    out = torch.matmul(pp, vp).reshape(G, Hk, M, Q * R, D).permute(0, 2, 1, 3, 4).reshape(n, Hk, Q, R, D)
    out = out + torch.matmul(p[..., P:].reshape(n, Hk, Q * R, O), vo).reshape(n, Hk, Q, R, D)
    out = out / torch.where(total > 0, total, 1.0)
    return (out.permute(0, 2, 1, 3, 4)[seq, i].reshape(-1, c["q_heads"], D).to(dtype),
            lse.permute(0, 2, 1, 3)[seq, i].reshape(-1, c["q_heads"]))


def _plain_window(s):
    c = s["case"]
    Hk, D, W, S, n = c["kv_heads"], c["dim"], c["window"], c["sinks"], c["seqs"]
    R, dev, dtype = c["q_heads"] // Hk, "cuda", s["q"].dtype
    slot, q_start = s["slot"].long(), s["q_start"].long()
    q_len, length = q_start[1:] - q_start[:-1], s["length"][slot].long()
    # queries in chunks of C; a chunk sees its window's span of keys and the sinks before it
    C = min(512, s["max_q"])
    chunks = (q_len + C - 1) // C
    owner = torch.repeat_interleave(torch.arange(n, device=dev), chunks)
    order = torch.arange(owner.numel(), device=dev) - (torch.cumsum(chunks, 0) - chunks)[owner]
    start = (length - q_len)[owner] + order * C
    seq = torch.repeat_interleave(torch.arange(n, device=dev), q_len)
    i = torch.arange(s["total_q"], device=dev) - q_start[seq]
    at_chunk, at = (torch.cumsum(chunks, 0) - chunks)[seq] + i // C, i % C
    q = torch.zeros((owner.numel(), C, Hk, R, D), device=dev)
    q[at_chunk, at] = s["q"].float().reshape(-1, Hk, R, D) * s["scale"]
    span = start[:, None] - W + 1 + torch.arange(W + C - 1, device=dev)
    sink = torch.arange(S, device=dev).expand(owner.numel(), S)
    pos = torch.cat([sink, span], 1)
    there = torch.cat([sink < span[:, :1], span >= 0], 1) & (pos < length[owner][:, None])
    table = s["table"][slot][owner]
    k, v = (_rows(s, x, table, pos.clamp(min=0)).permute(0, 2, 1, 3).contiguous() for x in (0, 1))
    p_at = start[:, None] + torch.arange(C, device=dev)
    seen = there[:, None] & (pos[:, None] <= p_at[..., None]) & \
        ((pos[:, None] > p_at[..., None] - W) | (pos[:, None] < S))
    scores = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(-1, Hk, C * R, D), k.transpose(-1, -2))
    p, total, lse = _softmax(scores.reshape(-1, Hk, C, R, S + W + C - 1), seen[:, None, :, None])
    out = torch.matmul(p.reshape(-1, Hk, C * R, S + W + C - 1), v).reshape(-1, Hk, C, R, D)
    out = out / torch.where(total > 0, total, 1.0)
    return (out.permute(0, 2, 1, 3, 4)[at_chunk, at].reshape(-1, c["q_heads"], D).to(dtype),
            lse.permute(0, 2, 1, 3)[at_chunk, at].reshape(-1, c["q_heads"]))


# ---------------------------------------------------------------------------
# 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    """Attention from its definition, sequence by sequence in 64 bits; the page operators compute no numbers."""
    if case["kind"] in ("fork", "compact"):
        return None
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    Hk, ps, scale = case["kv_heads"], case["page"], s["scale"]
    R = case["q_heads"] // Hk
    starts, slots, lengths = (s[x].tolist() for x in ("q_start", "slot", "length"))
    out = torch.zeros((s["total_q"], case["q_heads"], case["dim"]), dtype=torch.float64, device="cuda")
    lse = torch.full((s["total_q"], case["q_heads"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, r in enumerate(slots):
        n, a, e = lengths[r], starts[b], starts[b + 1]
        row = s["table"][r, :_pages_of(n, ps)].long()
        keys, values = (s["data"][0, x][row].permute(1, 0, 2, 3).reshape(Hk, -1, case["dim"])[:, :n].double()
                        for x in (0, 1))
        for at in range(a, e, 256):
            stop = min(e, at + 256)
            p = torch.arange(n - e + at, n - e + stop, device="cuda")
            lo = max(0, int(p[0]) - case["window"] + 1) if case["kind"] == "window" else 0
            near = torch.arange(lo, int(p[-1]) + 1, device="cuda")
            j = torch.cat([torch.arange(min(lo, case.get("sinks", 0)), device="cuda"), near])
            seen = j <= p[:, None]
            if case["kind"] == "window":
                seen = seen & ((j > p[:, None] - case["window"]) | (j < case["sinks"]))
            q = s["q"][at:stop].double().reshape(-1, Hk, R, case["dim"]).permute(1, 2, 0, 3)
            x = torch.matmul(q, keys[:, None, j].transpose(-1, -2)) * scale
            x = x.masked_fill(~seen, -math.inf)
            z = torch.logsumexp(x, -1)
            w = torch.where(torch.isinf(z)[..., None], 0.0, torch.exp(x - z[..., None]))
            y = torch.matmul(w, values[:, None, j])
            out[at:stop] = y.permute(2, 0, 1, 3).reshape(stop - at, -1, case["dim"])
            lse[at:stop] = z.permute(2, 0, 1).reshape(stop - at, -1)
    return dict(out=out, lse=lse)
