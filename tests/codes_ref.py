"""Plain forms of the 8-bit cache and the beam operators for the tests, on the host in 64 bits."""
import math

import numpy as np

MOST = {"bf16": 1.875 * 2.0 ** 127, "f16": 61440.0}
# e4m3: sign, four bits of exponent with a bias of 7, three of mantissa; 0x7f is NaN
TABLE = np.asarray([(8 + c % 8) * 2.0 ** (c // 8 - 10) if c >= 8 else c * 2.0 ** -9 for c in range(127)])


def values(codes, scales):
    """codes uint8 [..][D], scales uint8 [..]."""
    size = np.where(codes & 127 == 127, np.nan, np.append(TABLE, np.nan)[codes & 127])
    return np.where(codes >= 128, -size, size) * np.exp2(scales[..., None].astype(np.float64) - 127)


def quantise(x, kind):
    """x float64 [..][D]: codes, scales and what they stand for."""
    x = np.clip(x, -MOST[kind], MOST[kind])
    top = np.abs(np.where(np.isnan(x), 0, x)).max(-1)
    f, k = np.frexp(top)  # top = f 2^k with f in [1/2, 1): 448 = 7/8 2^9
    e = np.where(top > 0, np.maximum(k - 9 + (f > 0.875), -117), -117)
    y = np.abs(x) / np.exp2(e.astype(np.float64))[..., None]
    y = np.where(np.isnan(y), 0, y)
    hi = np.minimum(np.searchsorted(TABLE, y), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = TABLE[hi] - y, y - TABLE[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    code = np.where(np.isnan(x), 127, np.where(np.signbit(x), code | 128, code)).astype(np.uint8)
    scale = (e + 127).astype(np.uint8)
    return code, scale, values(code, scale)


def reorder(pages, slot, parent):
    """The cache's books (kv_ref.Pages) after a reordering: grants."""
    n, ps = len(slot), pages.ps
    there = [0 <= s < pages.length.size for s in slot]
    born = [there[i] and 0 <= parent[i] < n and there[parent[i]] for i in range(n)]
    rows = [pages.table[s].copy() if there[i] else None for i, s in enumerate(slot)]
    lens = [int(pages.length[s]) if there[i] else 0 for i, s in enumerate(slot)]
    takers = {}
    for i in range(n):
        if there[i]:
            takers.setdefault(parent[i], []).append(i)
    for i in range(n):
        if there[i] and i not in takers:
            for p in rows[i]:
                if pages._held(p):
                    pages.refs[p] -= 1
    heir = {p: p if p in t else t[0] for p, t in takers.items()}
    source = {}
    for i in range(n):
        if born[i] and heir[parent[i]] != i and lens[parent[i]] % ps:
            page = rows[parent[i]][lens[parent[i]] // ps]
            if pages._held(page):
                source[i] = page
    free = pages._free()
    granted, taken = [], 0
    picked = {}
    for i in range(n):
        ok = born[i]
        if i in source:
            ok = taken < len(free)
            if ok:
                picked[i] = free[taken]
            taken += 1
        granted.append(int(ok))
    for i in range(n):
        if not there[i]:
            continue
        s, p = slot[i], parent[i]
        if not granted[i]:
            pages.table[s], pages.length[s] = -1, 0
        elif heir[p] == i:
            pages.table[s], pages.length[s] = rows[p], lens[p]
        else:
            full = lens[p] // ps
            pages.table[s] = -1
            pages.table[s, :full] = rows[p][:full]
            for page in rows[p][:full]:
                if pages._held(page):
                    pages.refs[page] += 1
            if i in picked:
                pages.table[s, full] = picked[i]
                pages.refs[picked[i]] = 1
                pages.data[:, :, picked[i]] = pages.data[:, :, source[i]]
            pages.length[s] = lens[p]
    return granted


def select(logits, score, beams, picks, done=None, end=0):
    """parent, token, score of each group's picks; logits float64 [rows][vocab] (exact), score float64."""
    rows, V = logits.shape
    parent, token = (np.full((rows // beams, picks), -1, np.int64) for _ in range(2))
    value = np.full((rows // beams, picks), -math.inf)
    for g in range(rows // beams):
        found = []
        for r in range(g * beams, (g + 1) * beams):
            s = score[r]
            if not s > -math.inf:
                continue
            if done is not None and done[r]:
                found.append((-s, r, -math.inf, end, s))
                continue
            x = np.where(np.isnan(logits[r]), -math.inf, logits[r])
            top = x.max()
            if top == -math.inf:
                continue
            if top == math.inf:
                hot = np.flatnonzero(x == math.inf)
                found += [(-(s - math.log(hot.size)), r, -math.inf, int(v), s - math.log(hot.size)) for v in hot[:picks]]
                continue
            lse = top + math.log(math.fsum(np.exp(x - top)))
            order = np.lexsort((np.arange(V), -x))[:picks]
            found += [(-(s - lse + x[v]), r, -x[v], int(v), s - lse + x[v]) for v in order if x[v] > -math.inf]
        for k, (_, r, _, v, z) in enumerate(sorted(found)[:picks]):
            parent[g, k], token[g, k], value[g, k] = r, v, z
    return parent, token, value
