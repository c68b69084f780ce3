"""Plain forms of the cache and attention operators for the tests: pages with
Python lists, attention in 64 bits, one query at a time, from the definition."""
import math

import numpy as np


class Pages:
    """A cache's books and data on the host; the same requests as the library."""

    def __init__(self, data, refs, table, length, page_size):
        self.data, self.refs, self.table, self.length = data.copy(), refs.copy(), table.copy(), length.copy()
        self.ps = page_size

    def _free(self):
        return [p for p in range(self.refs.size) if self.refs[p] == 0]

    def _held(self, page):
        return 0 <= page < self.refs.size

    def _serve(self, needs):
        """Page lists for needs[i] (None: invalid by itself), or None for a refused request."""
        free, run, got = self._free(), 0, []
        for n in needs:
            if n is not None:
                run += n
            got.append(None if n is None or run > len(free) else free[run - n:run])
        return got

    def extend(self, slot, tokens):
        ps, needs = self.ps, []
        for s, t in zip(slot, tokens):
            ok = 0 <= s < self.length.size and t >= 0 and self.length[s] + t <= self.table.shape[1] * ps
            needs.append(-(-(self.length[s] + t) // ps) - -(-self.length[s] // ps) if ok else None)
        got = self._serve(needs)
        for s, t, g in zip(slot, tokens, got):
            if g is None:
                continue
            at = -(-self.length[s] // ps)
            self.table[s, at:at + len(g)] = g
            self.refs[g] = 1
            self.length[s] += t
        return [int(g is not None) for g in got]

    def fork(self, parent, child, tokens):
        ps, needs = self.ps, []
        slots = range(self.length.size)
        for p, s, t in zip(parent, child, tokens):
            ok = p in slots and s in slots and p != s and t >= 0 and self.length[s] == 0 and t <= self.length[p]
            needs.append((int(t % ps > 0 and self._held(self.table[p, t // ps]))) if ok else None)
        got = self._serve(needs)
        for p, s, t, g in zip(parent, child, tokens, got):
            if g is None:
                continue
            full = t // ps
            for j in range(full):
                self.table[s, j] = self.table[p, j]
                if self._held(self.table[p, j]):
                    self.refs[self.table[p, j]] += 1
            if t % ps:
                self.table[s, full] = g[0] if g else -1
            if g:
                self.refs[g[0]] = 1
                self.data[:, :, g[0]] = self.data[:, :, self.table[p, full]]
            self.length[s] = t
        return [int(g is not None) for g in got]

    def release(self, slot, begin=None, end=None):
        ps = self.ps
        for i, s in enumerate(slot):
            if not 0 <= s < self.length.size:
                continue
            pages = range(self.table.shape[1])
            if begin is not None:
                have = min(int(end[i]), int(self.length[s]))
                pages = range(-(-max(0, int(begin[i])) // ps), max(0, have) // ps)
            for j in pages:
                if self._held(self.table[s, j]):
                    self.refs[self.table[s, j]] -= 1
                self.table[s, j] = -1
            if begin is None:
                self.length[s] = 0

    def compact(self):
        used = [p for p in range(self.refs.size) if self.refs[p]]
        U = len(used)
        holes = [p for p in range(U) if not self.refs[p]]
        to = dict(zip(sorted((p for p in used if p >= U), reverse=True), holes))
        refs = np.zeros_like(self.refs)
        for p in used:
            refs[to.get(p, p)] = self.refs[p]
        table = self.table.copy()
        for i in np.ndindex(table.shape):
            table[i] = to.get(table[i], table[i])
        for a, b in to.items():
            self.data[:, :, b] = self.data[:, :, a]
        return table, refs, U

    def append(self, layer, k, v, slot, q_start):
        for b, s in enumerate(slot):
            if not 0 <= s < self.length.size:
                continue
            for t in range(q_start[b], q_start[b + 1]):
                pos = self.length[s] - (q_start[b + 1] - t)
                if pos < 0 or not self._held(self.table[s, pos // self.ps]):
                    continue
                page = self.table[s, pos // self.ps]
                self.data[layer, 0, page, :, pos % self.ps] = k[t]
                self.data[layer, 1, page, :, pos % self.ps] = v[t]


def attention(q, data, table, length, slot, q_start, page_size, scale, window=0, sinks=0):
    """q float64 [total][q_heads][D]; data float64 [2][pages][kv_heads][page][D].  Returns out, lse, and, for the error
    bound, sum of weights times |v|, the largest sum |q_d k_d| * scale and the largest |score| of each query head."""
    total, Hq, D = q.shape
    Hk = data.shape[2]
    G = Hq // Hk
    out, mass = np.zeros((total, Hq, D)), np.zeros((total, Hq, D))
    lse = np.full((total, Hq), -math.inf)
    size, top = np.zeros((total, Hq)), np.zeros((total, Hq))
    for b, s in enumerate(slot):
        a, e = q_start[b], q_start[b + 1]
        if not 0 <= s < len(length):
            continue
        for t in range(a, e):
            p = length[s] - (e - t)
            j = np.arange(p + 1)
            if window:
                j = j[(j > p - window) | (j < sinks)]
            page = table[s, j // page_size] if j.size else j
            j, page = j[(page >= 0) & (page < data.shape[1])], page[(page >= 0) & (page < data.shape[1])]
            if not j.size:
                continue
            K, V = data[0][page, :, j % page_size], data[1][page, :, j % page_size]  # [keys][Hk][D]
            for h in range(Hq):
                k, v = K[:, h // G], V[:, h // G]
                x = k @ q[t, h] * scale
                m = x.max()
                w = np.exp(x - m)
                l = w.sum()
                out[t, h], mass[t, h] = w @ v / l, w @ np.abs(v) / l
                lse[t, h] = m + math.log(l)
                size[t, h] = (np.abs(k) @ np.abs(q[t, h])).max() * scale
                top[t, h] = np.abs(x).max()
    return out, lse, mass, size, top


def bounds(out, lse, mass, size, top, unit, keys, vmax, dim):
    """Bounds of the error of 16-bit attention with exact inputs: unit is the rounding of the type (2^-8 bfloat16, 2^-11
    float16).  A score summed in binary32 is off by at most d = (dim + 2) 2^-24 sum |q k| and, in the exponent, by the
    rounding of its scaled value, 4 2^-24 |score|, so a weight by e^2d; a weight is rounded once more to 16 bits (unit,
    or half the smallest subnormal of float16, 2^-25, for each key), the sums and the join in binary32 add 2^-18, and the
    result is rounded to 16 bits (unit |out|, or 2^-25)."""
    d = ((dim + 2) * size + 8 * (1 + top)) * 2.0 ** -24
    rel = unit + 2 * d + 2.0 ** -18
    tiny = 2.0 ** -25
    b_out = rel[..., None] * mass + (unit * (1 + rel[..., None])) * (np.abs(out) + rel[..., None] * mass) \
        + tiny * keys * vmax + tiny
    b_lse = d + 2.0 ** -20 * (1 + np.where(np.isfinite(lse), np.abs(lse), 0))
    return b_out, b_lse
