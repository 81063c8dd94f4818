"""CPU oracle for the 8-bit key/value cache, the attention over it and the handling of a cache's pages.

TEST INFRASTRUCTURE ONLY, like layer_ops.py: plain NumPy in 64 bits, sharing no code with the library.
"""
from __future__ import annotations

import numpy as np

CELL, MOST = 16, 61440.0
# what the codes 0 .. 126 stand for (127, which is no number in e4m3, never comes from a number)
NUMBERS = np.array([(m / 8 if e == 0 else 1 + m / 8) * 2.0 ** (max(e, 1) - 7) for e in range(16) for m in range(8)][:127])


def e4m3(x):
    """Codes of the numbers nearest to x, ties to the even code."""
    a = np.abs(np.asarray(x, np.float64))
    high = np.minimum(np.searchsorted(NUMBERS, a), 126)
    low = np.maximum(high - 1, 0)
    up, down = NUMBERS[high] - a, a - NUMBERS[low]
    code = np.where((up < down) | ((up == down) & (high % 2 == 0)), high, low)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def value(code):
    c = np.asarray(code, np.int64)
    return np.where(c >= 128, -1.0, 1.0) * np.append(NUMBERS, np.nan)[c % 128]


def scale_for(x):
    """The smallest power of two from 2^-15 up that takes the largest of x into the codes' range."""
    top, e = float(np.abs(x).max(initial=0.0)), -15
    while top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Kv8Cache:
    """A cache as the header describes it, written and read cell by cell."""

    def __init__(self, raw, heads, dim, page):
        self.raw, self.heads, self.dim, self.page = np.asarray(raw, np.uint8), heads, dim, page
        self.bytes = 2 * CELL * dim + 16
        assert self.raw.shape[1] == heads * page * (2 * dim + 1)
        r, d = np.arange(CELL)[:, None], np.arange(dim)[None]
        self.places = (d // 64 * 1024 + r * 64 + d % 64,
                       CELL * dim + 512 * (d // 32) + 64 * (d % 8) + 16 * (r % 8 // 2) + 4 * (d % 32 // 8) + 2 * (r // 8) + r % 2)

    def cell(self, page, at, h):
        first = (h * (self.page // CELL) + at // CELL) * self.bytes
        return self.raw[page, first:first + self.bytes]

    def store(self, table, length, k, v):
        """New tokens k, v fp16 [n][heads][dim] of a request that has `length` tokens with them: the values that their codes stand for (NaN for
        tokens that are passed over)."""
        length = int(min(max(length, 0), len(table) * self.page))
        n = len(k)
        out = [np.full(k.shape, np.nan), np.full(k.shape, np.nan)]
        start = length - n
        for first in range(max(start, 0) // CELL * CELL, length, CELL) if n else ():
            old, end = min(max(start - first, 0), CELL), min(CELL, length - first)
            page = int(table[first // self.page])
            for h in range(self.heads):
                cell = self.cell(page, first % self.page, h) if 0 <= page < len(self.raw) else None
                for side, x in enumerate((k, v)):
                    x = np.clip(x[first + old - start:first + end - start, h].astype(np.float64), -MOST, MOST)
                    scale = scale_for(x)
                    if cell is not None:
                        codes, kept = cell[self.places[side]], cell[32 * self.dim + 4 * side:][:4].copy().view(np.float32)
                        if old:
                            before, was = codes[:old].copy(), float(kept[0])
                            scale = max(scale, was)
                            if scale > was:
                                codes[:old] = e4m3(value(before) * was / scale)
                        else:
                            codes[:] = 0
                            cell[32 * self.dim + 8:] = 0
                        codes[old:end] = e4m3(x / scale)
                        cell[self.places[side]] = codes
                        cell[32 * self.dim + 4 * side:][:4] = np.array([scale], np.float32).view(np.uint8)
                    out[side][first + old - start:first + end - start, h] = value(e4m3(x / scale)) * scale
        return out

    def load(self, table, t, h, side):
        """Token t's key or value of head h, or None."""
        page = int(table[t // self.page])
        if not 0 <= page < len(self.raw):
            return None
        cell = self.cell(page, t % self.page, h)
        return value(cell[self.places[side][t % CELL]]) * float(cell[32 * self.dim + 4 * side:][:4].copy().view(np.float32)[0])


def attention(q, cache, table, length, scale, cap=0.0, window=0, sinks=0):
    """A request's new tokens, q [n][q_heads][dim]: (y like q, spread, reach [n][q_heads], keys [n]) in 64 bits.  spread = sum p |v| / sum p, reach =
    the largest |scale| * sum |q_d k_d| of a key, keys = how many count."""
    q = np.asarray(q, np.float64)
    n, heads, dim = q.shape
    group = heads // cache.heads
    length = int(min(max(length, 0), len(table) * cache.page))
    y, spread, reach, count = np.zeros_like(q), np.zeros_like(q), np.zeros(q.shape[:2]), np.zeros(n, int)
    there = [t for t in range(length) if 0 <= int(table[t // cache.page]) < len(cache.raw)]
    for h in range(cache.heads):
        sides = [{t: cache.load(table, t, h, side) for t in there} for side in (0, 1)]
        for i in range(n):
            at = length - n + i
            keys = [t for t in there if t <= at and (not window or t > at - window or t < sinks)]
            count[i] = len(keys)
            if not keys:
                continue
            k, v = (np.stack([s[t] for t in keys]) for s in sides)
            for j in range(h * group, (h + 1) * group):
                z = scale * (k @ q[i, j])
                if cap:
                    z = cap * np.tanh(z / cap)
                p = np.exp(z - z.max())
                y[i, j], spread[i, j] = p @ v / p.sum(), p @ np.abs(v) / p.sum()
                reach[i, j] = abs(scale) * (np.abs(k) @ np.abs(q[i, j])).max()
    return y, spread, reach, count


class Pages:
    """The state of a cache's pages: a table, a count for each page, and caches [layers][pages][bytes]."""

    def __init__(self, table, ref, cache, page=16):
        self.table, self.ref, self.cache, self.page = np.array(table, np.int64), np.array(ref, np.int64), np.array(cache), page

    def is_page(self, p):
        return 0 <= p < len(self.ref)

    def named(self, rows, start, stop):
        """(row, entry) of a call, in its order."""
        for r, a, b in zip(rows, start, stop):
            if 0 <= r < len(self.table):
                for e in range(max(a, 0), min(b, self.table.shape[1])):
                    yield r, e

    def lowest(self):
        free = np.flatnonzero(self.ref <= 0)
        if not len(free):
            return -1
        self.ref[free[0]] = 1
        return int(free[0])

    def take(self, rows, start, stop):
        short = 0
        for r, e in self.named(rows, start, stop):
            self.table[r, e] = self.lowest()
            short += self.table[r, e] < 0
        return int(short)

    def free(self, rows, start, stop):
        for r, e in self.named(rows, start, stop):
            if self.is_page(self.table[r, e]):
                self.ref[self.table[r, e]] -= 1
            self.table[r, e] = -1

    def fork(self, parent, child, length):
        short, rows = 0, len(self.table)
        pairs = [(a, b, min(max(n, 0), self.table.shape[1] * self.page)) for a, b, n in zip(parent, child, length) if 0 <= a < rows and 0 <= b < rows]
        for a, b, n in pairs:
            for e in range(n // self.page):
                p = self.table[a, e]
                self.table[b, e] = p if self.is_page(p) else -1
                if self.is_page(p):
                    self.ref[p] += 1
        for a, b, n in pairs:
            if n % self.page:
                e = n // self.page
                p = self.table[a, e]
                new = self.lowest() if self.is_page(p) else -1
                short += self.is_page(p) and new < 0
                self.table[b, e] = new
                if new >= 0:
                    self.cache[:, new] = self.cache[:, p]
        return int(short)

    def copy(self, src, dst):
        for a, b in zip(src, dst):
            if self.is_page(a) and self.is_page(b):
                self.cache[:, b] = self.cache[:, a]

    def compact(self):
        used = self.ref > 0
        live = int(used.sum())
        for new, old in zip(np.flatnonzero(~used[:live]), live + np.flatnonzero(used[live:])):
            self.cache[:, new] = self.cache[:, old]
            self.ref[new], self.ref[old] = self.ref[old], 0
            self.table[self.table == old] = new
        return live
