"""CPU oracle for the operators around the packed projections: low-rank adapters, head norms with rotation, the 4-bit
key/value cache and the attention over it.

TEST INFRASTRUCTURE ONLY, like spdp_oracle.py: plain NumPy in 64 bits, sharing no code with the library.  Next to each result
stands what its error bound is made of (sums of absolute values), so that the tests' tolerances can be written as arithmetic.
"""
from __future__ import annotations

import numpy as np


def lora(X, adapter, A, B, base, scales=None, ranks=None):
    """(y, t_part, b_part) in 64 bits: y = base + s B (A x); t_part = s |B| (|A| |x|), b_part = s |B| |A x|."""
    X, A, B = (np.asarray(a, np.float64) for a in (X, A, B))
    y = np.array(base, np.float64)
    t_part, b_part = np.zeros_like(y), np.zeros_like(y)
    for n, a in enumerate(np.asarray(adapter)):
        if not 0 <= a < len(A):
            continue
        r = A.shape[1] if ranks is None else int(min(max(ranks[a], 0), A.shape[1]))
        s = 1.0 if scales is None else float(scales[a])
        t = A[a, :r] @ X[n]
        y[n] += s * (B[a, :, :r] @ t)
        t_part[n] = abs(s) * (np.abs(B[a, :, :r]) @ (np.abs(A[a, :r]) @ np.abs(X[n])))
        b_part[n] = abs(s) * (np.abs(B[a, :, :r]) @ np.abs(t))
    return y, t_part, b_part


def norm_rope(x, weight, eps, pos, inv_freq, sections, adjacent):
    """(y, size) in 64 bits for heads x [N][H][D]; size = |a| + |b| of the two values that y was turned from."""
    x = np.array(x, np.float64)
    if weight is not None:
        x = x / np.sqrt(np.mean(x * x, -1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    size = np.abs(x)
    pairs = 0 if inv_freq is None else len(inv_freq)
    if pairs:
        pos = np.atleast_2d(np.asarray(pos, np.float64))
        axis = np.repeat(np.arange(len(sections)), sections)
        angle = (pos[axis] * np.asarray(inv_freq, np.float64)[:, None]).T[:, None, :]
        first, second = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if adjacent else (slice(0, pairs), slice(pairs, 2 * pairs))
        a, b = x[..., first].copy(), x[..., second].copy()
        x[..., first], x[..., second] = a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)
        size[..., first] = size[..., second] = np.abs(a) + np.abs(b)
    return x, size


def kv4_codes(x):
    """fp16 rows [..., D] -> (codes uint8 [..., D], scales fp16 [..., D/32])."""
    f = np.asarray(x, np.float16).astype(np.float64).reshape(*x.shape[:-1], -1, 32)
    scale = (np.abs(f).max(-1) / 7.0).astype(np.float16)
    s = scale.astype(np.float64)[..., None]
    code = np.where(s > 0, np.clip(np.rint(f / np.where(s > 0, s, 1.0)), -7, 7), 0.0) + 8
    return code.reshape(x.shape).astype(np.uint8), scale


def kv4_values(codes, scales):
    return (codes.astype(np.float64) - 8.0) * np.repeat(scales.astype(np.float64), 32, -1)


class Kv4Cache:
    """A cache as the header describes it, written and read element by element."""

    def __init__(self, raw, heads, dim, page):
        self.raw, self.heads, self.dim, self.page = np.asarray(raw, np.uint8), heads, dim, page
        self.groups = dim // 32
        assert self.raw.shape[1] == heads * page * (dim + dim // 8)
        d = np.arange(dim)
        self.nibble = 8 * ((d % 32) // 8 * self.groups + d // 32) + d % 8          # of the row, low nibbles first

    def _at(self, slot, h, side):
        """(page, byte of the row of codes, byte of its scales)."""
        page, at = divmod(int(slot), self.page)
        n, m = self.page * self.dim // 2, self.page * self.groups * 2
        head = h * 2 * (n + m)
        return page, head + side * n + at * self.dim // 2, head + 2 * n + side * m + at * self.groups * 2

    def store(self, slot, k, v):
        """k, v: fp16 [heads][dim]."""
        if not 0 <= slot < len(self.raw) * self.page:
            return
        for side, rows in enumerate((k, v)):
            codes, scales = kv4_codes(rows)
            for h in range(self.heads):
                page, row, sc = self._at(slot, h, side)
                nibbles = np.zeros(self.dim, np.uint8)
                nibbles[self.nibble] = codes[h]
                self.raw[page, row:row + self.dim // 2] = nibbles[0::2] | nibbles[1::2] << 4
                self.raw[page, sc:sc + 2 * self.groups] = scales[h].view(np.uint8)

    def load(self, slot, h, side):
        page, row, sc = self._at(slot, h, side)
        by = self.raw[page, row:row + self.dim // 2]
        nibbles = np.stack([by & 15, by >> 4], -1).reshape(-1)
        return kv4_values(nibbles[self.nibble], self.raw[page, sc:sc + 2 * self.groups].view(np.float16))


def attention(q, cache, table, length, scale, cap=0.0, window=0):
    """One request, q [q_heads][dim]: (y [q_heads][dim], spread, reach, keys) in 64 bits.  spread = sum p |v| / sum p, reach = the largest
    |scale| * sum |q_d k_d| of a key, keys = how many count."""
    q = np.asarray(q, np.float64)
    group = len(q) // cache.heads
    length = int(min(max(length, 0), len(table) * cache.page))
    keys = [t for t in range(max(0, length - window) if window else 0, length) if 0 <= table[t // cache.page] < len(cache.raw)]
    y, spread, reach = np.zeros_like(q), np.zeros_like(q), np.zeros(len(q))
    if not keys:
        return y, spread, reach, 0
    for h in range(cache.heads):
        slots = [int(table[t // cache.page]) * cache.page + t % cache.page for t in keys]
        k, v = (np.stack([cache.load(s, h, side) for s in slots]) for side in (0, 1))
        for i in range(h * group, (h + 1) * group):
            z = scale * (k @ q[i])
            if cap:
                z = cap * np.tanh(z / cap)
            p = np.exp(z - z.max())
            y[i], spread[i] = p @ v / p.sum(), p @ np.abs(v) / p.sum()
            reach[i] = abs(scale) * (np.abs(k) @ np.abs(q[i])).max()
    return y, spread, reach, len(keys)
