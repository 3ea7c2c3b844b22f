"""The 4-bit key/value cache, page assignment and rotary positions in numpy, 64 bits, written from their definitions (include/rsa.h).
Test infrastructure only."""
from __future__ import annotations

import numpy as np

from oracle import cache_oracle as co

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def round_e2m1(x: np.ndarray) -> np.ndarray:
    """Nearest values of e2m1 of |x| <= 6; on ties the one of the even code."""
    a = np.abs(x)
    code = np.zeros(a.shape, dtype=int)
    for i in range(1, 8):
        mid = (LEVELS[i - 1] + LEVELS[i]) / 2
        code = np.where((a > mid) | ((a == mid) & (i % 2 == 0)), i, code)
    return np.copysign(LEVELS[code], x)


def stored(row: np.ndarray, run: int) -> np.ndarray:
    """What is held of one row [d]: a scale to each `run` channels; NaN where one of them is not finite, infinity from 2^128 on."""
    out = np.zeros_like(row)
    for i in range(0, len(row), run):
        x = row[i:i + run]
        if not np.isfinite(x).all():
            out[i:i + run] = np.nan
            continue
        e = co.least_exponent(float(np.abs(x).max()), 6.0, -124)
        y = np.ldexp(round_e2m1(np.ldexp(x, -e)), e)
        out[i:i + run] = np.where(np.abs(y) >= 2.0 ** 128, np.copysign(np.inf, y), y)
    return out


class Cache(co.Cache):
    """The cache of cache_oracle with 4-bit pages: a Page's ek and ev are not used."""

    def _write_block(self, page, h, off, k, v):
        p = self.held.get((page, h))
        if p is None:
            p = self.held[page, h] = co.Page(self.block, self.d)
        for i in range(len(k)):
            p.k[off + i], p.v[off + i] = stored(k[i], 32), stored(v[i], self.d)
        n = off + len(k)
        mean = np.where(np.isfinite(p.k[:n]), p.k[:n], 0.0).sum(0) / n
        p.em = co.least_exponent(float(np.abs(mean).max()), 127.0, -100)
        p.mean = np.rint(np.ldexp(mean, -p.em)).astype(np.int64)

    def attend(self, *args, **kw):
        """cache_oracle's, with A = sum p |v| / sum p: a weight's rounding to bf16 costs an output at most 2^-8 of that."""
        out = super().attend(*args, **kw)
        return {**out, "A": self._weighted(*args, **kw)}

    def _weighted(self, Q, kv_len, q_len, scale, causal, lists=None, group=0):
        other = Cache(self.hk, self.d, self.block, self.table, self.pages)
        other.held = {at: _absolute(p) for at, p in self.held.items()}
        return co.Cache.attend(other, Q, kv_len, q_len, scale, causal, lists, group)["O"]


def _absolute(p):
    q = co.Page(*p.k.shape)
    q.k, q.v = p.k, np.abs(p.v)
    return q


# ---- pages ---------------------------------------------------------------------------------------
def assign(table, free_pages, free_count, kv_len, add, t, block, pages, shared=None):
    """(table, free list as far as it is valid, new lengths, starts, counts, positions, slots); all as lists or int arrays. The list `shared` goes
    down in place where a sequence takes pages below it."""
    table = np.array(table)
    batch, width = table.shape
    free = list(free_pages[:max(0, min(int(free_count), pages))])
    held = [min(max(int(n), 0), width * block) for n in kv_len]
    add = [min(int(x), t) for x in add]
    new, start, count = list(held), list(held), [0] * batch
    for b in range(batch):
        if add[b] < 0:
            new[b] = start[b] = max(0, held[b] + add[b])
            for e in range(-(-new[b] // block), -(-held[b] // block)):
                p = table[b, e]
                if 0 <= p < pages and not (shared is not None and e < shared[b]) and len(free) < pages:
                    free.append(int(p))
                table[b, e] = -1
    have, asked = len(free), 0
    pos, slot = np.full((batch, t), -1), np.full((batch, t), -1)
    for b in range(batch):
        if add[b] < 0 or held[b] + add[b] > width * block:
            continue
        if shared is not None and add[b] > 0 and held[b] % block and held[b] // block < shared[b]:      # into a page of others
            continue
        first, last = -(-held[b] // block), -(-(held[b] + add[b]) // block)
        asked += last - first
        if last > first and asked > have:
            continue
        for e in range(first, last):
            table[b, e] = free.pop()
        if shared is not None and last > first:
            shared[b] = min(shared[b], first)
        new[b], count[b] = held[b] + add[b], add[b]
        for i in range(add[b]):
            pos[b, i] = held[b] + i
            p = table[b, pos[b, i] // block]
            slot[b, i] = p * block + pos[b, i] % block if 0 <= p < pages else -1
    return table, free, new, start, count, pos, slot


# ---- rotary positions ----------------------------------------------------------------------------
def rotate(x, pos, freq, pairing, axis_pairs, factor=1.0, inverse=False):
    """x [b, h, t, d] fp64, pos [axes, b, t]: turned rows, and the sum of the magnitudes behind each output."""
    n = len(freq)
    axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs)
    angle = np.moveaxis(pos[axis], 0, -1).astype(np.longdouble)[:, None] * freq   # [b, 1, t, n]; 2^-33 at 2^31 radians, where 64 bits leave 2^-22
    c, s = np.cos(angle).astype(np.float64) * factor, np.sin(angle).astype(np.float64) * (-factor if inverse else factor)
    first, second = (slice(0, n), slice(n, 2 * n)) if pairing == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    y, size = x.copy(), np.zeros_like(x)
    y[..., first], y[..., second] = x[..., first] * c - x[..., second] * s, x[..., first] * s + x[..., second] * c
    size[..., first] = size[..., second] = factor * (np.abs(x[..., first]) + np.abs(x[..., second]))
    return y, size
