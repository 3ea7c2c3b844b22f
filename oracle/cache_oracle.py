"""The 8-bit key/value cache in numpy, 64 bits, written from its definition (include/rsa.h): which values a write leaves, which
blocks a score selects, what the attention over them is. Test infrastructure only."""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

LARGEST = 448.0                  # of e4m3


def least_exponent(amax: float, largest: float, least: int) -> int:
    """The least e >= `least` with amax <= largest * 2^e."""
    if amax == 0:
        return least
    e = math.frexp(amax)[1] - math.frexp(largest)[1] - 1
    while Fraction(amax) > Fraction(largest) * Fraction(2) ** e:
        e += 1
    return max(e, least)


def round_e4m3(x: np.ndarray) -> np.ndarray:
    """Nearest values of e4m3 (even on ties) of |x| <= 448; not finite: NaN."""
    x = np.asarray(x, dtype=np.float64)
    fin = np.isfinite(x)
    a = np.where(fin, np.abs(x), 0.0)
    step = np.ldexp(1.0, np.maximum(np.frexp(np.maximum(a, 2.0 ** -6))[1] - 1, -6) - 3)
    return np.where(fin, np.rint(np.where(fin, x, 0.0) / step) * step, np.nan)


class Page:
    """Values of one (page, key/value head) and the exponents that they are held over."""

    def __init__(self, block, d):
        self.k = np.zeros((block, d))
        self.v = np.zeros((block, d))
        self.ek = self.ev = self.em = 0
        self.mean = np.zeros(d, dtype=np.int64)


class Cache:
    def __init__(self, heads_kv, d, block, table, pages):
        self.hk, self.d, self.block, self.pages = heads_kv, d, block, pages
        self.table = np.asarray(table)
        self.held = {}                                    # (page, head) -> Page

    def page_of(self, b, blk):
        if blk < 0 or blk >= self.table.shape[1]:
            return -1
        p = int(self.table[b, blk])
        return p if 0 <= p < self.pages else -1

    def write(self, K, V, start, count=None):
        """K, V [batch, heads_kv, t, d] fp64."""
        t = K.shape[2]
        for b in range(K.shape[0]):
            s, n = int(start[b]), t if count is None else min(int(count[b]), t)
            if s < 0 or n <= 0:
                continue
            for blk in range(s // self.block, (s + n - 1) // self.block + 1):
                page = self.page_of(b, blk)
                if page < 0:
                    continue
                lo, hi = max(s, blk * self.block), min(s + n, (blk + 1) * self.block)
                for h in range(self.hk):
                    self._write_block(page, h, lo - blk * self.block, K[b, h, lo - s:hi - s], V[b, h, lo - s:hi - s])

    def _write_block(self, page, h, off, k, v):
        p = self.held.setdefault((page, h), Page(self.block, self.d))
        for x, name in ((k, "k"), (v, "v")):
            fin = np.where(np.isfinite(x), np.abs(x), 0.0)
            e = least_exponent(float(fin.max()), LARGEST, -126)
            if off:
                e = max(e, getattr(p, "e" + name))
            full = np.zeros((self.block, self.d))
            full[:off] = round_e4m3(np.ldexp(getattr(p, name)[:off], -e))
            full[off:off + len(x)] = round_e4m3(np.ldexp(x, -e))
            setattr(p, name, np.ldexp(full, e))
            setattr(p, "e" + name, e)
        n = off + len(k)
        total = np.where(np.isfinite(p.k), p.k, 0.0).sum(0)     # exact: at most 128 terms of one scale
        mean = total / n
        p.em = least_exponent(float(np.abs(mean).max()), 127.0, -100)
        p.mean = np.rint(np.ldexp(mean, -p.em)).astype(np.int64)

    def rows(self, b, h, lo, hi):
        """Tokens lo..hi-1 (K, V) and which of them have a page."""
        K, V, there = np.zeros((hi - lo, self.d)), np.zeros((hi - lo, self.d)), np.zeros(hi - lo, dtype=bool)
        for t in range(lo, hi):
            p = self.held.get((self.page_of(b, t // self.block), h))
            if p is not None:
                K[t - lo], V[t - lo], there[t - lo] = p.k[t % self.block], p.v[t % self.block], True
        return K, V, there

    def select(self, Q, kv_len, q_len, group, keep, first, last, causal):
        """Q [batch, heads, t, d] fp64 -> {(b, head, group): ascending list}."""
        B, H, t, d = Q.shape
        G, out = H // self.hk, {}
        for b in range(B):
            kv, ql = int(kv_len[b]), t if q_len is None else min(int(q_len[b]), t)
            for h in range(self.hk):
                for g in range(-(-t // group)):
                    t0, t1 = g * group, min(g * group + group, ql)
                    if t1 <= t0 or kv <= 0:
                        out[b, h, g] = []
                        continue
                    p0, p1 = kv - ql + t0, kv - ql + t1 - 1
                    seen = -(-kv // self.block) if not causal else p1 // self.block + 1
                    vis = [m for m in range(max(seen, 0)) if self.page_of(b, m) >= 0]
                    q = Q[b, h * G:h * G + G, t0:t1]
                    q = np.where(np.isfinite(q), q, 0.0).sum((0, 1))
                    q8 = np.rint(np.ldexp(q, -least_exponent(float(np.abs(q).max()), 127.0, -100)))
                    must = [m for m in vis if m < first or (last and p0 // self.block - last < m <= p1 // self.block)]
                    score = {}
                    for m in vis:
                        p = self.held[self.page_of(b, m), h]
                        score[m] = float(np.ldexp(float(p.mean @ q8), p.em))
                    rest = sorted((m for m in vis if m not in must), key=lambda m: (-score[m], m))
                    out[b, h, g] = sorted(must + rest[:max(0, keep - len(must))])
        return out

    def attend(self, Q, kv_len, q_len, scale, causal, lists=None, group=0):
        """Outputs, log-sum-exps and the parts of the error bound of every row. 2^-11 A is what the weights' rounding to fp16 costs an
        output: half a step is 2^-11 p, from 2^-14 on down 2^-25, and never more than the weight itself, so A = sum min(max(p, 2^-14), 2^11 p) |v|
        over sum p, the largest p being 1. S is the largest sum |q||k| * scale, n the number of keys; nothing is left for `vmax`, which is 0. NaN where a
        row is not a query."""
        B, H, t, d = Q.shape
        G = H // self.hk
        scale = scale or d ** -0.5
        O, A = np.full((B, H, t, d), np.nan), np.full((B, H, t, d), np.nan)
        lse, S, n = (np.full((B, H, t), np.nan) for _ in range(3))
        vmax = np.zeros((B, H, t))
        isq = np.zeros((B, H, t), dtype=bool)
        for b in range(B):
            kv, ql = max(int(kv_len[b]), 0), t if q_len is None else min(int(q_len[b]), t)
            for hk in range(self.hk):
                K, V, there = self.rows(b, hk, 0, kv)
                for i in range(max(ql, 0)):
                    end = min(max(kv - ql + i + 1, 0), kv) if causal else kv
                    if lists is None:
                        keys = np.arange(end)
                    else:
                        own = lists[b, hk, i // group]
                        keys = np.concatenate([np.arange(m * self.block, min((m + 1) * self.block, end)) for m in own if m >= 0 and m * self.block < end] or [np.zeros(0, int)]).astype(int)
                    keys = keys[there[keys]]
                    for h in range(hk * G, hk * G + G):
                        isq[b, h, i] = True
                        if not len(keys):
                            O[b, h, i], A[b, h, i], lse[b, h, i], S[b, h, i], n[b, h, i] = 0, 0, -np.inf, 0, 0
                            continue
                        with np.errstate(invalid="ignore"):
                            s = (K[keys] @ Q[b, h, i]) * scale
                            m = s.max()
                            p = np.exp(s - m)
                            O[b, h, i] = p @ V[keys] / p.sum()
                            A[b, h, i] = np.minimum(np.maximum(p, 2.0 ** -14), 2.0 ** 11 * p) @ np.abs(V[keys]) / p.sum()
                            lse[b, h, i] = np.log(p.sum()) + m
                            S[b, h, i] = (np.abs(K[keys]) @ np.abs(Q[b, h, i])).max() * scale
                        n[b, h, i] = len(keys)
        return dict(O=O, A=A, lse=lse, S=S, n=n, vmax=vmax, isq=isq)
