"""Plain implementation of the paged 8-bit K/V cache in 64 bits (numpy, loops),
from the definitions in include/daf.h; test infrastructure only.

Codes are held as the values that they stand for, K and V both as
[layer][page][head][token][feature].
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 64
MIN_EXP = -100


def e4m3(x):
    """Nearest e4m3 value, ties to even, of |x| <= 448; NaN stays."""
    x = np.asarray(x, np.float64)
    with np.errstate(divide="ignore", invalid="ignore"):
        e = np.floor(np.log2(np.abs(x)))
    step = np.exp2(np.maximum(np.where(np.isfinite(e), e, -6), -6) - 3)
    return np.rint(x / step) * step


def scale_for(top: float) -> float:
    if top == 0:
        return 0.0
    e = MIN_EXP
    while top > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** e


class CacheOracle:
    def __init__(self, layers, pages, heads, d, n_seqs, max_seq_pages):
        shape = (layers, pages, heads)
        self.code = {n: np.zeros(shape + (PAGE, d)) for n in "kv"}
        self.scale = {n: np.zeros(shape) for n in "kv"}
        self.table = np.full((n_seqs, max_seq_pages), -1, np.int64)
        self.len = np.zeros(n_seqs, np.int64)
        self.refs = np.zeros(pages, np.int64)

    # -- rows ----------------------------------------------------------------------
    def positions(self, cu, seq, pos):
        """Per request: its sequence and the positions of its rows."""
        for b in range(len(cu) - 1):
            n = cu[b + 1] - cu[b]
            L = self.len[seq[b]]
            yield b, seq[b], (np.arange(L - n, L) if pos is None else np.asarray(pos[cu[b]:cu[b + 1]]))

    def page(self, s, i):
        """Page id of a sequence's i-th page, None if it is not there."""
        p = self.table[s, i]
        return int(p) if 0 <= p < len(self.refs) else None

    def write(self, layer, cu, seq, pos, k, v, most):
        """k, v: float64 rows; most: the dtype's largest finite value."""
        for b, s, at in self.positions(cu, seq, pos):
            L = int(self.len[s])
            before = max(L - len(at), 0) if pos is None else L
            ok = (at >= 0) & (at < L)
            for pg in sorted(set((at[ok] // PAGE).tolist())):
                p = self.page(s, pg)
                if p is None:
                    continue
                here = ok & (at // PAGE == pg)
                slots = at[here] - pg * PAGE
                stay = np.setdiff1d(np.arange(min(max(before - pg * PAGE, 0), PAGE)), slots)
                for name, rows in (("k", k), ("v", v)):
                    x = np.clip(rows[cu[b]:cu[b + 1]][here], -most, most)  # [rows][heads][d]
                    for h in range(x.shape[1]):
                        finite = np.abs(x[:, h][~np.isnan(x[:, h])])
                        new = scale_for(float(finite.max()) if finite.size else 0.0)
                        old = self.scale[name][layer, p, h] if len(stay) else 0.0
                        sc = max(old, new)
                        block = np.zeros_like(self.code[name][layer, p, h])
                        if len(stay):
                            # every slot that is not written follows the scale
                            block = e4m3(self.code[name][layer, p, h] * (old / sc)) if sc else \
                                self.code[name][layer, p, h].copy()
                        block[slots] = e4m3(x[:, h] / sc) if sc else np.where(np.isnan(x[:, h]), np.nan, 0.0)
                        self.code[name][layer, p, h] = block
                        self.scale[name][layer, p, h] = sc

    def read(self, layer, cu, seq, pos):
        heads, d = self.code["k"].shape[2], self.code["k"].shape[4]
        out = {n: np.zeros((cu[-1], heads, d)) for n in "kv"}
        for b, s, at in self.positions(cu, seq, pos):
            for j, t in enumerate(at):
                p = self.page(s, t // PAGE) if 0 <= t < self.len[s] else None
                if p is not None:
                    for n in "kv":
                        out[n][cu[b] + j] = self.code[n][layer, p, :, t % PAGE] * self.scale[n][layer, p][:, None]
        return out["k"], out["v"]

    def attn(self, layer, cu, seq, pos, q, scale):
        """o [rows][Hq][D], lse [Hq][rows], and what bounds of the rounding errors take:
        sum of weights * |v| and the largest sum |q| |k| * scale of a visible key."""
        rows, hq, d = q.shape
        heads = self.code["k"].shape[2]
        o, mean = np.zeros((rows, hq, d)), np.zeros((rows, hq, d))
        lse, size = np.full((hq, rows), -np.inf), np.zeros((hq, rows))
        for b, s, at in self.positions(cu, seq, pos):
            L = int(self.len[s])
            pages = [self.page(s, i) for i in range(-(-L // PAGE))]
            there = np.repeat([p is not None for p in pages], PAGE)[:L].astype(bool)
            if not L:
                continue
            ids = [0 if p is None else p for p in pages]
            for h in range(heads):
                kk = np.concatenate([self.code["k"][layer, p, h] * self.scale["k"][layer, p, h] for p in ids])[:L]
                vv = np.concatenate([self.code["v"][layer, p, h] * self.scale["v"][layer, p, h] for p in ids])[:L]
                for j, t in enumerate(at):
                    see = there & (np.arange(L) <= t)
                    if not see.any():
                        continue
                    for hh in range(h * (hq // heads), (h + 1) * (hq // heads)):
                        r = cu[b] + j
                        x = kk[see] @ q[r, hh] * scale
                        m = x.max()
                        w = np.exp(x - m)
                        o[r, hh] = w @ vv[see] / w.sum()
                        mean[r, hh] = w @ np.abs(vv[see]) / w.sum()
                        lse[hh, r] = m + math.log(w.sum())
                        size[hh, r] = (np.abs(kk[see]) @ np.abs(q[r, hh])).max() * scale
        return o, lse, mean, size

    # -- pages ---------------------------------------------------------------------
    def free_ids(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def used(self, s):
        return -(-int(self.len[s]) // PAGE)

    def extend(self, seq, n_new):
        top = self.table.shape[1] * PAGE
        if len(set(seq)) < len(seq) or any(not 0 <= s < len(self.len) for s in seq) or any(n < 0 for n in n_new) or \
                any(self.len[s] + n > top for s, n in zip(seq, n_new)):
            return -1
        need = [-(-(int(self.len[s]) + n) // PAGE) - self.used(s) for s, n in zip(seq, n_new)]
        ids = self.free_ids()
        if sum(need) > len(ids):
            return sum(need) - len(ids)
        for s, n, c in zip(seq, n_new, need):
            for i in range(self.used(s), self.used(s) + c):
                self.table[s, i] = ids.pop(0)
                self.refs[self.table[s, i]] = 1
                for x in self.scale.values():
                    x[:, self.table[s, i]] = 0
            self.len[s] += n
        return 0

    def copy(self, src, dst):
        for a, b in zip(src, dst):
            if 0 <= a < len(self.refs) and 0 <= b < len(self.refs):
                for n in "kv":
                    self.code[n][:, b] = self.code[n][:, a]
                    self.scale[n][:, b] = self.scale[n][:, a]

    def fork(self, src, dst):
        n = len(self.len)
        if any(not 0 <= s < n for s in list(src) + list(dst)) or len(set(dst)) < len(dst) or set(src) & set(dst) or \
                any(self.len[s] for s in dst):
            return -1
        ids = self.free_ids()
        need = sum(1 for s in src if self.len[s] % PAGE and self.page(s, int(self.len[s]) // PAGE) is not None)
        if need > len(ids):
            return need - len(ids)
        for a, b in zip(src, dst):
            full = int(self.len[a]) // PAGE
            for i in range(self.used(a)):
                p = int(self.table[a, i])
                if i < full or not 0 <= p < len(self.refs):
                    self.table[b, i] = p
                    if 0 <= p < len(self.refs):
                        self.refs[p] += 1
                else:
                    self.table[b, i] = ids.pop(0)
                    self.refs[self.table[b, i]] = 1
                    self.copy([p], [self.table[b, i]])
            self.len[b] = self.len[a]
        return 0

    def unshare(self, cu, seq, pos):
        if len(set(seq)) < len(seq) or any(not 0 <= s < len(self.len) for s in seq):
            return -1
        want = []
        for _, s, at in self.positions(cu, seq, pos):
            if (np.diff(at) <= 0).any():
                return -1
            for i in sorted({int(t) // PAGE for t in at if 0 <= t < self.len[s]}):
                p = self.page(s, i)
                if p is not None and self.refs[p] > 1:
                    want.append((s, i, p))
        ids = self.free_ids()
        if len(want) > len(ids):
            return len(want) - len(ids)
        for (s, i, p), q in zip(want, ids):
            self.copy([p], [q])
            self.table[s, i] = q
            self.refs[q] = 1
            self.refs[p] -= 1
        return 0

    def free(self, seq):
        for s in seq:
            if not 0 <= s < len(self.len):
                continue
            for i in range(self.used(s)):
                p = self.page(s, i)
                if p is not None:
                    self.refs[p] -= 1
                self.table[s, i] = -1
            self.len[s] = 0

    def compact(self):
        live = [p for p, r in enumerate(self.refs) if r > 0]
        n = len(live)
        to = dict(zip([p for p in live if p >= n], [p for p in range(n) if self.refs[p] <= 0]))
        self.copy(list(to), list(to.values()))
        for a, b in to.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        for s in range(len(self.len)):
            for i in range(self.used(s)):
                self.table[s, i] = to.get(int(self.table[s, i]), self.table[s, i])
        return n
