"""The serving operators in 64 bits: head norms and rotation, attention over a paged
cache, the bookkeeping of its pages, and sampling from given numbers."""
from __future__ import annotations

import math

import numpy as np


def norm_rope(x, weight, eps, cos, sin, interleaved):
    """x [n][heads][dim]; weight [dim] or None; cos, sin [n][rot / 2]."""
    x = np.array(x, np.float64)
    if weight is not None:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    h = cos.shape[1]
    if h == 0:
        return x
    a, b = ([2 * i for i in range(h)], [2 * i + 1 for i in range(h)]) if interleaved else \
        (list(range(h)), list(range(h, 2 * h)))
    c, s = np.asarray(cos, np.float64)[:, None], np.asarray(sin, np.float64)[:, None]
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def visible(place, length, window, sinks):
    """Keys that the token at `place` sees in a sequence of `length` tokens (a mask)."""
    j = np.arange(length)
    m = j <= place
    if window:
        m &= (place - j < window) | (j < sinks)
    return m


def attend_row(q, keys, values, seen, scale):
    """One query over keys, values [n][dim]: (out, lse, sum of p |v|, largest scale sum |q k|)."""
    at = np.nonzero(seen)[0]
    if at.size == 0:
        return np.zeros(values.shape[1]), -math.inf, np.zeros(values.shape[1]), 0.0
    k, v = np.asarray(keys[at], np.float64), np.asarray(values[at], np.float64)
    s = scale * (k @ np.asarray(q, np.float64))
    top = s.max()
    p = np.exp(s - top)
    p /= p.sum()
    with np.errstate(all="ignore"):
        return (p @ v, float(top + np.log(np.exp(s - top).sum())), p @ np.abs(v),
                float(abs(scale) * (np.abs(k) @ np.abs(np.asarray(q, np.float64))).max()))


class Pages:
    """The page table, lengths and reference counts, and each page's contents as a list of marks."""

    def __init__(self, n_pages, page, n_seqs, width):
        self.page, self.width = page, width
        self.refs = [0] * n_pages
        self.table = [[-1] * width for _ in range(n_seqs)]
        self.len = [0] * n_seqs
        self.data = [[(p, i) for i in range(page)] for p in range(n_pages)]

    def _part(self, s):
        """The page that sequence s ends inside of, or None."""
        at, left = divmod(self.len[s], self.page)
        return self.table[s][at] if left and at < self.width and self.table[s][at] >= 0 else None

    def _copy(self, src, dst, tokens):
        self.data[dst][:tokens] = list(self.data[src][:tokens])

    def _take(self, plans):
        """plans: pages wanted by each item; the free pages they get, or the number missing."""
        free = [p for p, r in enumerate(self.refs) if r == 0]
        if sum(plans) > len(free):
            return None, sum(plans) - len(free)
        it = iter(free)
        return [[next(it) for _ in range(n)] for n in plans], 0

    def extend(self, seqs, add):
        want, left_out = [], 0
        for s, a in zip(seqs, add):
            if not (0 <= s < len(self.len)) or a < 0 or self.len[s] + a > self.width * self.page:
                left_out += 1
                want.append(None)
                continue
            part = self._part(s) if a else None
            copy = part is not None and self.refs[part] > 1
            up = lambda n: -(-n // self.page)  # noqa: E731
            # the first page that is missing: the one that the sequence ends inside of, where it is not there
            first = self.len[s] // self.page if a and part is None else up(self.len[s])
            want.append((copy, part, up(self.len[s] + a) - first, first))
        got, missing = self._take([0 if w is None else w[0] + w[2] for w in want])
        if got is None:
            return missing, left_out
        for s, a, w, ids in zip(seqs, add, want, got):
            if w is None:
                continue
            n = self.len[s]
            for p in ids:
                self.refs[p] = 1
            if w[0]:
                self._copy(w[1], ids[0], n % self.page)
                self.refs[w[1]] -= 1
                self.table[s][n // self.page] = ids[0]
                ids = ids[1:]
            self.table[s][w[3]:w[3] + len(ids)] = ids
            self.len[s] = n + a
        return 0, left_out

    def fork(self, src, dst):
        want, left_out = [], 0
        for s, d in zip(src, dst):
            n = len(self.len)
            if not (0 <= s < n and 0 <= d < n) or s == d or self.len[d] != 0:
                left_out += 1
                want.append(None)
                continue
            want.append(self._part(s))
        ok = [w is not None or (0 <= s < len(self.len) and 0 <= d < len(self.len) and s != d and self.len[d] == 0)
              for w, s, d in zip(want, src, dst)]
        got, missing = self._take([int(w is not None) for w in want])
        if got is None:
            return missing, left_out
        for s, d, w, ids, good in zip(src, dst, want, got, ok):
            if not good:
                continue
            full = self.len[s] // self.page
            row = self.table[s][:full] + ids
            for p in self.table[s][:full]:
                if p >= 0:
                    self.refs[p] += 1
            if ids:
                self.refs[ids[0]] = 1
                self._copy(w, ids[0], self.len[s] % self.page)
            self.table[d] = row + [-1] * (self.width - len(row))
            self.len[d] = self.len[s]
        return 0, left_out

    def free(self, seqs, begin=None, end=None):
        for i, s in enumerate(seqs):
            if not 0 <= s < len(self.len):
                continue
            n = self.len[s]
            lo = max(0, begin[i]) if begin is not None else 0
            cut = end is None or end[i] >= n
            last = self.width if cut else end[i] // self.page
            for j in range(-(-lo // self.page), min(last, self.width)):
                if self.table[s][j] >= 0:
                    self.refs[self.table[s][j]] -= 1
                    self.table[s][j] = -1
            if cut:
                self.len[s] = min(n, lo)

    def compact(self):
        n = sum(r > 0 for r in self.refs)
        moves = list(zip([p for p in range(n, len(self.refs)) if self.refs[p]],
                         [p for p in range(n) if not self.refs[p]]))
        to = dict(moves)
        for a, b in moves:
            self.data[b] = list(self.data[a])
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.table = [[to.get(p, p) for p in row] for row in self.table]
        return n


ONE = 1 << 40


def sample(logits, shares, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(id, share of the kept weights, ids kept) of one row.

    shares: exp((l - max) / T) of every id in float32, as the operator takes them.
    """
    x = np.where(np.isnan(logits), -np.inf, np.asarray(logits, np.float64))
    if not x.size or x.max() == -np.inf:
        return -1, 0.0, 0
    order = sorted(range(len(x)), key=lambda i: (-x[i], i))
    if not temperature > 0 or not top_p > 0 or not min_p <= 1:
        return order[0], 1.0, 1
    w = [int(round(float(s) * ONE)) for s in shares]  # (a float32 share times 2^40 rounds half to even)
    k = top_k if 0 < top_k < len(x) else len(x)
    limit = min(float(top_p), 1.0) * float(sum(w[i] for i in order[:k]))
    kept, before = [], 0
    for rank, i in enumerate(order[:k]):
        if rank and not (float(before) < limit):
            break
        if rank == 0 or (w[i] > 0 and shares[i] >= np.float32(min_p)):
            kept.append(i)
        before += w[i]
    kept.sort()
    total = sum(w[i] for i in kept)
    at = min(int(max(float(u), 0.0) * float(total)), total - 1)
    run = 0
    for i in kept:
        run += w[i]
        if run > at:
            return i, w[i] / total, len(kept)
    raise AssertionError
