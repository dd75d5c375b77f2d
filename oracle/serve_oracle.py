"""The calls around the paged cache in float64 and whole numbers: rotation at given positions, the pages of a step, verification of drafts."""
from __future__ import annotations

import numpy as np


def frequencies(base, rot, scaling="none", factor=1.0, length=0.0, fast=32.0, slow=1.0):
    got = []
    for j in range(rot // 2):
        if scaling == "ntk" and rot > 2:
            got.append((base * factor ** (rot / (rot - 2.0))) ** (-2.0 * j / rot))
            continue
        f = base ** (-2.0 * j / rot)
        if scaling == "linear":
            f /= factor
        if scaling == "yarn":
            turns = length * f / (2.0 * np.pi)
            stays = 0.0 if turns < slow else 1.0 if turns > fast else (turns - slow) / (fast - slow)
            f = stays * f + (1.0 - stays) * f / factor
        got.append(f)
    return np.array(got)


def rope(x, pos, freq, halves=True, gain=1.0, transposed=False):
    """x [n, heads, d]; rows of negative position become NaN.  Angles in extended precision."""
    half = len(freq)
    angle = np.asarray(pos, dtype=np.longdouble)[:, None, None] * np.asarray(freq, dtype=np.longdouble)
    c, s = gain * np.cos(angle), gain * np.sin(angle) * (-1 if transposed else 1)
    first = np.arange(half) if halves else 2 * np.arange(half)
    second = first + (half if halves else 1)
    y = np.array(x, dtype=np.longdouble)
    a, b = y[..., first], y[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    y[np.asarray(pos) < 0] = np.nan
    return y.astype(np.float64)


class Pages:
    """A pool's pages, sequence by sequence and page by page."""

    def __init__(self, n_seq, max_pages, n_pages, page):
        self.page, self.n_pages, self.max_pages = page, n_pages, max_pages
        self.start, self.rows = [0] * n_seq, [[] for _ in range(n_seq)]      # rows: pages that a sequence holds
        self.free = list(range(n_pages))

    def step(self, fresh, n_tok, grow=None):
        """cu, pos, slot, lack; `missing`: entries behind a sequence's pages that become -1."""
        cu, missing, need = [0], [0] * len(self.rows), []
        for b in range(len(self.rows)):
            self.start[b] = max(self.start[b] + (0 if grow is None else int(grow[b])), 0)
            n = min(max(int(fresh[b]), 0), n_tok - cu[-1])
            self.start[b] = min(self.start[b], 2 ** 31 - 1 - n)
            cu.append(cu[-1] + n)
            need.append(min(-(-(self.start[b] + n) // self.page), self.max_pages))
        for b, n in enumerate(need):
            self.free += self.rows[b][n:]
            self.rows[b] = self.rows[b][:n]
        for b, n in enumerate(need):
            while len(self.rows[b]) < n and self.free:
                self.rows[b].append(self.free.pop(0))
            missing[b] = n - len(self.rows[b])
        pos, slot = [-1] * n_tok, [-1] * n_tok
        for b in range(len(self.rows)):
            for i in range(cu[b], cu[b + 1]):
                p = self.start[b] + i - cu[b]
                pos[i] = p
                if p // self.page < len(self.rows[b]) and 0 <= self.rows[b][p // self.page] < self.n_pages:
                    slot[i] = self.rows[b][p // self.page] * self.page + p % self.page
        self.missing = missing
        return np.array(cu), np.array(pos), np.array(slot, dtype=np.int64), sum(missing)


def _probability(row):
    row = np.asarray(row, dtype=np.float64)
    return np.where(np.isfinite(row) & (row > 0), row, 0.0)


def verify(target, tokens, cu, u, draft=None):
    """out, a list a sequence of its new tokens, and how far the drawn number is from the nearest border, relative to the sum."""
    got, margins = [], []
    vocab = target.shape[1]
    for b in range(len(cu) - 1):
        lo, hi = cu[b], cu[b + 1]
        new, margin = [], np.inf
        if hi == lo:
            got.append(new)
            margins.append(margin)
            continue
        at = lo
        while at + 1 < hi:
            x = int(tokens[at + 1])
            if not 0 <= x < vocab:
                break
            q = 1.0 if draft is None else _probability(draft[at + 1][x])
            if not float(u[at + 1]) * q < _probability(target[at][x]):
                break
            new.append(x)
            at += 1
        p = w = _probability(target[at])
        if at + 1 < hi:
            if draft is not None:
                w = np.maximum(p - _probability(draft[at + 1]), 0.0)
            elif 0 <= tokens[at + 1] < vocab:
                w = p.copy()
                w[tokens[at + 1]] = max(p[tokens[at + 1]] - 1.0, 0.0)
        if not w.sum() > 0:
            w = p
        if not w.sum() > 0:
            new.append(-1)
        else:
            sums, r = np.cumsum(w), float(u[lo])
            if r >= 1.0:
                new.append(int(np.flatnonzero(w)[-1]))
            else:
                r = (r if r > 0 else 0.0) * sums[-1]
                new.append(int(np.argmax(sums > r)))
                if r > 0:
                    margin = float(np.min(np.abs(sums - r))) / sums[-1]
        got.append(new)
        margins.append(margin)
    return got, margins
