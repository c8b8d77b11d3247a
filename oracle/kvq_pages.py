"""The 4-bit cache's pages in plain numpy: a pool of them, the ranges of their keys, their scores, and picks.

Definitions (include/rollpack.h): pages of 64 tokens; a page's score for a KV head is, over the query heads of the KV head,
the largest sum_d max(q_d, 0) largest_d + min(q_d, 0) smallest_d.
"""
from __future__ import annotations

import numpy as np

PAGE = 64


def pages(n: int) -> int:
    return -(-n // PAGE)


class Pool:
    """Sequences' pages out of a list of free ones, whose end is taken first."""

    def __init__(self, free, n_seqs: int, max_context: int):
        self.n_pages, self.free, self.max_context = len(free), list(free), max_context
        self.table = [[] for _ in range(n_seqs)]
        self.contexts = [0] * n_seqs
        self.missing = 0

    def fit(self, lengths, n_rows: int, max_rows=None, max_context=None):
        """(error, row offsets, positions, slots); with an error nothing changes and there are no rows."""
        max_rows = n_rows if max_rows is None else max_rows
        max_context = self.max_context if max_context is None else max_context
        lengths = [int(x) for x in lengths]
        old = self.contexts
        need = sum(max(0, pages(n) - pages(c)) for n, c in zip(lengths, old))
        back = sum(max(0, pages(c) - pages(n)) for n, c in zip(lengths, old))
        rows = sum(max(0, n - c) for n, c in zip(lengths, old))
        self.missing = 0
        error = 0
        if any(not 0 <= n <= max_context for n in lengths):
            error = 2
        elif need > back + len(self.free):
            error, self.missing = 1, need - back - len(self.free)
        elif rows > n_rows:
            error = 3
        elif any(n - c > max_rows for n, c in zip(lengths, old)):
            error = 5
        if error:
            return error, np.zeros(len(lengths) + 1, np.int32), np.full(n_rows, -1, np.int32), np.full(n_rows, -1, np.int32)
        returned = []
        for b, n in enumerate(lengths):
            returned += self.table[b][pages(n):]
            del self.table[b][pages(n):]
        self.free += returned[::-1]
        off, positions, slots = [0], [], []
        for b, n in enumerate(lengths):
            while len(self.table[b]) < pages(n):
                self.table[b].append(self.free.pop())
            positions += range(old[b], n)
            slots += [self.table[b][t // PAGE] * PAGE + t % PAGE for t in range(old[b], n)]
            off.append(len(positions))
        self.contexts = lengths
        pad = [-1] * (n_rows - len(positions))
        return 0, np.array(off, np.int32), np.array(positions + pad, np.int32), np.array(slots + pad, np.int32)


def key_ranges(k) -> np.ndarray:
    """k [ctx, n_kv, hd] that the cache holds -> [pages, n_kv, 2, hd]; a NaN makes both ends of its dimension NaN."""
    out = np.empty((pages(len(k)), k.shape[1], 2, k.shape[2]))
    for p in range(len(out)):
        part = k[p * PAGE:(p + 1) * PAGE]
        out[p, :, 0], out[p, :, 1] = np.min(part, 0), np.max(part, 0)
    return out


def page_scores(q, ranges, pos, columns: int):
    """q [n, n_q, hd] at positions pos; ranges [pages, n_kv, 2, hd].  ([n, n_kv, columns], the same of magnitudes)."""
    n, n_q, _ = q.shape
    n_kv = ranges.shape[1]
    g = n_q // n_kv
    out = np.full((n, n_kv, columns), -np.inf)
    mag = np.zeros((n, n_kv, columns))
    up, down = np.where(q > 0, q, 0.0), np.where(q < 0, q, 0.0)
    up, down = np.where(np.isnan(q), q, up), np.where(np.isnan(q), q, down)
    for i in range(n):
        for p in range(min(pages(int(pos[i]) + 1), columns)):
            for h in range(n_kv):
                s = slice(h * g, (h + 1) * g)
                with np.errstate(invalid="ignore"):
                    x = up[i, s] @ ranges[p, h, 1] + down[i, s] @ ranges[p, h, 0]
                    out[i, h, p] = np.nan if np.isnan(x).any() else x.max()
                    mag[i, h, p] = (np.abs(up[i, s]) @ np.abs(ranges[p, h, 1]) + np.abs(down[i, s]) @ np.abs(ranges[p, h, 0])).max()
    return out, mag


def pick(scores, seen: int, first: int, last: int, n: int) -> np.ndarray:
    """One list: scores [pages], of which the row sees `seen`."""
    if seen <= n:
        got = list(range(seen))
    else:
        always = [p for p in range(seen) if p < first or p >= seen - last]
        rest = [p for p in range(first, seen - last)]
        key = {p: (0 if np.isnan(scores[p]) else 1, 0.0 if np.isnan(scores[p]) else -float(scores[p]), p) for p in rest}
        got = sorted(always + sorted(rest, key=key.get)[:n - first - last])
    return np.array(got + [-1] * (n - len(got)), np.int32)


def listed_tokens(picks, pos: int) -> np.ndarray:
    """The positions that a row at `pos` attends to with this list (pages that it does not see count nothing)."""
    if pos < 0:
        return np.zeros(0, np.int64)
    t = [np.arange(p * PAGE, min((p + 1) * PAGE, pos + 1)) for p in picks if 0 <= p <= pos // PAGE]
    return np.concatenate(t) if t else np.zeros(0, np.int64)
