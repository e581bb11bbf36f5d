"""Reference of the page operations: one entry at a time, with Python sets.

TEST INFRASTRUCTURE ONLY.  The rules of ``include/isv.h`` written out serially.
"""
from __future__ import annotations

import numpy as np

BT, NONE = 16, -1


def blocks(n: int, most: int, open_in_pool: int):
    """(blocks that a length covers, whether it had to be clamped)."""
    if n < 0:
        return 0, True
    b = n // BT + (1 if open_in_pool and n % BT else 0)
    return min(b, most), b > most


def _valid(page, n_pages):
    return 0 <= page < n_pages


def live(rows, n_pages):
    return {int(x) for row in rows for x in row if _valid(x, n_pages)}


class Free:
    def __init__(self, used, n_pages):
        self.ids = iter(sorted(set(range(n_pages)) - used))
        self.short = False

    def take(self):
        x = next(self.ids, NONE)
        self.short = self.short or x == NONE
        return x


def fork(table, lens, parent, most, open_in_pool, n_pages):
    """(table, lens, copy_src, copy_dst, ran out of pages)"""
    R = len(parent)
    out = np.full((R, most), NONE, np.int64)
    n = np.zeros(R, np.int64)
    src, dst = np.full(R, NONE, np.int64), np.full(R, NONE, np.int64)
    seen, private = set(), []
    for s, p in enumerate(parent):
        if not 0 <= p < len(lens):
            continue
        n[s] = lens[p]
        b, _ = blocks(int(n[s]), most, open_in_pool)
        out[s, :b] = table[p, :b]
        if p in seen and open_in_pool and n[s] > 0 and n[s] % BT and n[s] // BT < most and _valid(out[s, b - 1], n_pages):
            private.append((s, b - 1))
        seen.add(int(p))
    keep = out.copy()
    for s, j in private:
        keep[s, j] = NONE
    free = Free(live(keep, n_pages), n_pages)
    for s, j in private:
        page = free.take()
        if page != NONE:
            src[s], dst[s] = out[s, j], page
        out[s, j] = page
    return out, n, src, dst, free.short


def resize(table, old, new, most, open_in_pool, n_pages):
    """(table, ran out of pages)"""
    out = np.full((len(old), most), NONE, np.int64)
    spans = []
    for s in range(len(old)):
        a, b = blocks(int(old[s]), most, open_in_pool)[0], blocks(int(new[s]), most, open_in_pool)[0]
        out[s, :min(a, b)] = table[s, :min(a, b)]
        spans.append((a, b))
    free = Free(live(out, n_pages), n_pages)
    for s, (a, b) in enumerate(spans):
        for j in range(a, b):
            out[s, j] = free.take()
    return out, free.short


def compact(table, lens, most, open_in_pool, n_pages):
    """(table, sources, destinations, live pages)"""
    out = np.full((len(lens), most), NONE, np.int64)
    for s in range(len(lens)):
        b, _ = blocks(int(lens[s]), most, open_in_pool)
        out[s, :b] = table[s, :b]
    used = live(out, n_pages)
    n = len(used)
    src = sorted(x for x in used if x >= n)
    dst = sorted(set(range(n)) - used)
    to = dict(zip(src, dst))
    for s in range(len(lens)):
        for j in range(most):
            out[s, j] = to.get(int(out[s, j]), out[s, j])
    return out, src, dst, n
