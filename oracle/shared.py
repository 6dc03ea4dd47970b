"""Plain counterparts of the operators for many requests that continue one context, written from their definitions in numpy: integers exactly, one
request, page or row at a time, the low-rank products in fp64."""
from __future__ import annotations

import numpy as np


def fork(table, lens, page, src, dst, free, fork_lens, taken, n_pages=1 << 30):
    """(table, lens, copies, used): child i becomes row dst[i], a copy of row src[i] up to fork_lens[i] tokens."""
    old, old_lens, table, lens = table, lens, table.copy(), lens.copy()
    B, cols = table.shape
    copies, used = np.zeros((len(src), 3), np.int32), 0
    copies[:, :2] = -1
    gone = set()
    for i, (s, d) in enumerate(zip(src, dst)):
        first = d not in gone
        gone.add(d)
        if not (0 <= s < B and 0 <= d < B and first and d not in src):
            continue
        n = int(old_lens[s]) if fork_lens is None else int(fork_lens[i])
        if n < 0 or n > old_lens[s] or n > cols * page:
            continue
        full, rest = divmod(n, page)
        if rest:
            at = taken + used
            used += 1
            if at >= len(free) or not 0 <= free[at] < n_pages:
                continue
            copies[i] = old[s, full], free[at], rest
            table[d, full] = free[at]
        table[d, :full] = old[s, :full]
        lens[d] = n
    return table, lens, copies, used


def _held(table, lens, page, n_pages):
    for b in range(len(lens)):
        for c in range(min(table.shape[1], -(-max(0, int(lens[b])) // page))):
            if 0 <= table[b, c] < n_pages:
                yield b, c


def release(table, lens, page, drop, n_pages):
    """(lens, references of every page, free list, its length)."""
    lens = lens.copy()
    lens[list(drop)] = 0
    refs = np.zeros(n_pages, np.int32)
    for b, c in _held(table, lens, page, n_pages):
        refs[table[b, c]] += 1
    free = [p for p in range(n_pages) if refs[p] == 0]
    return lens, refs, np.array(free + [-1] * (n_pages - len(free)), np.int32), len(free)


def compact(table, lens, page, n_pages):
    """(table, new id of every page, moves, pages in use)."""
    live = sorted({int(table[b, c]) for b, c in _held(table, lens, page, n_pages)})
    n = len(live)
    movers, holes = [p for p in live if p >= n], [p for p in range(n) if p not in set(live)]
    remap = np.full(n_pages, -1, np.int32)
    for p in live:
        remap[p] = p
    for s, d in zip(movers, holes):
        remap[s] = d
    new = table.copy()
    for b, c in _held(table, lens, page, n_pages):
        new[b, c] = remap[table[b, c]]
    return new, remap, np.array([[s, d, page] for s, d in zip(movers, holes)], np.int32).reshape(-1, 3), n


def copy_tokens(cache, copies):
    """The cache [pages, heads, page, D] after copying tokens 0 .. n - 1 of a page to another for every entry."""
    out = cache.copy()
    for s, d, n in copies:
        if s >= 0 and d >= 0:
            out[d, :, :n] = cache[s, :, :n]
    return out


def lora(x, a, b, ranks, scales, adapters, base):
    """fp64 rows base + scale (x A^T) B^T, and the sum of the products' magnitudes."""
    y, mag = base.astype(np.float64).copy(), np.abs(base.astype(np.float64))
    for m, i in enumerate(adapters):
        if 0 <= i < len(ranks) and ranks[i] > 0:
            r = min(int(ranks[i]), a.shape[1])
            xa, aa, bb = x[m].astype(np.float64), a[i, :r].astype(np.float64), b[i, :, :r].astype(np.float64)
            y[m] += float(scales[i]) * (bb @ (aa @ xa))
            mag[m] += abs(float(scales[i])) * (np.abs(bb) @ (np.abs(aa) @ np.abs(xa)))
    return y, mag
