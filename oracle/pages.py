"""Pages that several sequences hold, one entry at a time, after the description in include/fspad.h -- TEST INFRASTRUCTURE, as the rest of this
package. Every function returns copies; its arguments stay as they are."""
from __future__ import annotations

import numpy as np


def _stack(free, n_free):
    return int(min(max(int(np.asarray(n_free).reshape(-1)[0]), 0), len(free)))


def _held(kv_len, P, width):
    return [min(-(-max(int(x), 0) // P), width) for x in kv_len]


def fork(src, dst, kv_len, table, free, n_free, shared, P, n_tokens=None):
    """(copy_src, copy_dst, kv_len_out, n_free_out, shared_out, granted, table)"""
    table, shared, lens = np.array(table, np.int64), np.array(shared, np.int64), np.array(kv_len, np.int64)
    (B, width), n_pages, top = table.shape, len(free), _stack(free, n_free)
    before, named, asked = lens.copy(), set(), 0
    rows = table.copy()
    copy_src, copy_dst, granted = (np.full(len(src), x, np.int64) for x in (-1, -1, 0))
    for f, (s, d) in enumerate(zip(src, dst)):
        s, d = int(s), int(d)
        first = d not in named
        named.add(d)
        if not (0 <= s < B and 0 <= d < B) or s == d or not first or before[d] > 0:
            continue
        have = max(int(before[s]), 0)
        n = have if n_tokens is None else int(n_tokens[f])
        if n < 0 or n > have or n > width * P:
            continue
        if n % P:
            asked += 1
            if asked > top:
                continue
            new = int(free[top - asked])
            table[d, n // P] = new
            if 0 <= rows[s, n // P] < n_pages and 0 <= new < n_pages:
                copy_src[f], copy_dst[f] = rows[s, n // P], new
        for i in range(n // P):
            table[d, i] = rows[s, i]
            if 0 <= rows[s, i] < n_pages:
                shared[rows[s, i]] += 1
        granted[f], lens[d] = 1, n
    return copy_src, copy_dst, lens, np.array([top - min(asked, top)]), shared, granted, table


def release(ended, kv_len, table, free, n_free, shared, P):
    """(kv_len_out, n_free_out, shared_out, free)"""
    free, lens = np.array(free, np.int64), np.array(kv_len, np.int64)
    holders = np.maximum(np.array(shared, np.int64), 0) + 1
    n_pages, top = len(free), _stack(free, n_free)
    gone = set()
    for b, n in enumerate(_held(kv_len, P, np.shape(table)[1])):
        if not ended[b]:
            continue
        lens[b] = 0
        for page in np.asarray(table)[b, :n]:
            if 0 <= page < n_pages:
                holders[page] -= 1
                if holders[page] <= 0:
                    gone.add(int(page))
    for page in sorted(gone):
        holders[page] = 1
        if top < n_pages:
            free[top] = page
            top += 1
    return lens, np.array([top]), holders - 1, free


def compact(kv_len, table, free, n_free, shared, P):
    """(copy_src, copy_dst, table, free, shared)"""
    table, shared, n_pages, top = np.array(table, np.int64), np.array(shared, np.int64), len(free), _stack(free, n_free)
    keep = n_pages - top
    stack = {int(x) for x in np.asarray(free)[:top] if 0 <= x < n_pages}
    movers, holes = [p for p in range(keep, n_pages) if p not in stack], [p for p in range(keep) if p in stack]
    to = dict(zip(movers, holes))
    copy_src, copy_dst = np.full(n_pages // 2, -1, np.int64), np.full(n_pages // 2, -1, np.int64)
    for i, (a, b) in enumerate(to.items()):
        copy_src[i], copy_dst[i] = a, b
        shared[b], shared[a] = shared[a], 0
    for b, n in enumerate(_held(kv_len, P, table.shape[1])):
        for i in range(n):
            table[b, i] = to.get(int(table[b, i]), table[b, i])
    return copy_src, copy_dst, table, np.array([n_pages - 1 - i if i < top else -1 for i in range(n_pages)]), shared


def copy(pages, copy_src, copy_dst):
    out = np.array(pages)
    for a, b in zip(copy_src, copy_dst):
        if 0 <= a < len(pages) and 0 <= b < len(pages):
            out[b] = pages[a]
    return out
