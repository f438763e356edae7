"""Requests that share pages (plain Python and float64), test infrastructure only.

* ``fork_requests`` goes through the requests one by one, with a list as the stack of free
  pages and a dictionary as the copies.  Parity: pinned by hand-worked steps and by the
  conservation of holds (tests/test_sharing_oracle.py).
* ``compact_pages`` pairs sorted lists.  Parity: pinned by hand and by the table's contents.
* ``normed`` is the norm of a head in float64.
* ``prefix_rows`` rewrites each member's row with the pages of its share's first member, so that
  ``oracle.serving.decode_attention`` over them is the definition of the shared attention.
"""
from __future__ import annotations

from typing import Optional, Sequence

import numpy as np

PAGE = 64


def fork_requests(parent, keep: Optional[Sequence[int]], seq_len, page_table, shares, free: Sequence[int],
                  num_pages: int) -> dict:
    """The state afterwards; ``free`` is a list whose last element is taken first; ``copies`` are
    (from, to) pages."""
    B, Hkv, max_blocks = page_table.shape
    old = [n if 0 <= n <= PAGE * max_blocks else 0 for n in map(int, seq_len)]
    src = [int(p) if 0 <= p < B else None for p in parent]
    new = []
    for b in range(B):
        n = 0 if src[b] is None else old[src[b]]
        new.append(n if keep is None or src[b] is None else min(n, max(int(keep[b]), 0)))
    free, wanted, there = list(free), 0, len(free)
    table = np.array(page_table, dtype=np.int64)
    rows, copies, holds = {}, [], {}

    def hold(page, n):
        if 0 <= page < num_pages:
            holds[page] = holds.get(page, 0) + n

    for b in range(B):
        r = src[b]
        if r == b and new[b] == old[b]:
            continue
        rows[b] = None
        for j in range(-(-old[b] // PAGE)):
            for h in range(Hkv):
                hold(int(page_table[b, h, j]), -1)
        if r is None:
            continue
        j, part = divmod(new[b], PAGE)
        copy = False
        if part:
            forks = [x for x in range(B) if src[x] == r]
            here = [x for x in forks if new[x] // PAGE == j and new[x] % PAGE]
            winner = r if r in here else min(here)
            others = any(new[x] // PAGE > j for x in forks)
            pages = [int(page_table[r, h, j]) for h in range(Hkv)]
            copy = others or winner != b or any(0 <= p < num_pages and shares[p] > 0 for p in pages)
        rows[b] = (r, j + (1 if part else 0), copy)
    final = list(new)
    for b in sorted(rows):
        if rows[b] is None:
            continue
        r, blocks, copy = rows[b]
        if copy:
            wanted += Hkv
            if wanted > there:
                final[b] = new[b] - new[b] % PAGE
                copy, blocks = False, blocks - 1
        for h in range(Hkv):
            for j in range(blocks - 1 if copy else blocks):
                table[b, h, j] = page_table[r, h, j]
                hold(int(page_table[r, h, j]), 1)
        if copy:
            for h in range(Hkv):
                table[b, h, blocks - 1] = page = free.pop()
                copies.append((int(page_table[r, h, blocks - 1]), int(page)))
    out = np.array(shares, dtype=np.int64)
    for page, n in holds.items():
        out[page] += n
    gone = np.flatnonzero(out < 0)
    out[gone] = 0
    free += [int(p) for p in gone]
    copies = [(x, y) for x, y in copies if 0 <= x < num_pages and 0 <= y < num_pages]
    return dict(seq_len=np.array(final), page_table=table, page_shares=out, free=free, copies=copies)


def compact_pages(seq_len, page_table, shares, free: Sequence[int], num_pages: int) -> dict:
    B, Hkv, max_blocks = page_table.shape
    empty = {int(p) for p in free if 0 <= p < num_pages}
    used = [p for p in range(num_pages) if p not in empty]
    inside = len(used)
    moved = dict(zip([p for p in used if p >= inside], sorted(p for p in empty if p < inside)))
    new_page = np.array([-1 if p in empty else moved.get(p, p) for p in range(num_pages)])
    table = np.array(page_table, dtype=np.int64)
    for b in range(B):
        n = int(seq_len[b])
        n = n if 0 <= n <= PAGE * max_blocks else 0
        for j in range(-(-n // PAGE)):
            for h in range(Hkv):
                if 0 <= table[b, h, j] < num_pages:
                    table[b, h, j] = new_page[table[b, h, j]]
    out = np.zeros(num_pages, dtype=np.int64)
    for p in used:
        out[new_page[p]] = 0 if shares is None else shares[p]
    return dict(new_page=new_page, page_table=table, page_shares=out, moved=moved,
                free=list(range(num_pages - 1, inside - 1, -1)))


def normed(x: np.ndarray, weight, eps: float) -> np.ndarray:
    """x [.., D] float64; weight [D] as it counts, or None."""
    if weight is None:
        return x
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(eps))) * weight


def prefix_rows(page_table, kv_len, share, share_len):
    """The rows that prefix_decode_attention reads: a member's prefix through its share's first member."""
    B, Hkv, max_blocks = page_table.shape
    rows = np.array(page_table)
    for s, n in enumerate(share_len):
        blocks = min(max(int(n) // PAGE, 0), max_blocks)
        members = [b for b in range(B) if share[b] == s and min(kv_len[b], PAGE * max_blocks) >= PAGE * blocks]
        for b in members:
            rows[b, :, :blocks] = page_table[members[0], :, :blocks]
    return rows
