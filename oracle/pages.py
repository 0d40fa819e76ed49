"""Oracle of the pages that several sequences share (NumPy integers): forks, plans and compaction,
row by row from the definitions in ``include/archer_ops.h``."""

from __future__ import annotations

import numpy as np

from .cache4 import pages


def fork(src, dst, length, page_size, table, refs):
    """Returns (table, refs, status) after the forks; inputs unchanged."""
    table, refs = np.array(table), np.array(refs)
    n_rows, width = table.shape
    ok = all(0 <= s < n_rows and 0 <= d < n_rows and 0 <= k <= width * page_size for s, d, k in zip(src, dst, length))
    if not ok or len(set(dst)) != len(dst) or set(dst) & set(src):
        return table, refs, 2
    for s, d, k in zip(src, dst, length):
        for j in range(pages(k, page_size)):
            table[d, j] = table[s, j]
            if 0 <= table[s, j] < len(refs):
                refs[table[s, j]] += 1
    return table, refs, 0


def plan(len_old, len_new, page_size, table, free_pages, pool, refs, slot_rows):
    """Returns (table, free_pages, pool, refs, row_off, slot_map, copy_src, copy_dst, status); inputs unchanged."""
    B, (_, width), n = len(len_old), np.shape(table), len(refs)
    table0, ring0, refs0 = np.array(table), np.array(free_pages), np.array(refs)
    table, ring, refs = table0.copy(), ring0.copy(), refs0.copy()
    head, count = int(pool[0]), int(pool[1])
    off, slots = np.zeros(B + 1, dtype=np.int64), np.full(slot_rows, -1, dtype=np.int64)
    src, dst = np.full(B, -1, dtype=np.int64), np.full(B, -1, dtype=np.int64)

    def refuse(status):
        return table0, ring0, np.array([head, count]), refs0, off * 0, slots * 0 - 1, src * 0 - 1, dst * 0 - 1, status

    if not (0 <= head < n and 0 <= count <= n):
        return refuse(4)
    if any(x < 0 or x > width * page_size for x in list(len_old) + list(len_new)):
        return refuse(2)
    have = [pages(x, page_size) for x in len_old]
    want = [pages(x, page_size) for x in len_new]
    writes = [len_new[b] > len_old[b] and len_old[b] % page_size != 0 for b in range(B)]
    touched = [p for b in range(B) for p in list(table[b, want[b]:have[b]]) + ([table[b, have[b] - 1]] if writes[b] else [])]
    if any(p < 0 or p >= n for p in touched):
        return refuse(4)
    dropped_by = {}
    for b in range(B):
        for j in range(want[b], have[b]):
            refs[table[b, j]] -= 1
            dropped_by[int(table[b, j])] = b          # the last one stays
    # who writes to a page, in row order
    writers = {}
    for b in range(B):
        if writes[b]:
            writers.setdefault(int(table[b, have[b] - 1]), []).append(b)
    copies = set()
    for p, rows in writers.items():
        keeper = rows[-1] if len(rows) == refs[p] else None
        if refs[p] > 1:
            copies |= {b for b in rows if b != keeper}
    given = [[int(p) for p in table[b, want[b]:have[b]] if refs[p] == 0 and dropped_by[int(p)] == b] for b in range(B)]
    takes = sum((b in copies) + max(want[b] - have[b], 0) for b in range(B))
    rows = sum(max(int(len_new[b]) - int(len_old[b]), 0) for b in range(B))
    gives = sum(len(g) for g in given)
    if gives > n - count:
        return refuse(4)
    if takes > count:
        return refuse(1)
    if rows > slot_rows:
        return refuse(3)
    front, back, at = head, head + count, 0
    for b in range(B):
        if b in copies:
            src[b], dst[b] = table[b, have[b] - 1], ring0[front % n]
            refs[src[b]] -= 1
            table[b, have[b] - 1] = dst[b]
            if 0 <= dst[b] < n:
                refs[dst[b]] = 1
            front += 1
        for j in range(have[b], want[b]):
            table[b, j] = ring0[front % n]
            if 0 <= table[b, j] < n:
                refs[table[b, j]] = 1
            front += 1
        for p in given[b]:
            ring[back % n] = p
            back += 1
        for p in range(int(len_old[b]), int(len_new[b])):
            page = table[b, p // page_size]
            slots[at] = page * page_size + p % page_size if 0 <= page < n else -1
            at += 1
        off[b + 1] = at
    return table, ring, np.array([front % n, count - takes + gives]), refs, off, slots, src, dst, 0


def compact(length, page_size, table, refs):
    """Returns (table, refs, free_pages, pool, move_src, move_dst, moves); inputs unchanged."""
    table, refs = np.array(table), np.array(refs)
    n = len(refs)
    U = int((refs > 0).sum())
    moved = [p for p in range(U, n) if refs[p] > 0]
    room = [p for p in range(U) if refs[p] <= 0]
    to = dict(zip(moved, room))
    out = table.copy()
    for b, k in enumerate(length):
        for j in range(pages(min(max(int(k), 0), table.shape[1] * page_size), page_size)):
            out[b, j] = to.get(int(table[b, j]), table[b, j])
    for s, d in to.items():
        refs[d], refs[s] = refs[s], 0
    src, dst, free = (np.full(k, -1, dtype=np.int64) for k in (n // 2, n // 2, n))
    src[:len(moved)], dst[:len(room)] = moved, room
    free[:n - U] = np.arange(U, n)
    return out, refs, free, np.array([0, n - U]), src, dst, len(moved)
