"""Helpers of the tests of states and paged caches: the definitions, written out row by row in plain Python."""
from __future__ import annotations

import numpy as np


def reorder(old, new, parent, length, beams):
    """old, new: [rows, tokens, ...] numpy arrays (new is old for an in-place call); what `new` has to hold after it."""
    out = new.copy()
    for i, p in enumerate(parent):
        if beams:
            if p == i or p // beams != i // beams or p < 0:
                continue
        elif not 0 <= p < len(old):
            continue
        n = old.shape[1] if length is None else min(max(int(length[p]), 0), old.shape[1])
        out[i, :n] = old[p, :n]
    return out


def fork(table, length, refs, parent, page_size, room, rows):
    """(table, length, refs, copies, status) of a fork; room: one number per new row.  None in copies' place: refused."""
    pages, (n_rows, columns) = len(refs), table.shape
    page = lambda e: 0 <= e < pages                                                                # noqa: E731
    counts = refs.astype(np.int64).copy()
    kids = {}
    for i, p in enumerate(parent):
        if 0 <= p < n_rows:
            kids.setdefault(int(p), []).append(i)
    tokens = [min(max(int(n), 0), columns * page_size) for n in length]
    for r in range(n_rows):
        for e in table[r]:
            if page(e):
                counts[e] -= 1
    new = np.full((rows, columns), -1, np.int64)
    fresh, missing = [], 0
    for i in range(rows):
        p = int(parent[i])
        if not 0 <= p < n_rows:
            continue
        leads, full = kids[p][0] == i, tokens[p] // page_size
        for c in range(columns):
            if leads or c < full:
                new[i, c] = table[p, c]
                if page(new[i, c]):
                    counts[new[i, c]] += 1
        until = -(-(tokens[p] + max(int(room[i]), 0)) // page_size)
        missing += max(0, until - columns)
        for c in range(full, min(until, columns)):
            if not page(new[i, c]):
                fresh.append((i, c, int(table[p, c]) if c == full and tokens[p] % page_size and page(table[p, c]) else None))
    free = [q for q in range(pages) if counts[q] <= 0]
    missing += max(0, len(fresh) - len(free))
    copies = np.full((rows, 2), -1, np.int64)
    if missing:
        old = np.full((rows, columns), -1, np.int64)
        keep = min(rows, n_rows)
        old[:keep] = table[:keep]
        lengths = np.zeros(rows, np.int64)
        lengths[:keep] = length[:keep]
        return old, lengths, refs.astype(np.int64), copies, np.array([(refs <= 0).sum(), min(missing, 2 ** 31 - 1), 0, 0])        # int32
    done = 0
    for (i, c, source), q in zip(fresh, free):
        new[i, c] = q
        counts[q] = 1
        if source is not None:
            copies[done] = source, q
            done += 1
    lengths = np.array([tokens[p] if 0 <= p < n_rows else 0 for p in parent], np.int64)
    return new, lengths, counts, copies, np.array([len(free) - len(fresh), 0, done, 0])


def compact(table, refs, keep):
    """(table, refs, map, moves, status)."""
    pages = len(refs)
    live = [p for p in range(pages) if refs[p] > 0]
    keep = len(live) if keep is None else min(keep, pages)
    where = np.array([p if refs[p] > 0 else -1 for p in range(pages)], np.int64)
    moves, missing = [], max(0, len(live) - keep)
    if not missing:
        moves = list(zip([p for p in live if p >= keep], [p for p in range(keep) if refs[p] <= 0]))
    for a, b in moves:
        where[a] = b
    counts = np.zeros(pages, np.int64)
    for p in live:
        counts[where[p]] = refs[p]
    new = np.where((table >= 0) & (table < pages), where[np.clip(table, 0, pages - 1)], table)
    return new, counts, where, moves, np.array([len(live), missing, len(moves), pages if missing else keep])
