"""Plain fp64 CPU oracle for the paged cache: block tables from lengths, rotary positions, rows in pages, attention over
pages.

TEST INFRASTRUCTURE ONLY: written from the definitions, one row, token or position at a time; it shares no code with the
HIP path and imports nothing from it.
"""
from __future__ import annotations

import numpy as np

from .decode_oracle import attend


def blocks(n: int, page: int) -> int:
    return -(-n // page)


def page_update(lens, n_new, table, ring, state, page, max_new, rows_per_seq=1):
    """Row after row, as the header describes it.  Returns (lens, table, ring, state, slots, granted), all new."""
    if rows_per_seq > 1:
        return _page_update_together(lens, n_new, table, ring, state, page, max_new, rows_per_seq)
    lens, table, ring = [int(x) for x in lens], np.array(table), np.array(ring)
    total, width = len(ring), table.shape[1]
    head, free = int(state[0]), int(state[1])
    queue = [int(ring[(head + i) % total]) for i in range(free)]
    given, granted, slots = [], [], np.full((len(lens), max_new), -1, dtype=np.int64)
    wanted = 0
    for r, m in enumerate(int(x) for x in n_new):
        held = blocks(lens[r], page)
        if m < 0:
            given += [int(x) for x in table[r, :held]]
            lens[r] = 0
            granted.append(-1)
            continue
        if lens[r] + m > width * page:
            granted.append(0)
            continue
        need = blocks(lens[r] + m, page) - held
        wanted += need
        if need and wanted > free:
            granted.append(0)
            continue
        for j in range(need):
            table[r, held + j] = queue.pop(0)
        for i in range(min(m, max_new)):
            p = lens[r] + i
            slots[r, i] = int(table[r, p // page]) * page + p % page
        lens[r] += m
        granted.append(m)
    taken = free - len(queue)
    for i, x in enumerate(given):
        ring[(head + free + i) % total] = x
    return (np.array(lens, np.int32), table, ring, np.array([(head + taken) % total, len(queue) + len(given)], np.int64), slots,
            np.array(granted, np.int32))


def _page_update_together(lens, n_new, table, ring, state, page, max_new, L):
    """The sequences that can be granted are found first; the others ask for nothing, and the rows go their way one by one."""
    asked, wanted, refused = np.array(n_new), 0, set()
    for s in range(0, len(lens), L):
        rows = [r for r in range(s, s + L) if asked[r] >= 0]
        if any(int(lens[r]) + int(asked[r]) > table.shape[1] * page for r in rows):
            refused |= set(rows)
            continue
        need = sum(blocks(int(lens[r]) + int(asked[r]), page) - blocks(int(lens[r]), page) for r in rows)
        wanted += need
        if need and wanted > int(state[1]):
            refused |= set(rows)
    return page_update(lens, [0 if r in refused else m for r, m in enumerate(asked)], table, ring, state, page, max_new)


def rotate(x, positions, inv_freq, axis=None, interleaved=False, inverse=False):
    """x [T][H][d]; positions [axes][T]; pair p turns by positions[axis[p]][t] * inv_freq[p]."""
    x = np.array(x, dtype=np.float64)
    half = len(inv_freq)
    for p in range(half):
        ang = positions[0 if axis is None else axis[p]].astype(np.float64) * float(inv_freq[p])
        c, s = np.cos(ang)[:, None], np.sin(ang)[:, None] * (-1.0 if inverse else 1.0)
        i, j = (2 * p, 2 * p + 1) if interleaved else (p, p + half)
        a, b = x[:, :, i].copy(), x[:, :, j].copy()
        x[:, :, i], x[:, :, j] = a * c - b * s, b * c + a * s
    return x


def gather(pages, table_row, n):
    """The first n positions of one row: pages [n_pages][Hkv][page][d] -> [Hkv][n][d]; pages that do not exist leave
    their positions out."""
    page = pages.shape[2]
    parts = []
    for b in range(blocks(n, page)):
        at = int(table_row[b])
        if 0 <= at < len(pages):
            parts.append(pages[at][:, :min(page, n - b * page)])
    return np.concatenate(parts, axis=1) if parts else np.zeros((pages.shape[1], 0, pages.shape[3]))


def attention(q, k_pages, v_pages, table, lens, scale=None):
    """q [R][Hq][d] -> [R][Hq][d]; zeros for a row without positions."""
    out = np.zeros(q.shape, dtype=np.float64)
    group = q.shape[1] // k_pages.shape[1]
    most = table.shape[1] * k_pages.shape[2]
    for r in range(len(q)):
        n = min(max(int(lens[r]), 0), most)
        k, v = gather(k_pages, table[r], n), gather(v_pages, table[r], n)
        for h in range(q.shape[1]):
            if k.shape[1]:
                out[r, h] = attend(q[r, h], k[h // group], v[h // group], scale)
    return out
