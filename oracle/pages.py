"""Oracle of the page calls (test infrastructure only): whose page is whose, written out as loops.

State: table [B, max_blocks] (a row's pages first, -1 behind them), kv_len [B], ref [num_blocks],
how many rows name a page.  New pages are the free ones (ref <= 0) of the lowest numbers.  Every
function returns new copies."""
from __future__ import annotations

import numpy as np


def _state(*arrays):
    return [np.array(a, np.int64, copy=True) for a in arrays]


def reserve(n_rows, table, kv_len, ref, block_size):
    """-> (ok, table, ref)."""
    table, kv, ref = _state(table, kv_len, ref)
    B, mb = table.shape
    free = [p for p in range(len(ref)) if ref[p] <= 0]
    ok = np.zeros(B, np.int64)
    asked = 0
    for b in range(B):
        n = int(n_rows[b])
        if n < 0 or kv[b] < 0 or kv[b] + n > mb * block_size:
            continue
        entries = [j for j in range(-(-int(kv[b] + n) // block_size)) if table[b, j] < 0]
        mine = free[asked:asked + len(entries)]
        asked += len(entries)
        if len(mine) < len(entries):
            continue
        ok[b] = 1
        for j, p in zip(entries, mine):
            table[b, j] = p
            ref[p] = 1
    return ok, table, ref


def fork(src, dst, table, kv_len, ref, block_size):
    """-> (ok, copy_src, copy_dst, table, kv_len, ref)."""
    before, _ = _state(table, ref)
    table, kv, ref = _state(table, kv_len, ref)
    B, mb = table.shape
    free = [p for p in range(len(ref)) if ref[p] <= 0]
    n = len(src)
    ok, cs, cd = np.zeros(n, np.int64), np.full(n, -1), np.full(n, -1)
    taken = 0
    for i in range(n):
        s, d = int(src[i]), int(dst[i])
        if not (0 <= s < B and 0 <= d < B) or before[d, 0] >= 0 or d in list(dst[:i]) or s in list(dst):
            continue
        if not 0 <= kv[s] <= mb * block_size:
            continue
        full, part = divmod(int(kv[s]), block_size)
        mine = before[s, :full + (part > 0)]
        if ((mine < 0) | (mine >= len(ref))).any():
            continue
        if part:
            taken += 1
            if taken > len(free):
                continue
            cs[i], cd[i] = before[s, full], free[taken - 1]
        ok[i] = 1
        table[d] = -1
        table[d, :full] = before[s, :full]
        for p in before[s, :full]:
            ref[p] += 1
        if part:
            table[d, full] = cd[i]
            ref[cd[i]] = 1
        kv[d] = kv[s]
    return ok, cs, cd, table, kv, ref


def free(seqs, table, kv_len, ref):
    """-> (table, kv_len, ref)."""
    table, kv, ref = _state(table, kv_len, ref)
    for b in seqs:
        if 0 <= b < len(table):
            for p in table[b][table[b] >= 0]:
                ref[p] -= 1
            table[b] = -1
            kv[b] = 0
    return table, kv, ref


def compact(table, ref):
    """-> (live pages, copy_src, copy_dst, table, ref)."""
    table, ref = _state(table, ref)
    live = int((ref > 0).sum())
    away = [p for p in range(len(ref) - 1, live - 1, -1) if ref[p] > 0]
    into = [p for p in range(live) if ref[p] <= 0]
    cs, cd = np.full(len(ref) // 2, -1), np.full(len(ref) // 2, -1)
    cs[:len(away)], cd[:len(into)] = away, into
    for s, d in zip(away, into):
        table[table == s] = d
        ref[d], ref[s] = ref[s], 0
    return live, cs, cd, table, ref
