"""Oracle of the paged cache in 8 bits (test infrastructure only).

The format: pools [num_blocks, Hkv, block_size, D] of e4m3 codes (OCP 8-bit float: sign, 4
exponent bits of bias 7, 3 fraction bits, no infinities, 0x7F / 0xFF not a number) and one
exponent byte e per 32 positions of a page and head; a code c stands for value(c) * 2^(e - 127).

What the writers compute, per sequence, touched group of 32 positions, head, and K or V:

  a    the largest size among the group's new values (of those that are finite)
  e(a) the least e of [16, 247] with a <= 448 * 2^(e - 127)
  e'   max(e(a), the group's byte) if the group holds older rows of the sequence, else e(a)
  new codes      nearest(value * 2^(127 - e')), where e' = 247 of sizes up to 240: the next code
                 would stand for 2^128, which a bf16 number does not reach
  older codes    nearest(value(code) * 2^(byte - e')), unchanged where e' is the byte

nearest: to the nearest e4m3 value, ties to the even code, 448 at most.  An infinity or NaN becomes
code 0x7F or 0xFF.
"""
from __future__ import annotations

import numpy as np

GROUP, EMIN, EMAX = 32, 16, 247


def _table():
    t = np.empty(256)
    for c in range(256):
        exp, frac = (c >> 3) & 15, c & 7
        v = (8 + frac) * 2.0 ** (exp - 10) if exp else frac * 2.0 ** -9
        t[c] = np.nan if exp == 15 and frac == 7 else (-v if c & 128 else v)
    return t


VALUES = _table()          # code -> number
_POSITIVE = VALUES[:127]   # increasing
_MIDDLE = (_POSITIVE[1:] + _POSITIVE[:-1]) / 2


def nearest(x):
    """Codes of the e4m3 values nearest to x (finite)."""
    x = np.asarray(x, np.float64)
    a = np.abs(x)
    code = np.searchsorted(_MIDDLE, a, side="left")     # ties: the lower one,
    tie = (code < 126) & (a == _MIDDLE[np.minimum(code, 125)])
    code = code + (tie & (code % 2 == 1))               # or the upper one if that is even
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def codes_at(x, e):
    """Codes of the numbers x at exponents e (of x's shape, or to be broadcast to it)."""
    limit = np.where(np.asarray(e) == EMAX, 240.0, 448.0)
    c = nearest(np.clip(_finite(x) * np.exp2(127.0 - e), -limit, limit))
    return np.where(np.isfinite(x), c, 0x7F + 128 * np.signbit(x)).astype(np.uint8)


def _finite(x):
    return np.where(np.isfinite(x), x, 0.0)


def decode(codes, exps):
    """Codes [..., rows, D] and exponents [..., rows / 32] -> the numbers they stand for."""
    scale = np.exp2(np.repeat(np.asarray(exps, np.float64) - 127, GROUP, axis=-1))
    return VALUES[np.asarray(codes)] * scale[..., None]


def encode(x):
    """x [..., rows, D], rows a multiple of 32 -> (codes, exponents)."""
    x = np.asarray(x, np.float64)
    g = x.reshape(x.shape[:-2] + (-1, GROUP, x.shape[-1]))
    e = exponent(np.abs(_finite(g)).max((-1, -2)))
    return codes_at(g, e[..., None, None]).reshape(x.shape), e.astype(np.uint8)


def exponent(a):
    """e(a), by trying every e."""
    a = np.asarray(a, np.float64)
    limits = 448 * np.exp2(np.arange(EMIN, EMAX + 1) - 127.0)
    return np.minimum(EMIN + np.searchsorted(limits, a, side="left"), EMAX)


def append(pool, exps, table, kv_len, new, n_new):
    """new [B, T, Hkv, D]: row j < n_new[b] goes to position kv_len[b] + j of sequence b.  A
    sequence whose n_new is outside [0, T] or that lacks a page for one of its rows is left as it is.
    Returns new copies (pool, exps)."""
    pool, exps = np.array(pool, copy=True), np.array(exps, copy=True)
    bs = pool.shape[2]
    for b in range(len(kv_len)):
        kv, n = int(kv_len[b]), int(n_new[b])
        if not 0 <= n <= new.shape[1] or kv < 0 or kv + n > table.shape[1] * bs:
            continue
        if not all(0 <= p < len(pool) for p in table[b, kv // bs:-(-(kv + n) // bs)]):
            continue
        for lo in range(kv // GROUP * GROUP, kv + n, GROUP):
            if n == 0:
                break
            page, row = int(table[b, lo // bs]), lo % bs
            old = max(0, kv - lo)                                  # older rows of the group
            hi = min(lo + GROUP, kv + n) - lo
            val = np.asarray(new[b, lo + old - kv:lo + hi - kv], np.float64).transpose(1, 0, 2)
            e = exponent(np.abs(_finite(val)).max((1, 2)))
            if old:
                was = exps[page, :, row // GROUP].astype(np.int64)
                e = np.maximum(e, was)
                v = VALUES[pool[page, :, row:row + old]] * np.exp2((was - e).astype(float))[:, None, None]
                pool[page, :, row:row + old] = nearest(v)
            pool[page, :, row + old:row + hi] = codes_at(val, e[:, None, None])
            exps[page, :, row // GROUP] = e
    return pool, exps


def commit(pool, exps, table, kv_len, tree, path, accept_len):
    """The accepted path's rows of tree [B, N, Hkv, D] are appended.  A sequence that failed
    acceptance (accept_len < 1), has accept_len above the path's width, names a node outside the
    tree or lacks a page is left as it is."""
    B, N = tree.shape[:2]
    path, n = np.asarray(path), np.array(accept_len, np.int64)
    for b in range(B):
        ok = 1 <= n[b] <= path.shape[1] and ((path[b, :n[b]] >= 0) & (path[b, :n[b]] < N)).all()
        n[b] = n[b] if ok else 0
    rows = np.stack([tree[b][np.clip(path[b], 0, N - 1)] for b in range(B)])
    return append(pool, exps, table, kv_len, rows, n)


def gather(pool, exps, table, n_blocks):
    """The first n_blocks pages of every sequence as a contiguous cache of numbers,
    [B, n_blocks * block_size, Hkv, D]."""
    values = decode(pool, exps)
    t = np.clip(np.asarray(table)[:, :n_blocks], 0, len(pool) - 1)
    x = values[t]                                                   # [B, pages, Hkv, rows, D]
    B, P, H, R, D = x.shape
    return x.transpose(0, 1, 3, 2, 4).reshape(B, P * R, H, D)
