"""Pins of the 8-bit cache's oracle and of the page calls' one: torch's own e4m3 conversion, the
rules written out, and what must hold whatever the calls did before."""
import numpy as np
import pytest
import torch

import oracle
from oracle import kv_fp8, pages


def test_codes_are_e4m3():
    codes = np.arange(256, dtype=np.uint8)
    ref = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(kv_fp8.VALUES, ref)
    finite = (codes & 0x7F) != 0x7F
    np.testing.assert_array_equal(kv_fp8.nearest(ref[finite]), codes[finite])  # zeros keep their signs


def test_nearest_is_the_library_cast():
    rng = np.random.default_rng(1)
    x = rng.standard_normal(200000) * np.exp2(rng.integers(-14, 9, 200000))
    pos = kv_fp8.VALUES[:127]
    mid = (pos[1:] + pos[:-1]) / 2
    x = np.concatenate([x, pos, -pos, mid, -mid, np.nextafter(mid, 1e9), np.nextafter(mid, 0)])
    x = np.clip(x, -448, 448).astype(np.float32)
    ref = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(kv_fp8.nearest(x), ref)
    assert kv_fp8.nearest([449.0, 1e9, -1e9]).tolist() == [0x7E, 0x7E, 0xFE]


def test_exponent_is_the_least_that_reaches():
    rng = np.random.default_rng(2)
    a = np.concatenate([np.exp2(rng.uniform(-130, 127, 500)), 448 * np.exp2(np.arange(-115.0, 119.0)),
                        np.nextafter(448 * np.exp2(np.arange(-115.0, 119.0)), np.inf), [0.0]])
    e = kv_fp8.exponent(a)
    limit = lambda e: 448 * np.exp2(e - 127.0)
    assert ((a <= limit(e)) | (e == kv_fp8.EMAX)).all()
    assert ((e == kv_fp8.EMIN) | (a > limit(e - 1))).all()


def test_round_trip_error():
    """A value comes back within half a step of its own: 2^-4 of it, or 2^-10 steps of the smallest
    codes' scale."""
    rng = np.random.default_rng(3)
    x = rng.standard_normal((3, 2, 96, 64)) * np.exp2(rng.integers(-8, 8, (3, 2, 96, 64)))
    codes, exps = kv_fp8.encode(x)
    back = kv_fp8.decode(codes, exps)
    scale = np.exp2(np.repeat(exps.astype(float) - 127, 32, -1))[..., None]
    assert (np.abs(back - x) <= np.maximum(np.abs(x) * 2.0 ** -4, scale * 2.0 ** -10)).all()


def test_append_by_rows():
    """Rows one at a time or at once: the same exponents, and numbers apart by the roundings that
    re-scaling a row costs, half a step each; other pages and rows are left alone."""
    rng = np.random.default_rng(4)
    H, D, bs, mb = 2, 64, 32, 3
    table = rng.permutation(8)[:2 * mb].reshape(2, mb)
    pool = rng.integers(0, 127, (8, H, bs, D)).astype(np.uint8)
    exps = rng.integers(100, 130, (8, H, 1)).astype(np.uint8)
    kv, T = np.array([5, 40]), 50
    new = rng.standard_normal((2, T, H, D)) * np.exp2(rng.integers(-3, 3, (2, T, H, 1)))
    n = np.array([T, 31])
    one = kv_fp8.append(pool, exps, table, kv, new, n)
    two, at = (pool, exps), kv.copy()
    for j in range(T):
        step = (j < n).astype(int)
        two = kv_fp8.append(*two, table, at, new[:, j:j + 1], step)
        at += step
    np.testing.assert_array_equal(one[1], two[1])
    a, b = kv_fp8.decode(*one), kv_fp8.decode(*two)
    unit = np.exp2(np.repeat(one[1].astype(float) - 127, 32, -1))[..., None]
    # a row is rounded once, then at most once per step up of its group's exponent (here 6)
    tol = 7 * np.maximum(np.maximum(np.abs(a), np.abs(b)) * 2.0 ** -4, unit * 2.0 ** -10)
    assert (np.abs(a - b) <= tol).all()
    touched = np.zeros((8, bs), bool)
    for s in range(2):
        for t in range(kv[s] // 32 * 32, kv[s] + n[s]):
            touched[table[s, t // bs], t % bs] = True
    keep = ~touched[:, None, :, None] & np.ones_like(pool, bool)
    np.testing.assert_array_equal(one[0][keep], pool[keep])
    # what was written is what was given, rounded at its group's scale
    got = kv_fp8.gather(*one, table, mb)
    for s in range(2):
        x = new[s, :n[s]]
        y = got[s, kv[s]:kv[s] + n[s]]
        e = np.array([[one[1][table[s, t // bs], h, 0] for h in range(H)]
                      for t in range(kv[s], kv[s] + n[s])], float)
        assert (np.abs(x - y) <= np.maximum(np.abs(x) * 2.0 ** -4, np.exp2(e - 137)[..., None])).all()


def test_append_refusals_and_commit():
    rng = np.random.default_rng(5)
    H, D, bs, mb = 1, 64, 32, 2
    table = np.arange(8).reshape(4, mb)
    pool = rng.integers(0, 127, (8, H, bs, D)).astype(np.uint8)
    exps = np.full((8, H, 1), 120, np.uint8)
    new = rng.standard_normal((4, 9, H, D))
    out = kv_fp8.append(pool, exps, table, [60, -1, 0, 0], new, [5, 1, 10, -1])
    assert (out[0] == pool).all() and (out[1] == exps).all()
    path = np.array([[0, 3, 8, -1], [0, 1, -1, -1], [0, 9, 1, 2], [0, 1, 2, 3]])
    n = [3, 0, 2, 5]
    kv = [30, 0, 0, 0]
    got = kv_fp8.commit(pool, exps, table, kv, new, path, n)
    want = kv_fp8.append(pool, exps, table, kv, new[:, [0, 3, 8]], [3, 0, 0, 0])
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])


def test_gather_is_the_cache_of_the_16_bit_oracle():
    """Over pages of one head size the sequences' rows come out as gather_paged orders them."""
    rng = np.random.default_rng(6)
    pool = rng.integers(0, 127, (6, 3, 32, 64)).astype(np.uint8)
    exps = np.full((6, 3, 1), 127, np.uint8)
    table = rng.permutation(6).reshape(2, 3)
    rows = kv_fp8.VALUES[pool].transpose(0, 2, 1, 3)          # [pages, rows, heads, D]
    np.testing.assert_array_equal(kv_fp8.gather(pool, exps, table, 3), oracle.gather_paged(rows, table, 3))


def consistent(table, ref, lens=None, bs=1):
    """Every page's count is the number of entries that name it; pages come first in a row."""
    counts = np.bincount(table[table >= 0].ravel(), minlength=len(ref))
    np.testing.assert_array_equal(counts, ref)
    held = (table >= 0).sum(1)
    for b in range(len(table)):
        assert (table[b, :held[b]] >= 0).all()
        if lens is not None:
            assert lens[b] <= held[b] * bs


@pytest.mark.parametrize("seed", range(8))
def test_page_calls_keep_their_books(seed):
    """Whatever calls follow each other: the counts are the entries', no page is handed out twice, a
    compacted pool's live pages are its first ones, and a copy has one source and one destination."""
    rng = np.random.default_rng(seed)
    B, mb, bs, nb = 6, 5, 32, 17
    table, kv, ref = np.full((B, mb), -1), np.zeros(B, int), np.zeros(nb, int)
    text = {}                                                # page -> what it holds (a row list)
    seqs = [[] for _ in range(B)]

    def read(b):
        return [text[table[b, t // bs]][t % bs] for t in range(kv[b])]

    for step in range(60):
        kind = rng.integers(4)
        if kind == 0:
            n = rng.integers(-1, 70, B)
            ok, table, ref = pages.reserve(n, table, kv, ref, bs)
            for b in np.flatnonzero(ok):
                for j in range(n[b]):
                    t = kv[b] + j
                    # a row is only written into a page of its own
                    if ref[table[b, t // bs]] == 1:
                        text.setdefault(table[b, t // bs], [None] * bs)[t % bs] = (step, b, j)
                        seqs[b].append((step, b, j))
                    else:
                        n[b] = j
                        break
                kv[b] += n[b]
        elif kind == 1:
            src, dst = rng.integers(-1, B + 1, 3), rng.integers(-1, B + 1, 3)
            ok, cs, cd, table, kv, ref = pages.fork(src, dst, table, kv, ref, bs)
            for i in np.flatnonzero(ok):
                if cs[i] >= 0:
                    text[cd[i]] = list(text[cs[i]])
                seqs[dst[i]] = list(seqs[src[i]])
        elif kind == 2:
            gone = rng.integers(-1, B + 1, 1)
            table, kv, ref = pages.free(gone, table, kv, ref)
            for b in gone:
                if 0 <= b < B:
                    seqs[b] = []
        else:
            live, cs, cd, table, ref = pages.compact(table, ref)
            moved = cs >= 0
            assert len(set(cs[moved]) | set(cd[moved])) == 2 * moved.sum()
            for s, d in zip(cs[moved], cd[moved]):
                text[d] = list(text.get(s, [None] * bs))
            assert (ref[:live] > 0).all() and (ref[live:] <= 0).all()
        consistent(table, ref, kv, bs)
        for b in range(B):
            assert read(b) == seqs[b]


def test_the_largest_numbers_stay_numbers():
    """At the largest exponent a code still stands for a number that bf16 and fp32 hold: the largest
    one of those, 240 * 2^120, for all sizes above 232 * 2^120 (halfway between codes 224 and 240; the
    even one is 224)."""
    bits = np.arange(0x7F60, 0x7F80, dtype=np.uint16)
    x = oracle.decode_bf16(np.concatenate([bits, bits | 0x8000])).reshape(1, 1, 64, 1).repeat(64, -1)
    codes, exps = kv_fp8.encode(x)
    back = kv_fp8.decode(codes, exps)
    assert (exps == 247).all() and np.isfinite(back.astype(np.float32)).all()
    assert (back.astype(np.float32).view(np.uint32) & 0xFFFF == 0).all()
    size = np.abs(x)
    assert (np.abs(back)[size > 232 * 2.0 ** 120] == 240 * 2.0 ** 120).all()
    assert (np.abs(back - x) <= 2.0 ** -4 * size).all() and (np.sign(back) == np.sign(x)).all()
    # rows in a cache whose exponents are smaller: older codes halve at least, so they fit as well
    pool, e = np.full((1, 1, 32, 64), 0x7E, np.uint8), np.full((1, 1, 1), 246, np.uint8)
    pool, e = kv_fp8.append(pool, e, np.zeros((1, 1), int), [16], x[:, :, 16:32].transpose(0, 2, 1, 3), [16])
    assert e[0, 0, 0] == 247 and (kv_fp8.VALUES[pool[0, 0, :16]] == 224).all()
    assert (np.abs(kv_fp8.VALUES[pool]) <= 240).all()


def test_what_is_no_number_costs_its_group_nothing_else():
    rng = np.random.default_rng(6)
    pool, exps = rng.integers(0, 127, (2, 1, 32, 64)).astype(np.uint8), np.full((2, 1, 1), 120, np.uint8)
    new = rng.standard_normal((1, 20, 1, 64))
    bad = new.copy()
    at = [(0, 3, 0, 5), (0, 3, 0, 6), (0, 11, 0, 7), (0, 19, 0, 63)]
    for i, x in zip(at, (np.inf, -np.inf, np.nan, -np.nan)):
        bad[i], new[i] = x, 0.0
    table = np.array([[1, 0]])
    want = kv_fp8.append(pool, exps, table, [7], new, [20])
    got = kv_fp8.append(pool, exps, table, [7], bad, [20])
    codes = [got[0][1, 0, 7 + i[1], i[3]] for i in at]
    assert codes[:2] == [0x7F, 0xFF] and all(c & 0x7F == 0x7F for c in codes)
    for i in at:
        got[0][1, 0, 7 + i[1], i[3]] = 0
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])


def test_a_fork_needs_every_page_of_its_source():
    """No trace of a fork whose source lacks a page: the partly filled one, a full one, one outside
    the pool; pages behind its rows do not matter."""
    table = np.full((8, 4), -1)
    table[0], table[1], table[2] = [0, 1, -1, -1], [0, -1, 2, -1], [3, 9, -1, -1]
    table[3] = [3, 4, -1, 77]
    kv, ref = np.array([70, 70, 64, 64, 0, 0, 0, 0]), np.array([2, 1, 1, 2, 1, 0, 0, 0])
    src, dst = [0, 1, 2, 3], [4, 5, 6, 7]
    ok, cs, cd, t, k, r = pages.fork(src, dst, table, kv, ref, 32)
    assert ok.tolist() == [0, 0, 0, 1] and (cs == -1).all() and (cd == -1).all()
    assert (t[4:7] == -1).all() and t[7].tolist() == [3, 4, -1, -1] and k[4:].tolist() == [0, 0, 0, 64]
    assert r.tolist() == [2, 1, 1, 3, 2, 0, 0, 0]
