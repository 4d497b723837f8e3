"""GPU parity of the page calls against the oracle's loops: tables, lengths, counts, lists and the
contents of pools, all exactly."""
import numpy as np
import pytest
import torch

from oracle import pages as ref_pages
from paper_2606_18394_amd import compact_pages, copy_pages, fork_pages, free_pages, reserve_pages
from helpers import dev_i32

pytestmark = pytest.mark.gpu


def state(rng, B, mb, nb, bs, fill, ahead=0.3):
    """Rows with some of the pool's pages, partly filled last ones, pages beyond kv_len in some."""
    order = rng.permutation(nb)
    bt = np.full((B, mb), -1, np.int64)
    kv = np.zeros(B, np.int64)
    at = 0
    for b in range(B):
        u = int(rng.integers(0, mb + 1)) if rng.random() > 0.2 else 0
        if at + u > int(nb * fill):
            u = 0
        bt[b, :u] = order[at:at + u]
        at += u
        used = max(0, u - (1 if rng.random() < ahead else 0))
        kv[b] = 0 if used == 0 else used * bs - (int(rng.integers(0, bs)) if rng.random() < 0.7 else 0)
    ref = np.zeros(nb, np.int64)
    np.add.at(ref, bt[bt >= 0], 1)
    return bt, kv, ref


def pool_set(rng, nb):
    """Pools of several types and page sizes: many pieces, one, odd bytes, one byte."""
    return [torch.from_numpy(rng.integers(0, 256, size=(nb,) + s).astype(np.uint8)).cuda().view(t)
            for s, t in (((2, 64, 256), torch.uint8), ((32, 16), torch.bfloat16), ((7, 3), torch.uint8),
                         ((1,), torch.uint8), ((4,), torch.int32), ((33, 1000), torch.uint8))]


def moved(pools, src, dst):
    want = [p.clone() for p in pools]
    for s, d in zip(src, dst):
        if s >= 0 and d >= 0:
            for w, p in zip(want, pools):
                w[int(d)] = p[int(s)]
    return want


def same(pools, want):
    return all(torch.equal(p.view(torch.uint8), w.view(torch.uint8)) for p, w in zip(pools, want))


def eq(t, a):
    return np.array_equal(t.cpu().numpy(), a)


SHAPES = [
    # (B, max_blocks, num_blocks, block_size, share of the pool in use)
    (1, 1, 1, 32, 1.0), (2, 3, 5, 32, 0.8), (7, 5, 40, 64, 0.9), (64, 9, 300, 256, 0.7),
    (300, 20, 9000, 32, 1.0), (4096, 3, 20011, 64, 0.5), (50, 700, 50000, 32, 0.9),
]


@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_reserve(case, offset):
    B, mb, nb, bs, fill = SHAPES[case]
    rng = np.random.default_rng(5000 + case)
    bt, kv, ref = state(rng, B, mb, nb, bs, fill)
    # few pages are left over, so that some sequences go without
    free = np.flatnonzero(ref == 0)
    ref[rng.permutation(free)[:int(len(free) * (0.5 if case % 2 else 0.0))]] = 1
    n = rng.integers(-1, 3 * bs, size=B)
    n[rng.random(B) < 0.2] = 0
    n[rng.random(B) < 0.05] = mb * bs + 1
    print(f"reserve {SHAPES[case]}", flush=True)
    ok, et, er = ref_pages.reserve(n, bt, kv, ref, bs)
    buf = dev_i32(np.concatenate([np.zeros(offset, np.int64), ref]))
    dt, dr, dk = dev_i32(bt), buf[offset:], dev_i32(kv)
    got = reserve_pages(dev_i32(n), dt, dk, dr, bs)
    assert eq(got, ok) and eq(dt, et) and eq(dr, er) and eq(dk, kv)


@pytest.mark.parametrize("short", [False, True])
@pytest.mark.parametrize("case", range(1, len(SHAPES)))
def test_fork(case, short):
    B, mb, nb, bs, fill = SHAPES[case]
    if nb > 20000:
        nb = 20000
    rng = np.random.default_rng(5100 + case)
    bt, kv, ref = state(rng, B, mb, nb, bs, fill * 0.8)
    if short:
        free = np.flatnonzero(ref == 0)
        ref[free[2:]] = 1
    n = min(1024, B)
    empty = np.flatnonzero(bt[:, 0] < 0)
    src = rng.integers(-1, B + 1, size=n)
    dst = rng.permutation(np.concatenate([empty, rng.integers(-1, B + 1, size=n)]))[:n]  # some twice
    print(f"fork {SHAPES[case]} n={n}", flush=True)
    ok, cs, cd, et, ek, er = ref_pages.fork(src, dst, bt, kv, ref, bs)
    pools = pool_set(rng, nb) if nb <= 9000 else pool_set(rng, nb)[2:5]
    want = moved(pools, cs, cd)
    dt, dk, dr = dev_i32(bt), dev_i32(kv), dev_i32(ref)
    got = fork_pages(dev_i32(src), dev_i32(dst), dt, dk, dr, bs, pools)
    assert eq(got[0], ok) and eq(got[1], cs) and eq(got[2], cd)
    assert eq(dt, et) and eq(dk, ek) and eq(dr, er) and same(pools, want)
    assert len(empty) == 0 or ok.any() or case < 3


@pytest.mark.parametrize("nb", [8192, 30011, 65537])
def test_pages_far_apart(nb):
    """A pool whose counts take several passes, most of them without a free page: the first, the last
    and the ones about a pass's end."""
    left = np.array(sorted({0, 8190, 8191, 8192, 8193, nb - 2, nb - 1} & set(range(nb))))
    ref = np.ones(nb, np.int64)
    ref[left] = 0
    B, mb, bs = 12, 4, 32
    for short in (0, 3):
        bt, kv = np.full((B, mb), -1, np.int64), np.zeros(B, np.int64)
        n = np.zeros(B, np.int64)
        n[:len(left) + short] = 5
        ok, et, er = ref_pages.reserve(n, bt, kv, ref, bs)
        dt, dk, dr = dev_i32(bt), dev_i32(kv), dev_i32(ref)
        got = reserve_pages(dev_i32(n), dt, dk, dr, bs)
        assert eq(got, ok) and eq(dt, et) and eq(dr, er) and ok.sum() == len(left) + B - min(B, len(left) + short)
        # forks of a row with one partly filled page
        bt[0, 0], kv[0] = 5, 7
        src, dst = np.zeros(len(left) + short, np.int64), np.arange(1, len(left) + short + 1)
        want = ref_pages.fork(src, dst, bt, kv, ref, bs)
        dt, dk, dr = dev_i32(bt), dev_i32(kv), dev_i32(ref)
        got = fork_pages(dev_i32(src), dev_i32(dst), dt, dk, dr, bs)
        assert all(eq(x, y) for x, y in zip(list(got) + [dt, dk, dr], want))
        assert want[0].sum() == len(left)


@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_free(case):
    B, mb, nb, bs, fill = SHAPES[case]
    rng = np.random.default_rng(5200 + case)
    bt, kv, ref = state(rng, B, mb, nb, bs, fill)
    empty = np.flatnonzero(bt[:, 0] < 0)
    if len(empty) and B > 2:   # shared pages
        _, _, _, bt, kv, ref = ref_pages.fork(rng.integers(0, B, size=len(empty)), empty, bt, kv, ref, bs)
    seqs = rng.integers(-2, B + 2, size=min(4096, B + 1))
    et, ek, er = ref_pages.free(list(dict.fromkeys(seqs.tolist())), bt, kv, ref)
    dt, dk, dr = dev_i32(bt), dev_i32(kv), dev_i32(ref)
    free_pages(dev_i32(seqs), dt, dk, dr)
    assert eq(dt, et) and eq(dk, ek) and eq(dr, er)


def test_copy():
    rng = np.random.default_rng(5300)
    nb = 257
    pools = pool_set(rng, nb)
    order = rng.permutation(nb)
    src, dst = order[:100].copy(), order[100:200].copy()
    src[7], dst[9], src[11], dst[13] = -1, -5, nb, nb
    keep = (src >= 0) & (src < nb) & (dst >= 0) & (dst < nb)
    want = moved(pools, src[keep], dst[keep])
    copy_pages(dev_i32(src), dev_i32(dst), pools)
    assert same(pools, want)
    # a page of pool views that begin anywhere
    flat = torch.from_numpy(rng.integers(0, 256, size=20 * 40 + 3).astype(np.uint8)).cuda()
    view = flat[3:].view(20, 40)
    want = moved([view], [1, 2], [5, 19])
    copy_pages(dev_i32([1, 2]), dev_i32([5, 19]), [view])
    assert same([view], want)


@pytest.mark.parametrize("share", [0.0, 0.1, 0.5, 0.95, 1.0])
@pytest.mark.parametrize("nb", [1, 2, 7, 1000, 4096, 20011])
def test_compact(nb, share):
    rng = np.random.default_rng(5400 + nb)
    B, mb = 13, max(1, nb // 10)
    alive = rng.permutation(nb)[:int(nb * share)]
    bt = np.full((B, mb), -1, np.int64)
    for i, p in enumerate(alive):
        if i < B * mb:
            bt[i % B, i // B] = p
    bt[0, :] = bt[1, :]                      # shared pages
    ref = np.zeros(nb, np.int64)
    np.add.at(ref, bt[bt >= 0], 1)
    ref[alive[B * mb:]] = 3                  # pages that other tables name
    live, cs, cd, et, er = ref_pages.compact(bt, ref)
    pools = pool_set(rng, nb) if nb <= 4096 else pool_set(rng, nb)[2:5]
    want = moved(pools, cs, cd)
    dt, dr = dev_i32(bt), dev_i32(ref)
    print(f"compact {nb} pages, {live} live", flush=True)
    got = compact_pages(dt, dr, pools)
    assert int(got[0]) == live and eq(got[1], cs) and eq(got[2], cd)
    assert eq(dt, et) and eq(dr, er) and same(pools, want)


@pytest.mark.parametrize("case", range(1, len(SHAPES)))
def test_fork_of_rows_that_lack_a_page(case):
    """Sources whose kv_len covers an entry that is no page (the partly filled one, any other, a
    number outside the pool) are not forked, take no page and leave the others' pages theirs."""
    B, mb, nb, bs, fill = SHAPES[case]
    nb = min(nb, 20000)
    rng = np.random.default_rng(5500 + case)
    bt, kv, ref = state(rng, B, mb, nb, bs, fill * 0.8)
    empty, rows = np.flatnonzero(bt[:, 0] < 0), np.flatnonzero(kv > 0)
    if len(empty) == 0 and len(rows) > 1:
        empty, rows = rows[-1:], rows[:-1]
        bt[empty], kv[empty] = -1, 0
    for b in rows[rng.random(len(rows)) < 0.4]:
        last = int(kv[b] - 1) // bs
        j = last if rng.random() < 0.5 else int(rng.integers(0, mb))     # (behind the rows: no matter)
        bt[b, j] = rng.choice([-1, -2 ** 31, nb, 2 ** 31 - 1])
    kv[rows[::7]] = mb * bs                                              # a length beyond the pages
    n = min(1024, 2 * len(empty))
    src = rng.choice(rows, size=n)
    dst = np.concatenate([empty, empty])[:n]
    ok, cs, cd, et, ek, er = ref_pages.fork(src, dst, bt, kv, ref, bs)
    pools = pool_set(rng, nb)[2:5]
    want = moved(pools, cs, cd)
    dt, dk, dr = dev_i32(bt), dev_i32(kv), dev_i32(ref)
    got = fork_pages(dev_i32(src), dev_i32(dst), dt, dk, dr, bs, pools)
    assert eq(got[0], ok) and eq(got[1], cs) and eq(got[2], cd)
    assert eq(dt, et) and eq(dk, ek) and eq(dr, er) and same(pools, want)
    assert case < 3 or (ok.any() and not ok[:len(empty)].all())
