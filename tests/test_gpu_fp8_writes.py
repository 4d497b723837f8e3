"""GPU parity of the 8-bit cache's writers against the oracle: codes, exponents and lengths bit for
bit over whole pools.  Every step but the rounding to a code is exact in fp32 as in fp64 (powers of
two, maxima of given numbers), so nothing may differ."""
import numpy as np
import pytest
import torch

import oracle
from oracle import kv_fp8
from paper_2606_18394_amd import append_paged_fp8, commit_path_paged_fp8, synth
from helpers import dev_bf16, dev_i32
from test_gpu_fp8_attention import dev_f8, dev_u8

pytestmark = pytest.mark.gpu


def values(rng, shape):
    """bf16 bits of many magnitudes, with zeros of both signs, exact borders (448 and 449 at some
    scale, halves between codes) and denormals among them."""
    x = rng.standard_normal(shape, dtype=np.float32) * np.exp2(rng.integers(-20, 20, size=shape[:-1] + (1,)))
    pick = rng.random(shape)
    x = np.where(pick < 0.02, 0.0, x)
    x = np.where((pick > 0.02) & (pick < 0.03), -0.0, x)
    x = np.where((pick > 0.03) & (pick < 0.05), 2.0 ** rng.integers(-30, 30, size=shape) * 1.75, x)
    x = np.where((pick > 0.05) & (pick < 0.06), 2.0 ** rng.integers(-30, 30, size=shape) * 1.0625, x)
    x = np.where((pick > 0.06) & (pick < 0.07), 2.0 ** -130, x)
    return synth.bf16_bits(x.astype(np.float32))


def pools(rng, nb, Hkv, bs, D):
    """Pools that hold something everywhere; exponents around those of the values."""
    codes = rng.integers(0, 256, size=(2, nb, Hkv, bs, D)).astype(np.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x11
    exps = rng.integers(100, 140, size=(2, nb, Hkv, bs // 32)).astype(np.uint8)
    exps[:, ::5] = 16
    return codes, exps


def check(k, e, table, kv, expect, kv_expect, dev):
    dk, dv, dke, dve, dkv = dev
    torch.cuda.synchronize()
    assert np.array_equal(dkv.cpu().numpy(), kv_expect)
    for d, ref in ((dke, expect[0][1]), (dve, expect[1][1])):
        assert np.array_equal(d.cpu().numpy(), ref)
    for d, ref in ((dk, expect[0][0]), (dv, expect[1][0])):
        assert np.array_equal(d.view(torch.uint8).cpu().numpy(), ref)


APPEND = [
    # (B, T, Hkv, D, block_size, max_blocks, kv_lens, n_new)
    (1, 1, 1, 64, 32, 1, [0], [1]),
    (3, 1, 2, 64, 32, 2, [31, 32, 63], None),
    (64, 1, 8, 128, 64, 4, [(37 * i) % 250 for i in range(64)], [i % 2 for i in range(64)]),
    (4, 33, 3, 128, 32, 5, [0, 1, 31, 127], [33, 32, 0, 33]),
    # refused: too many, negative, no room by one, a negative length; the last lands on the capacity
    (5, 40, 5, 64, 64, 2, [10, 10, 89, -1, 88], [41, -1, 40, 3, 40]),
    (2, 70, 4, 128, 128, 2, [100, 186], [70, 70]),
    (1, 300, 8, 128, 256, 3, [77], None),
    (3, 1000, 2, 64, 32, 40, [0, 5, 255], [1000, 999, 1000]),
    (2, 515, 7, 128, 1024, 2, [1500, 3], [515, 0]),
]


@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append(case):
    B, T, Hkv, D, bs, mb, kvl, n = APPEND[case]
    print(f"append case {APPEND[case][:6]}", flush=True)
    rng = np.random.default_rng(4000 + case)
    bt, nb = synth.block_table(rng, B, mb, 2)
    codes, exps = pools(rng, nb, Hkv, bs, D)
    new = [values(rng, (B, T, Hkv, D)) for _ in range(2)]
    kvl = np.array(kvl, np.int32)
    rows = np.full(B, T) if n is None else np.array(n)
    dev = [dev_f8(codes[0]), dev_f8(codes[1]), dev_u8(exps[0]), dev_u8(exps[1]), dev_i32(kvl)]
    append_paged_fp8(dev_bf16(new[0]), dev_bf16(new[1]), *dev[:4], dev_i32(bt), dev[4],
                     n_new=None if n is None else dev_i32(rows))
    expect = [kv_fp8.append(codes[i], exps[i], bt, kvl, oracle.decode_bf16(new[i]), rows) for i in range(2)]
    ok = (rows >= 0) & (rows <= T) & (kvl >= 0) & (kvl + rows <= mb * bs)
    check(codes, exps, bt, kvl, expect, kvl + np.where(ok, rows, 0), dev)


@pytest.mark.parametrize("D", [64, 128])
def test_append_row_by_row(D):
    """Single rows one after the other, over several groups: a group's exponent only grows, and its
    codes follow it."""
    rng = np.random.default_rng(D)
    B, Hkv, bs, mb = 3, 2, 32, 3
    bt, nb = synth.block_table(rng, B, mb)
    codes, exps = pools(rng, nb, Hkv, bs, D)
    kvl = np.array([0, 20, 31], np.int32)
    dev = [dev_f8(codes[0]), dev_f8(codes[1]), dev_u8(exps[0]), dev_u8(exps[1]), dev_i32(kvl)]
    expect = [(codes[0], exps[0]), (codes[1], exps[1])]
    dbt = dev_i32(bt)
    for step in range(45):
        new = [values(rng, (B, 1, Hkv, D)) for _ in range(2)]
        append_paged_fp8(dev_bf16(new[0]), dev_bf16(new[1]), *dev[:4], dbt, dev[4])
        expect = [kv_fp8.append(*expect[i], bt, kvl + step, oracle.decode_bf16(new[i]), np.ones(B))
                  for i in range(2)]
    check(codes, exps, bt, kvl, expect, kvl + 45, dev)


COMMIT = [
    # (B, N, Hkv, D, block_size, max_blocks, Dmax)
    (1, 64, 8, 128, 256, 3, 9),
    (6, 40, 8, 128, 32, 5, 7),
    (6, 63, 1, 64, 64, 3, 13),
    (6, 2048, 2, 128, 32, 10, 200),
    (16, 64, 4, 64, 128, 4, 17),
]


@pytest.mark.parametrize("case", range(len(COMMIT)))
def test_commit(case):
    """Sequence 1 failed acceptance, 2 would pass its pages, 3 names a node outside the tree, 4 has an
    accept_len above Dmax, 5 a negative node; sequence 0 lands on the capacity."""
    B, N, Hkv, D, bs, mb, Dmax = COMMIT[case]
    print(f"commit case {COMMIT[case]}", flush=True)
    rng = np.random.default_rng(4100 + case)
    bt, nb = synth.block_table(rng, B, mb, 1)
    codes, exps = pools(rng, nb, Hkv, bs, D)
    tree = [values(rng, (B, N, Hkv, D)) for _ in range(2)]
    n = rng.integers(1, Dmax + 1, size=B).astype(np.int32)
    path = np.full((B, Dmax), -1, np.int32)
    for b in range(B):
        path[b, :n[b]] = rng.integers(0, N, size=n[b])   # (a node may come twice)
    kvl = rng.integers(0, mb * bs - Dmax + 1, size=B).astype(np.int32)
    kvl[0] = mb * bs - n[0]
    if B > 5:
        n[1] = -1
        kvl[2] = mb * bs - n[2] + 1
        path[3, n[3] - 1] = N
        n[4] = Dmax + 1
        path[5, 0] = -1
    dev = [dev_f8(codes[0]), dev_f8(codes[1]), dev_u8(exps[0]), dev_u8(exps[1]), dev_i32(kvl)]
    commit_path_paged_fp8(dev_bf16(tree[0]), dev_bf16(tree[1]), dev_i32(path), dev_i32(n), *dev[:4],
                          dev_i32(bt), dev[4])
    expect = [kv_fp8.commit(codes[i], exps[i], bt, kvl, oracle.decode_bf16(tree[i]), path, n)
              for i in range(2)]
    grown = np.where((np.arange(B) >= 1) & (np.arange(B) <= 5) & (B > 5), 0, n)
    check(codes, exps, bt, kvl, expect, kvl + grown, dev)


@pytest.mark.parametrize("T,Hkv", [(3, 2), (300, 8)])
def test_lacking_pages(T, Hkv):
    """A sequence that has no page for one of its rows is left as it is: entries that were never
    filled, numbers outside the pool, the last of many pages; the others get their rows."""
    rng = np.random.default_rng(T)
    B, D, bs, mb = 6, 64, 32, 100
    bt, nb = synth.block_table(rng, B, mb)
    kvl = np.array([0, 40, 31, 32 * 70 + 5, 64, 17], np.int32)
    bt[0, 0] = -1
    bt[1, (40 + T - 1) // bs] = nb
    bt[2, 10 if T == 3 else 5] = -7          # short: behind its rows, so nothing is lacking
    bt[4, 2 + (T - 1) // bs] = -1
    kvl[3] = mb * bs - T
    codes, exps = pools(rng, nb, Hkv, bs, D)
    new = [values(rng, (B, T, Hkv, D)) for _ in range(2)]
    rows = np.full(B, T)
    gets = np.array([0, 0, T == 3, 1, 0, 1])
    expect = [kv_fp8.append(codes[i], exps[i], bt, kvl, oracle.decode_bf16(new[i]), rows * gets) for i in range(2)]
    same = kv_fp8.append(codes[0], exps[0], bt, kvl, oracle.decode_bf16(new[0]), rows)
    assert all(np.array_equal(x, y) for x, y in zip(same, expect[0]))
    dev = [dev_f8(codes[0]), dev_f8(codes[1]), dev_u8(exps[0]), dev_u8(exps[1]), dev_i32(kvl)]
    append_paged_fp8(dev_bf16(new[0]), dev_bf16(new[1]), *dev[:4], dev_i32(bt), dev[4])
    check(codes, exps, bt, kvl, expect, kvl + T * gets, dev)
    path = np.tile(np.arange(T), (B, 1))
    dev = [dev_f8(codes[0]), dev_f8(codes[1]), dev_u8(exps[0]), dev_u8(exps[1]), dev_i32(kvl)]
    commit_path_paged_fp8(dev_bf16(new[0]), dev_bf16(new[1]), dev_i32(path), dev_i32(rows), *dev[:4],
                          dev_i32(bt), dev[4])
    check(codes, exps, bt, kvl, expect, kvl + T * gets, dev)


def test_many_pages_are_all_looked_at():
    """More than 64 pages for one sequence's rows, and the last of them is missing."""
    rng = np.random.default_rng(9)
    B, T, Hkv, D, bs, mb = 2, 2900, 1, 64, 32, 100
    bt, nb = synth.block_table(rng, B, mb)
    kvl = np.array([100, 100], np.int32)
    bt[1, (100 + T - 1) // bs] = -1
    codes, exps = pools(rng, nb, Hkv, bs, D)
    new = [values(rng, (B, T, Hkv, D)) for _ in range(2)]
    dev = [dev_f8(codes[0]), dev_f8(codes[1]), dev_u8(exps[0]), dev_u8(exps[1]), dev_i32(kvl)]
    append_paged_fp8(dev_bf16(new[0]), dev_bf16(new[1]), *dev[:4], dev_i32(bt), dev[4])
    expect = [kv_fp8.append(codes[i], exps[i], bt, kvl, oracle.decode_bf16(new[i]), [T, 0]) for i in range(2)]
    check(codes, exps, bt, kvl, expect, kvl + np.array([T, 0]), dev)


@pytest.mark.parametrize("T,Hkv", [(16, 1), (40, 2), (300, 8)])
def test_the_largest_numbers(T, Hkv):
    """Rows with the largest bf16 numbers of both signs, some of them behind older rows: codes that
    stand for bf16 numbers, and an attention over them that gives numbers."""
    from paper_2606_18394_amd import tree_verify_attention_paged_fp8
    rng = np.random.default_rng(T)
    B, D, bs, mb = 3, 64, 64, 8
    bt, nb = synth.block_table(rng, B, mb)
    kvl = np.array([0, 40, 63], np.int32)
    codes, exps = pools(rng, nb, Hkv, bs, D)
    new = [values(rng, (B, T, Hkv, D)) for _ in range(2)]
    # anywhere among the keys; among the values once per column, so that a sum of theirs stays finite
    for x, huge in zip(new, (rng.random(new[0].shape) < 0.05,
                             np.arange(T)[:, None, None] == rng.integers(0, T, size=(B, 1, Hkv, D)))):
        x[huge] = 0x7F60 + rng.integers(0, 32, size=huge.sum()) | rng.integers(0, 2, size=huge.sum()) << 15
    dev = [dev_f8(codes[0]), dev_f8(codes[1]), dev_u8(exps[0]), dev_u8(exps[1]), dev_i32(kvl)]
    append_paged_fp8(dev_bf16(new[0]), dev_bf16(new[1]), *dev[:4], dev_i32(bt), dev[4])
    expect = [kv_fp8.append(codes[i], exps[i], bt, kvl, oracle.decode_bf16(new[i]), [T] * B) for i in range(2)]
    check(codes, exps, bt, kvl, expect, kvl + T, dev)
    assert (expect[1][1] == 247).any()
    for c, e in expect:   # (codes behind a sequence's last row are not its)
        rows = kv_fp8.gather(c, e, bt, mb)
        for b in range(B):
            assert np.isfinite(rows[b, :kvl[b] + T].astype(np.float32)).all()
    # queries of zeros: every score is 0, and the output the mean of the values
    q = torch.zeros(B, 1, 2 * Hkv, D, dtype=torch.bfloat16, device="cuda")
    one = torch.zeros(B, 1, Hkv, D, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    tree_verify_attention_paged_fp8(q, *dev[:4], dev_i32(bt), one, one, None, out, kv_len=dev[4])
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("T,Hkv,D", [(1, 2, 64), (20, 3, 128), (300, 8, 128)])
def test_what_is_no_number_costs_its_group_nothing_else(T, Hkv, D):
    """Infinities and NaN among the rows: codes that are no numbers there, and everything else,
    exponents and older rows too, as without them."""
    rng = np.random.default_rng(100 + T)
    B, bs, mb = 3, 32, 12
    bt, nb = synth.block_table(rng, B, mb)
    kvl = np.array([0, 20, 63], np.int32)
    codes, exps = pools(rng, nb, Hkv, bs, D)
    new = [values(rng, (B, T, Hkv, D)) for _ in range(2)]
    for x in new:
        odd = rng.random(x.shape) < 0.01
        odd[:, 0, :, 3] = True
        x[odd] = rng.choice(np.array([0x7F80, 0xFF80, 0x7FC0, 0xFFC1, 0x7FFF, 0x7F81], np.uint16), odd.sum())
    new[0][:, -1, 0] = 0x7F80                            # a whole row
    dev = [dev_f8(codes[0]), dev_f8(codes[1]), dev_u8(exps[0]), dev_u8(exps[1]), dev_i32(kvl)]
    append_paged_fp8(dev_bf16(new[0]), dev_bf16(new[1]), *dev[:4], dev_i32(bt), dev[4])
    expect = [kv_fp8.append(codes[i], exps[i], bt, kvl, oracle.decode_bf16(new[i]), [T] * B) for i in range(2)]
    for i in range(2):
        assert ((expect[i][0] & 0x7F) == 0x7F).any() and expect[i][1].max() < 247
        got = dev[i].view(torch.uint8).cpu().numpy()
        no = (expect[i][0] & 0x7F) == 0x7F
        assert ((got[no] & 0x7F) == 0x7F).all() and np.array_equal(got[~no], expect[i][0][~no])
        assert np.array_equal(dev[2 + i].cpu().numpy(), expect[i][1])
    assert np.array_equal(dev[4].cpu().numpy(), kvl + T)
