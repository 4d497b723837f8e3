"""Serving from a paged KV cache held in 8 bits: the work of its operators, case by case.

The cache: pools [num_blocks, Hkv, block_size, D] of e4m3 codes for K and V, and one exponent
byte e for each group of 32 positions of a page and head, [num_blocks, Hkv, block_size / 32]; a
code stands for code * 2^(e - 127).  Position t of sequence b is row t % block_size of page
block_table[b, t // block_size].

  attend   the verification attention over such a cache (N = 1: single-token decoding)
  append   new K/V rows are quantised into the sequences' pages (prompts, decode steps)
  commit   the same for the accepted path of a draft tree
  fork, recycle, compact   which page belongs to whom: sequences that share their pages,
           sequences that end while others grow, a pool whose live pages are drawn together

  own                  False: run() is plain torch; True: the package's calls
  listed()             the cases
  draw(rng)            one more case of the same ranges
  prepare(case, seed)  what a program has in hand before the call, on the GPU
  run(state)           one pass; its outputs, whole
  work(case)           bytes and flops a pass cannot do without
  exact(case, seed)    the computed numbers in 64 bits

Head shapes, tree sizes and cache lengths are those of the package's workloads and tests; the odd
sizes are generic.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

F8 = torch.float8_e4m3fn
GROUP = 32          # positions that share an exponent
EMIN, EMAX = 16, 247  # exponents that writers use

# (query heads, KV heads, head dim)
HEADS = [(4, 2, 64), (32, 8, 128), (32, 4, 128), (64, 8, 128), (16, 8, 64), (8, 8, 128)]


def _attend(name, B, heads, L, lo, N, depth, page):
    """kv_len is drawn from [lo, L]; depth 0: a chain."""
    Hq, Hkv, D = heads
    return {"name": name, "kind": "attend", "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "L": L, "lo": lo,
            "N": N, "depth": depth, "page": page}


def listed():
    return [
        # the smallest call: one token of one user on a short prompt of a small model
        _attend("decode_tiny", 1, (4, 2, 64), 200, 200, 1, 0, 32),
        # a loaded server between drafts: single tokens of 64 sequences of very different lengths
        _attend("decode_batch", 64, (32, 8, 128), 8192, 512, 1, 0, 64),
        # batch 16, root + 32 drafts, ragged caches
        _attend("verify_serving", 16, (32, 4, 128), 4096, 300, 33, 8, 64),
        # two users with whole books in the cache and a small tree each
        _attend("verify_long", 2, (32, 8, 128), 131072, 120000, 16, 6, 256),
        # the largest draft budget on the widest target
        _attend("verify_big_tree", 1, (64, 8, 128), 8192, 8192, 512, 16, 128),
        # prompts of four users enter the cache, the second chunks of two of them
        {"name": "append_prefill", "kind": "append", "B": 4, "Hkv": 8, "D": 128, "T": 8192, "lo": 2000,
         "L": 3001, "page": 256},
        # one token each of 64 sequences: groups that are partly filled
        {"name": "append_decode", "kind": "append", "B": 64, "Hkv": 8, "D": 128, "T": 1, "lo": 1,
         "L": 8191, "page": 64},
        # one user's accepted path
        {"name": "commit_one", "kind": "commit", "B": 1, "Hkv": 8, "D": 128, "N": 64, "depth": 8,
         "L": 4096, "page": 256},
        # a batch's accepted paths, out of the largest trees
        {"name": "commit_batch", "kind": "commit", "B": 32, "Hkv": 8, "D": 128, "N": 512, "depth": 16,
         "L": 2048, "page": 64},
        # eight prompts, each continued in eight ways
        {"name": "fork", "kind": "fork", "B": 64, "parents": 8, "Hkv": 8, "D": 128, "L": 4090, "page": 64},
        # a quarter of 256 sequences end, the others grow by a page or so
        {"name": "recycle", "kind": "recycle", "B": 256, "Hkv": 2, "D": 64, "L": 2048, "page": 32,
         "grow": 50},
        # a pool of 4096 pages of which a third is alive
        {"name": "compact", "kind": "compact", "B": 64, "Hkv": 8, "D": 128, "pages": 4096, "live": 0.33,
         "page": 64},
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_once(rng):
    kind = rng.choice(["attend"] * 5 + ["append"] * 2 + ["commit"] * 2 + ["fork", "recycle", "compact"])
    Hq, Hkv, D = rng.choice(HEADS)
    page = rng.choice([32, 64, 128, 256])
    B = _log_int(rng, 1, 64)
    if kind == "attend":
        L = _log_int(rng, 64, 131072)
        N = 1 if rng.random() < 0.3 else _log_int(rng, 2, 512)
        depth = 0 if N == 1 or rng.random() < 0.2 else rng.randint(max(2, (N - 1).bit_length()), 16)
        return {"kind": kind, "B": B, "Hq": Hq, "Hkv": Hkv, "D": D, "L": L, "lo": rng.choice([L, L // 16]),
                "N": N, "depth": depth, "page": page}
    c = {"kind": kind, "B": B, "Hkv": Hkv, "D": D, "page": page}
    if kind == "append":
        T = rng.choice([1, _log_int(rng, 1, 64), _log_int(rng, 64, 8192)])
        return {**c, "T": T, "lo": rng.choice([T, 0]), "L": _log_int(rng, 1, 8192)}
    if kind == "commit":
        return {**c, "N": _log_int(rng, 8, 512), "depth": rng.randint(4, 16), "L": _log_int(rng, 32, 8192)}
    if kind == "fork":
        B = max(2, B)
        return {**c, "B": B, "parents": _log_int(rng, 1, max(1, B // 2)), "L": _log_int(rng, 32, 8192)}
    if kind == "recycle":
        return {**c, "B": _log_int(rng, 2, 256), "L": _log_int(rng, 64, 8192), "grow": _log_int(rng, 1, 500)}
    return {**c, "pages": _log_int(rng, 64, 4096), "live": round(rng.uniform(0.1, 0.9), 3)}


def draw(rng):
    """One more case; redrawn while it would cost more than the largest listed ones."""
    while True:
        c = _draw_once(rng)
        w = work(c)
        rows = {"attend": c.get("L"), "append": c.get("L", 0) + c.get("T", 0), "compact": 0}
        pool = c["B"] * rows.get(c["kind"], c.get("L", 0)) * c["Hkv"] * c["D"]
        if w["bytes"] > 5.5e8 or w["flops"] > 1.4e11 or pool > 5.4e8:
            continue
        if c["kind"] == "compact" and c["pages"] * c["page"] * c["Hkv"] * c["D"] > 2.7e8:
            continue
        return c


# ------------------------------------------------------------------ inputs


def _rng(seed, salt=0):
    return np.random.default_rng([seed, salt])


def _gen(seed, salt=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1000003 + salt)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16)


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _tree(r, N, depth):
    """A random tree, every parent before its children; depth 0: a chain."""
    parent = np.arange(-1, N - 1, dtype=np.int32)
    if depth:
        dep = np.zeros(N, np.int64)
        for i in range(1, N):
            p = int(r.integers(0, i))
            while dep[p] >= depth:
                p = int(parent[p])
            parent[i] = p
            dep[i] = dep[p] + 1
    return parent


def _lens(case, seed, lo, hi):
    """One length per sequence; the extremes are among them."""
    kv = _rng(seed, 2).integers(lo, hi + 1, size=case["B"])
    kv[0] = hi
    return kv


def _pool(g, pages, case):
    """Codes and exponents of a filled pool: normal values of many magnitudes; a few channels of
    the keys are larger than the others."""
    Hkv, D, bs = case["Hkv"], case["D"], case["page"]
    wide = torch.ones(D, device="cuda")
    wide[torch.randperm(D, generator=g, device="cuda")[:4]] = 6.0
    both = []
    for scale in (wide, torch.ones(D, device="cuda")):
        x = torch.randn(pages, Hkv, bs // GROUP, GROUP, D, generator=g, device="cuda") * scale
        _, ex = torch.frexp(x.abs().amax((-1, -2)) / 448)
        codes = torch.ldexp(x, -ex[..., None, None]).to(F8).view(pages, Hkv, bs, D)
        both += [codes, (ex + 127).to(torch.uint8)]
        del x
    k, ke, v, ve = both
    return {"k": k, "v": v, "ke": ke, "ve": ve}


def _table(seed, lens, page, width, total):
    """Rows of shuffled pages of the pool's `total`: a row's own first, -1 behind them."""
    used = [-(-int(n) // page) for n in lens]
    order = _rng(seed, 3).permutation(total).astype(np.int32)
    bt = np.full((len(used), width), -1, np.int32)
    at = 0
    for b, u in enumerate(used):
        bt[b, :u] = order[at:at + u]
        at += u
    return bt


def _owned(case, seed, g, bt, kv, pages):
    """Table, lengths and counts in one buffer (so that a pass can put them back at once), and the pool."""
    ref = np.zeros(pages, np.int32)
    np.add.at(ref, bt[bt >= 0], 1)
    whole = np.concatenate([bt.ravel(), np.asarray(kv, np.int32), ref]).astype(np.int32)
    s = {"case": case, "start": _i32(whole), "now": _i32(whole)}
    n, B = bt.size, bt.shape[0]
    s["table"], s["kv_len"] = s["now"][:n].view(bt.shape), s["now"][n:n + B]
    s["ref"] = s["now"][n + B:]
    s.update(_pool(g, pages, case))
    return s


def prepare(case, seed):
    kind, B, Hkv, D, page = (case[k] for k in ("kind", "B", "Hkv", "D", "page"))
    g = _gen(seed, 7)
    if kind == "attend":
        N, Hq = case["N"], case["Hq"]
        kv = _lens(case, seed, case["lo"], case["L"])
        width = -(-case["L"] // page)
        pages = B * width + 3
        bt = _table(seed, kv, page, width, pages)
        r = _rng(seed, 1)
        s = {"case": case, "table": _i32(bt), "kv_len": _i32(kv),
             "parent": _i32(np.stack([_tree(r, N, case["depth"]) for _ in range(B)])),
             "q": _normal(g, B, N, Hq, D), "kt": _normal(g, B, N, Hkv, D), "vt": _normal(g, B, N, Hkv, D),
             "out": torch.empty(B, N, Hq, D, dtype=torch.bfloat16, device="cuda")}
        s.update(_pool(g, pages, case))
        return s
    if kind in ("append", "commit"):
        rows = case["T"] if kind == "append" else case["depth"] + 1
        kv = _lens(case, seed, case["L"] // 8, case["L"])
        width = -(-(case["L"] + rows) // page)
        pages = B * width + 3
        bt = _table(seed, kv + rows, page, width, pages)
        s = {"case": case, "table": _i32(bt), "kv0": _i32(kv), "kv_len": _i32(kv)}
        s.update(_pool(g, pages, case))
        if kind == "append":
            n = _rng(seed, 5).integers(case["lo"], case["T"] + 1, size=B)
            n[0] = case["T"]
            s.update(n=_i32(n), kt=_normal(g, B, rows, Hkv, D), vt=_normal(g, B, rows, Hkv, D))
        else:
            # paths as acceptance writes them: root first, increasing nodes, -1 behind them
            N, r = case["N"], _rng(seed, 5)
            n = r.integers(1, min(rows, N) + 1, size=B)
            path = np.full((B, rows), -1, np.int32)
            for b in range(B):
                path[b, 1:n[b]] = np.sort(r.choice(np.arange(1, N), n[b] - 1, replace=False))
                path[b, 0] = 0
            s.update(n=_i32(n), path=_i32(path), kt=_normal(g, B, N, Hkv, D), vt=_normal(g, B, N, Hkv, D))
        return s
    if kind == "fork":
        # the first sequences are prompts, the other rows are empty and take their continuations
        P = case["parents"]
        kv = np.zeros(B, np.int64)
        kv[:P] = _rng(seed, 2).integers(case["L"] // 2, case["L"] + 1, size=P)
        width = -(-case["L"] // page) + 1
        pages = P * width + B
        bt = _table(seed, kv, page, width, pages)
        s = _owned(case, seed, g, bt, kv, pages)
        s["dst"] = _i32(_rng(seed, 6).permutation(np.arange(P, B)))
        s["src"] = _i32(np.arange(B - P) % P)
        return s
    if kind == "recycle":
        kv = _lens(case, seed, case["L"] // 4, case["L"])
        width = -(-(case["L"] + case["grow"]) // page)
        pages = B * -(-case["L"] // page)
        bt = _table(seed, kv, page, width, pages)
        s = _owned(case, seed, g, bt, kv, pages)
        s["ended"] = _i32(_rng(seed, 6).permutation(B)[:max(1, B // 4)])
        more = np.full(B, case["grow"])
        more[s["ended"].cpu().numpy()] = 0
        s["more"] = _i32(more)
        return s
    # compact: `live` of the pool's pages belong to somebody, some of them to two sequences
    pages = case["pages"]
    r = _rng(seed, 6)
    alive = r.permutation(pages)[:max(1, int(pages * case["live"]))]
    per = -(-len(alive) // B)
    bt = np.full((B, per + 2), -1, np.int32)
    for b in range(B):
        mine = alive[b * per:(b + 1) * per]
        bt[b, :len(mine)] = mine
        if b and len(mine) and bt[b - 1, 0] >= 0:
            bt[b, 0] = bt[b - 1, 0] if r.random() < 0.3 else bt[b, 0]
    return _owned(case, seed, g, bt, (bt >= 0).sum(1) * page, pages)


# ------------------------------------------------------------------ a pass, plain


def _values(codes, exps):
    """Codes [..., rows, D] and exponents [..., rows / 32] as the fp32 numbers they stand for."""
    x = codes.float().unflatten(-2, (-1, GROUP))
    return torch.ldexp(x, (exps.int() - 127)[..., None, None]).flatten(-3, -2)


def _twice(r):
    """Relations of up to twice as many steps."""
    return ((r @ r) > 0).float()


def _ancestors(parent):
    """[B, N, N]: whether u is v or one of its ancestors; parent None: a chain."""
    N = parent.shape[-1]
    up = torch.arange(N, device="cuda") == parent[..., None]
    r = (up | torch.eye(N, dtype=torch.bool, device="cuda")).float()
    return _twice(_twice(_twice(_twice(_twice(_twice(_twice(_twice(_twice(r)))))))))


def _plain_attend(s):
    case = s["case"]
    B, N, Hq, Hkv, D = (case[k] for k in ("B", "N", "Hq", "Hkv", "D"))
    G, at = Hq // Hkv, s["table"].long().clamp(min=0)
    # [B, pages, Hkv, page, D] -> [B, Hkv, rows, D]
    k = _values(s["k"][at], s["ke"][at]).transpose(1, 2).flatten(2, 3)
    v = _values(s["v"][at], s["ve"][at]).transpose(1, 2).flatten(2, 3)
    rows = k.shape[2]
    q = s["q"].float().unflatten(2, (Hkv, G)).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D)
    kt, vt = s["kt"].float().transpose(1, 2).contiguous(), s["vt"].float().transpose(1, 2).contiguous()
    past = torch.arange(rows, device="cuda") < s["kv_len"][:, None]
    cache = (q @ k.transpose(2, 3).contiguous()) * D ** -0.5
    cache = torch.where(past[:, None, None], cache, -math.inf)
    tree = (q @ kt.transpose(2, 3).contiguous()) * D ** -0.5
    seen = (_ancestors(s["parent"]) > 0).repeat_interleave(G, 1)
    tree = torch.where(seen[:, None], tree, -math.inf)
    m = torch.maximum(cache.amax(-1, True), tree.amax(-1, True))
    cache, tree = torch.exp(cache - m), torch.exp(tree - m)
    total = cache.sum(-1, True) + tree.sum(-1, True)
    v = torch.where(past[:, None, :, None], v, 0.0)
    o = (cache @ v + tree @ vt) / total
    s["out"].copy_(o.unflatten(2, (N, G)).transpose(1, 2).reshape(B, N, Hq, D))
    return s["out"]


def _exponent(a):
    """The least e of the range with a <= 448 * 2^(e - 127)."""
    frac, ex = torch.frexp(a)
    e = torch.where(a > 0, ex - 9 + (frac > 0.875).int() + 127, 0)
    return e.clamp(EMIN, EMAX)


def _plain_write(s, x, pool, exps, ok_n):
    """x [B, rows, Hkv, D] goes behind the kv_len rows of each sequence, ok_n[b] of them."""
    B, rows, Hkv, D = x.shape
    bs, kv = pool.shape[2], s["kv_len"].long()
    groups = (rows + GROUP - 2) // GROUP + 1
    group = kv[:, None] // GROUP + torch.arange(groups, device="cuda")               # [B, groups]
    pos = group[..., None] * GROUP + torch.arange(GROUP, device="cuda")              # [B, groups, 32]
    end = (kv + ok_n)[:, None, None]
    touched = (group * GROUP < end[..., 0]) & (ok_n > 0)[:, None]
    new = touched[..., None] & (pos >= kv[:, None, None]) & (pos < end)
    old = touched[..., None] & (pos < kv[:, None, None])
    at = (pos - kv[:, None, None]).clamp(0, rows - 1)
    val = x.float()[torch.arange(B, device="cuda")[:, None, None], at]               # [B, g, 32, H, D]
    page = s["table"].long().gather(1, (group * GROUP // bs).clamp(max=s["table"].shape[1] - 1)).clamp(min=0)
    e_new = _exponent(torch.where(new[..., None, None], val.abs(), 0.0).amax((2, 4)))  # [B, g, H]
    place = group * GROUP % bs // GROUP
    e_old = exps[page, :, place].int()
    e = torch.where(old.any(-1)[..., None], torch.maximum(e_old, e_new), e_new)
    code = torch.ldexp(val, (127 - e)[:, :, None, :, None])
    row = pos % bs
    was = pool.view(torch.uint8)[page[..., None], :, row].view(F8).float()            # [B, g, 32, H, D]
    was = torch.ldexp(was, (e_old - e)[:, :, None, :, None])
    code = torch.where(new[..., None, None], code, was).to(F8)
    write = new | old
    b, gi, r = write.nonzero(as_tuple=True)
    pool.view(torch.uint8)[page[b, gi], :, row[b, gi, r]] = code.view(torch.uint8)[b, gi, r]
    b, gi = touched.nonzero(as_tuple=True)
    exps[page[b, gi], :, place[b, gi]] = e[b, gi].to(torch.uint8)


def _plain_grow(s):
    s["kv_len"].copy_(s["kv0"])
    n = s["n"].long()
    kt, vt = s["kt"], s["vt"]
    if "path" in s:
        at = s["path"].long().clamp(min=0)[..., None, None].expand(-1, -1, *kt.shape[2:])
        kt, vt = kt.gather(1, at), vt.gather(1, at)
    _plain_write(s, kt, s["k"], s["ke"], n)
    _plain_write(s, vt, s["v"], s["ve"], n)
    s["kv_len"] += s["n"]


def _free_first(ref):
    """The pages, free ones first, each kind by its number, and how many are free."""
    return torch.argsort((ref > 0).int(), stable=True), (ref == 0).sum()


def _plain_fork(s):
    page, src, dst = s["case"]["page"], s["src"].long(), s["dst"].long()
    table, ref = s["table"], s["ref"]
    kv = s["kv_len"][src].long()
    full, part = kv // page, kv % page > 0
    free, count = _free_first(ref)
    rank = part.long().cumsum(0) - 1
    ok = ~part | (rank < count)
    fresh = free[rank.clamp(0, free.numel() - 1)]
    copy = part & ok
    rows, col = table[src].long(), torch.arange(table.shape[1], device="cuda")
    last = rows.gather(1, full.clamp(max=table.shape[1] - 1)[:, None])[:, 0]
    mine = torch.where(col < full[:, None], rows, -1)
    mine = torch.where((col == full[:, None]) & part[:, None], fresh[:, None], mine)
    shared = (col < full[:, None]) & ok[:, None]
    ref.index_add_(0, rows.clamp(min=0).flatten(), shared.int().flatten())
    ref.index_add_(0, torch.where(copy, fresh, 0), copy.int())
    table[dst] = torch.where(ok[:, None], mine.int(), table[dst])
    s["kv_len"][dst] = torch.where(ok, kv.int(), s["kv_len"][dst])
    # (a fork without a copy copies a page onto itself)
    src_page = torch.where(copy, last, rows[:, 0].clamp(min=0))
    dst_page = torch.where(copy, fresh, rows[:, 0].clamp(min=0))
    for p in (s["k"], s["v"], s["ke"], s["ve"]):
        p = p.view(torch.uint8)
        p[dst_page] = p[src_page]
    return ok.int()


def _plain_recycle(s):
    page, table, kv, ref = s["case"]["page"], s["table"], s["kv_len"], s["ref"]
    gone = s["ended"].long()
    rows = table[gone].long()
    ref.index_add_(0, rows.clamp(min=0).flatten(), -(rows >= 0).int().flatten())
    table[gone] = -1
    kv[gone] = 0
    need = (kv.long() + s["more"] + page - 1) // page
    ask = (torch.arange(table.shape[1], device="cuda") < need[:, None]) & (table < 0)
    n = ask.sum(1)
    free, count = _free_first(ref)
    ok = (n.cumsum(0) <= count) | (n == 0)
    give = ask & ok[:, None]
    fresh = free[(ask.flatten().long().cumsum(0) - 1).clamp(0, free.numel() - 1)].view(table.shape)
    table.copy_(torch.where(give, fresh.int(), table))
    ref.index_add_(0, torch.where(give, fresh, 0).flatten(), give.int().flatten())
    return ok.int()


def _plain_compact(s):
    table, ref = s["table"], s["ref"]
    ids = torch.arange(ref.numel(), device="cuda")
    live = ref > 0
    n = live.sum()
    into = ~live & (ids < n)
    away = live & (ids >= n)
    dst = torch.argsort((~into).int(), stable=True)                   # ascending free pages first
    src = ids.numel() - 1 - torch.argsort((~away.flip(0)).int(), stable=True)  # descending live ones first
    moved = ids < into.sum()
    # page y is taken from page source[y]
    source = ids.clone().scatter_(0, torch.where(moved, dst, dst), torch.where(moved, src, dst))
    remap = ids.clone().scatter_(0, torch.where(moved, src, src), torch.where(moved, dst, src))
    for p in (s["k"], s["v"], s["ke"], s["ve"]):
        p = p.view(torch.uint8)
        p.copy_(p[source])
    table.copy_(torch.where(table >= 0, remap[table.long().clamp(min=0)].int(), table))
    ref.copy_(torch.where(away, 0, ref[source]))
    return n.int().view(1)


# ------------------------------------------------------------------ a pass


def run(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "attend":
        if own:
            import paper_2606_18394_amd as tv
            return tv.tree_verify_attention_paged_fp8(
                s["q"], s["k"], s["v"], s["ke"], s["ve"], s["table"], s["kt"], s["vt"], s["parent"],
                s["out"], kv_len=s["kv_len"])
        return _plain_attend(s)
    pools = (s["k"], s["v"], s["ke"], s["ve"])
    if kind in ("append", "commit"):
        # every pass starts at the same lengths, so that it writes the same rows
        if own:
            import paper_2606_18394_amd as tv
            s["kv_len"].copy_(s["kv0"])
            if kind == "append":
                tv.append_paged_fp8(s["kt"], s["vt"], *pools, s["table"], s["kv_len"], n_new=s["n"])
            else:
                tv.commit_path_paged_fp8(s["kt"], s["vt"], s["path"], s["n"], *pools, s["table"],
                                         s["kv_len"])
        else:
            _plain_grow(s)
        return s["k"], s["v"], s["ke"], s["ve"], s["kv_len"]
    # every pass starts from the same owners
    s["now"].copy_(s["start"])
    if own:
        import paper_2606_18394_amd as tv
        if kind == "fork":
            said = tv.fork_pages(s["src"], s["dst"], s["table"], s["kv_len"], s["ref"], case["page"], pools)[0]
        elif kind == "recycle":
            tv.free_pages(s["ended"], s["table"], s["kv_len"], s["ref"])
            said = tv.reserve_pages(s["more"], s["table"], s["kv_len"], s["ref"], case["page"])
        else:
            said = tv.compact_pages(s["table"], s["ref"], pools)[0]
    else:
        said = {"fork": _plain_fork, "recycle": _plain_recycle, "compact": _plain_compact}[kind](s)
    if kind == "recycle":
        return said, s["table"], s["kv_len"], s["ref"]
    return (said, s["table"], s["kv_len"], s["ref"]) + pools


# ------------------------------------------------------------------ accounts


def work(case):
    kind, B, Hkv, D, page = (case[k] for k in ("kind", "B", "Hkv", "D", "page"))
    row = Hkv * D
    if kind == "attend":
        N, Hq = case["N"], case["Hq"]
        keys = (case["lo"] + case["L"]) / 2
        nbytes = B * (2 * keys * (row + Hkv / GROUP) + 4 * N * row + 4 * N * Hq * D + 4 * N + 4 * keys / page)
        return {"bytes": nbytes, "flops": 4 * D * Hq * B * N * (keys + (case["depth"] or N) / 2 + 1)}
    if kind in ("append", "commit"):
        n = (case["lo"] + case["T"]) / 2 if kind == "append" else case["depth"] / 2 + 1
        return {"bytes": 6 * B * n * row, "flops": 0}
    of_page = 2 * page * (row + Hkv / GROUP)
    if kind == "fork":
        forks = B - case["parents"]
        return {"bytes": 2 * forks * of_page + 8 * forks * case["L"] * 0.75 / page, "flops": 0}
    if kind == "recycle":
        return {"bytes": 8 * B * case["L"] / page, "flops": 0}
    pages, live = case["pages"], case["live"]
    return {"bytes": 2 * pages * live * (1 - live) * of_page + 8 * pages, "flops": 0}


# ------------------------------------------------------------------ 64 bits


def _exact_attend(s):
    case = s["case"]
    B, N, Hq, Hkv, D = (case[k] for k in ("B", "N", "Hq", "Hkv", "D"))
    G = Hq // Hkv
    parent, kv = s["parent"].cpu().numpy(), s["kv_len"].cpu().numpy()
    out = torch.empty(B, N, Hq, D, dtype=torch.float64, device="cuda")
    for b in range(B):
        anc = np.zeros((N, N), dtype=bool)
        for i in range(N):
            if i:
                anc[i] = anc[parent[b, i]]
            anc[i, i] = True
        n = int(kv[b])
        mine = s["table"][b, :-(-n // case["page"])].long()
        vis = torch.ones(N, n + N, dtype=torch.bool, device="cuda")
        vis[:, n:] = torch.from_numpy(anc).cuda()
        vis = vis.repeat_interleave(G, 0)
        for h in range(Hkv):
            keys = []
            for pool, exps, tree in ((s["k"], s["ke"], s["kt"]), (s["v"], s["ve"], s["vt"])):
                scale = torch.exp2(exps[mine, h].double() - 127).flatten().repeat_interleave(GROUP)
                x = pool[mine, h].double().reshape(-1, D) * scale[:, None]
                keys.append(torch.cat([x[:n], tree[b, :, h].double()]))
            q = s["q"][b, :, h * G:(h + 1) * G].reshape(N * G, D).double()
            sc = (q @ keys[0].t()) * D ** -0.5
            o = torch.softmax(sc.masked_fill(~vis, -math.inf), -1) @ keys[1]
            out[b, :, h * G:(h + 1) * G] = o.reshape(N, G, D)
    return out


def _nearest(x):
    """fp64 values of at most 448 in size, rounded to e4m3: 4 significant bits, steps of 2^-9 at least."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(x / step) * step


def _exact_grow(s):
    case, page = s["case"], s["case"]["page"]
    table, kv, n = (s[k].cpu().numpy() for k in ("table", "kv0", "n"))
    done = []
    for pool, exps, new in ((s["k"], s["ke"], s["kt"]), (s["v"], s["ve"], s["vt"])):
        pool, exps = pool.double(), exps.double()
        for b in range(case["B"]):
            x = new[b, :n[b]] if "path" not in s else new[b][s["path"][b, :n[b]].long()]
            x = x.double()
            at = int(kv[b])
            while at < kv[b] + n[b]:
                lo = at // GROUP * GROUP
                hi = min(lo + GROUP, int(kv[b] + n[b]))
                p, r0 = int(table[b, lo // page]), lo % page
                mine = x[at - int(kv[b]):hi - int(kv[b])].transpose(0, 1)            # [Hkv, rows, D]
                a = mine.abs().amax((1, 2))
                e = torch.ceil(torch.log2(a.clamp(min=1e-300) / 448)) + 127
                e = e.clamp(EMIN, EMAX)
                if at > lo:
                    was = exps[p, :, r0 // GROUP]
                    e = torch.maximum(e, was)
                    old = pool[p, :, r0:r0 + at - lo]
                    pool[p, :, r0:r0 + at - lo] = _nearest(old * torch.exp2(was - e)[:, None, None])
                pool[p, :, r0 + at - lo:r0 + hi - lo] = _nearest(mine * torch.exp2(127 - e)[:, None, None])
                exps[p, :, r0 // GROUP] = e
                at = hi
        done.append(pool)
    return done[0], done[1], None, None, None


def exact(case, seed):
    if case["kind"] == "attend":
        return _exact_attend(prepare(case, seed))
    if case["kind"] in ("append", "commit"):
        return _exact_grow(prepare(case, seed))
    return None  # whole numbers and copies
