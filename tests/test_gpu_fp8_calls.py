"""How the calls of the 8-bit cache and of its pages are made: the native half of the binding and the
Python half, streams, graphs, several calls at once, and a server's steps one after the other."""
import numpy as np
import pytest
import torch

import oracle
from oracle import kv_fp8, pages as ref_pages
import paper_2606_18394_amd as tv
from paper_2606_18394_amd import binding, synth
from helpers import dev_bf16, dev_i32
from test_gpu_fp8_attention import case_inputs, dev_f8, dev_u8, oracle_and_bound

pytestmark = pytest.mark.gpu


def attention_args(case):
    q, k, v, ke, ve, bt, kt, vt, parent, kvl = case_inputs(case)
    return [dev_bf16(q), dev_f8(k), dev_f8(v), dev_u8(ke), dev_u8(ve), dev_i32(bt), dev_bf16(kt),
            dev_bf16(vt), dev_i32(parent), torch.empty(*q.shape, dtype=torch.bfloat16, device="cuda")], \
        dev_i32(kvl)


def bits(t):
    return t.view(torch.int16).cpu().numpy().copy()


def serving_state(seed=0, Hkv=2, D=64, bs=32, mb=6, nb=40, B=4):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    z = dict(dtype=torch.uint8, device="cuda")
    pools = [torch.zeros(nb, Hkv, bs, D, **z).view(torch.float8_e4m3fn) for _ in range(2)]
    exps = [torch.zeros(nb, Hkv, bs // 32, **z) for _ in range(2)]
    table = torch.full((B, mb), -1, dtype=torch.int32, device="cuda")
    kv, ref = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (B, nb))

    def rows(n, heads=Hkv):
        return torch.randn(B, n, heads, D, generator=g, device="cuda").to(torch.bfloat16)

    return pools + exps, table, kv, ref, rows


@pytest.mark.parametrize("native", [True, False])
def test_both_halves_of_the_binding(native, monkeypatch):
    """The same results from either half; the native one is there and does these calls."""
    if native:
        assert binding._direct is not None or binding.load_library() and binding._direct is not None
    args, kv = attention_args(8)
    tv.tree_verify_attention_paged_fp8(*args, kv_len=kv)
    first = bits(args[9])
    cache, table, kvl, ref, rows = serving_state()
    if native:
        assert binding._direct.attention(*args, kv, None, None) is args[9]
    else:
        monkeypatch.setattr(binding, "_direct", None)
        args[9].zero_()
        tv.tree_verify_attention_paged_fp8(*args, kv_len=kv)
    assert np.array_equal(bits(args[9]), first)
    ok = tv.reserve_pages(torch.full_like(kvl, 70), table, kvl, ref, 32)
    assert ok.tolist() == [1] * 4 and table[:, :3].flatten().tolist() == list(range(12))
    tv.append_paged_fp8(rows(70), rows(70), *cache, table, kvl)
    tree = rows(5), rows(5)
    tv.commit_path_paged_fp8(*tree, dev_i32([[0, 2, 3, -1]] * 4), dev_i32([3, 2, 1, -1]), *cache, table, kvl)
    assert kvl.tolist() == [73, 72, 71, 70]
    tv.free_pages(dev_i32([1]), table, kvl, ref)
    ok, src, dst = tv.fork_pages(dev_i32([0]), dev_i32([1]), table, kvl, ref, 32, cache)
    assert ok.tolist() == [1] and src.tolist() == [2] and dst.tolist() == [3]
    assert table[1].tolist() == [0, 1, 3, -1, -1, -1] and torch.equal(cache[0][2].view(torch.uint8),
                                                                      cache[0][3].view(torch.uint8))
    with pytest.raises(TypeError, match="kv_len must be"):
        tv.tree_verify_attention_paged_fp8(*args, kv_len=kv.long())
    with pytest.raises(ValueError, match="contiguous"):
        tv.append_paged_fp8(rows(4)[:, ::2], rows(2), *cache, table, kvl)
    with pytest.raises(ValueError, match="has shape"):
        tv.append_paged_fp8(rows(4), rows(3), *cache, table, kvl)
    with pytest.raises(RuntimeError, match="TV_ERR_SHAPE"):
        tv.reserve_pages(kvl, table, kvl, ref, 48)
    with pytest.raises(RuntimeError, match="TV_ERR_WORKSPACE"):
        big, kvb = attention_args(4)
        tv.tree_verify_attention_paged_fp8(*big, kv_len=kvb,
                                           workspace_tensor=torch.zeros(64, dtype=torch.uint8, device="cuda"))


def test_serving_steps():
    """A server's life on the 8-bit cache, against the oracle after every step: prompts, a fork, draft
    trees verified and committed, single tokens, an end, a compaction."""
    B, Hq, Hkv, D, bs, mb, nb, N = 4, 8, 2, 64, 32, 6, 40, 9
    cache, table, kv, ref, rows = serving_state(1, Hkv, D, bs, mb, nb, B)
    host = [c.view(torch.uint8).cpu().numpy() for c in cache]   # K, V codes, K, V exponents
    t, k, r = table.cpu().numpy(), kv.cpu().numpy(), ref.cpu().numpy()
    rng = np.random.default_rng(1)
    f64 = lambda x: x.double().cpu().numpy()  # noqa: E731

    def reserve(n):
        nonlocal t, r
        ok = tv.reserve_pages(dev_i32(n), table, kv, ref, bs)
        want, t, r = ref_pages.reserve(n, t, k, r, bs)
        assert np.array_equal(ok.cpu().numpy(), want)

    def put(new, n, path=None):
        nonlocal k
        for i in range(2):
            host[i], host[2 + i] = (kv_fp8.append(host[i], host[2 + i], t, k, f64(new[i]), n) if path is None
                                    else kv_fp8.commit(host[i], host[2 + i], t, k, f64(new[i]), path, n))
        k = k + np.maximum(n, 0)

    def same():
        assert np.array_equal(table.cpu().numpy(), t) and np.array_equal(kv.cpu().numpy(), k)
        assert np.array_equal(ref.cpu().numpy(), r)
        live = np.unique(t[t >= 0])
        for c, h in zip(cache, host):
            assert np.array_equal(c.view(torch.uint8).cpu().numpy()[live], h[live])

    # prompts of three sequences
    n = np.array([70, 0, 33, 100])
    reserve(n)
    new = rows(100), rows(100)
    tv.append_paged_fp8(*new, *cache, table, kv, n_new=dev_i32(n))
    put(new, n)
    same()
    # sequence 1 continues sequence 3
    tv.fork_pages(dev_i32([3]), dev_i32([1]), table, kv, ref, bs, cache)
    _, cs, cd, t, k, r = ref_pages.fork([3], [1], t, k, r, bs)
    for h in host:
        h[cd[0]] = h[cs[0]]
    same()
    for step in range(4):
        q, kt, vt = rows(N, Hq), rows(N), rows(N)
        tree = np.stack([synth.random_tree(rng, N, 4) for _ in range(B)])
        out = torch.empty_like(q)
        tv.tree_verify_attention_paged_fp8(q, *cache, table, kt, vt, dev_i32(tree), out, kv_len=kv)
        b16 = lambda x: x.view(torch.int16).cpu().numpy().view(np.uint16)  # noqa: E731
        want, tol = oracle_and_bound(b16(q), *host, t, b16(kt), b16(vt), tree, k)
        assert (np.abs(f64(out) - want) <= tol).all()
        path = np.full((B, 5), -1)
        n = rng.integers(1, 5, size=B)
        for b in range(B):
            node = int(rng.integers(0, N))
            line = []
            while node >= 0:
                line.append(node)
                node = tree[b, node]
            line = line[::-1][:n[b]]
            n[b] = len(line)
            path[b, :n[b]] = line
        reserve(n)
        tv.commit_path_paged_fp8(kt, vt, dev_i32(path), dev_i32(n), *cache, table, kv)
        put((kt, vt), n, path)
        same()
        # a single token each
        one = rows(1), rows(1)
        reserve(np.ones(B, int))
        tv.append_paged_fp8(*one, *cache, table, kv)
        put(one, np.ones(B, int))
        same()
    # sequence 3 ends, which leaves the pages that it shares with sequence 1
    tv.free_pages(dev_i32([3]), table, kv, ref)
    t, k, r = ref_pages.free([3], t, k, r)
    same()
    live, src, dst = tv.compact_pages(table, ref, cache)
    want, cs, cd, t, r = ref_pages.compact(t, r)
    for h in host:
        for s, d in zip(cs, cd):
            if s >= 0:
                h[d] = h[s]
    assert int(live) == want
    same()


def test_graph_replays():
    """A step captured once and replayed, with eager work between the replays: every replay gives
    what the eager calls give from the same state."""
    cache, table, kv, ref, rows = serving_state(2)
    tv.reserve_pages(torch.full_like(kv, 180), table, kv, ref, 32)
    tv.append_paged_fp8(rows(90), rows(90), *cache, table, kv)
    q, kt, vt, out = rows(7, 4), rows(7), rows(7), rows(7, 4)
    parent, path, n = dev_i32([[-1, 0, 1, 0, 3, 3, 0]] * 4), dev_i32([[0, 3, 5]] * 4), dev_i32([3, 1, 2, 3])
    state = cache + [table, kv, ref]
    before = [x.clone() for x in state]

    def step():
        tv.tree_verify_attention_paged_fp8(q, *cache, table, kt, vt, parent, out, kv_len=kv)
        tv.commit_path_paged_fp8(kt, vt, path, n, *cache, table, kv)
        tv.append_paged_fp8(kt, vt, *cache, table, kv)
        tv.free_pages(dead, table, kv, ref)
        tv.fork_pages(src, dst, table, kv, ref, 32, cache, ok=said[0], copy_src=said[1], copy_dst=said[2])
        tv.reserve_pages(more, table, kv, ref, 32, ok=ok)
        tv.compact_pages(table, ref, cache, n_live=live, copy_src=moves[0], copy_dst=moves[1])

    dead, src, dst, more = dev_i32([2]), dev_i32([0]), dev_i32([2]), dev_i32([20, 0, 5, 40])
    said = [torch.empty(1, dtype=torch.int32, device="cuda") for _ in range(3)]
    moves = [torch.empty(20, dtype=torch.int32, device="cuda") for _ in range(2)]
    ok, live = (torch.empty(m, dtype=torch.int32, device="cuda") for m in (4, 1))

    def restore():
        for x, y in zip(state, before):
            x.view(torch.uint8).copy_(y.view(torch.uint8))

    def result():
        torch.cuda.synchronize()
        return [x.view(torch.uint8).cpu().clone() for x in state + said + moves + [ok, live, out]]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    eager = result()
    restore()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for _ in range(4):
        restore()
        graph.replay()
        got = result()
        assert all(torch.equal(a, b) for a, b in zip(got, eager))
        restore()
        step()
        got = result()
        assert all(torch.equal(a, b) for a, b in zip(got, eager))


def test_two_streams_at_once():
    """Calls on two streams with workspaces of their own, in flight together."""
    jobs = [attention_args(c) for c in (4, 10)]
    want = []
    for args, kv in jobs:
        tv.tree_verify_attention_paged_fp8(*args, kv_len=kv)
        want.append(bits(args[9]))
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (args, kv) in zip(streams, jobs):
            with torch.cuda.stream(s):
                for _ in range(10):
                    tv.tree_verify_attention_paged_fp8(*args, kv_len=kv)
    torch.cuda.synchronize()
    for (args, _), w in zip(jobs, want):
        assert np.array_equal(bits(args[9]), w)


def test_graphs_of_one_stream_at_once(monkeypatch):
    """Graphs captured on one stream, replayed on two streams at the same time and beside eager
    calls: each has a workspace of its own, cleared by itself, and its calls share it."""
    jobs = [attention_args(c) for c in (4, 10)]
    want = []
    for args, kv in jobs:
        tv.tree_verify_attention_paged_fp8(*args, kv_len=kv)
        want.append(bits(args[9]))
    lib = binding.load_library()
    sizes = [(*a[0].shape[:3], a[6].shape[2], a[0].shape[3], a[5].shape[1] * a[1].shape[2]) for a, _ in jobs]
    assert all(lib.tv_tree_verify_attention_paged_fp8_workspace(*s) > 1 << 15 for s in sizes)  # both split
    given = []
    real = binding._capture_workspace
    assert lib.tv_capture_id(torch.cuda.current_stream().cuda_stream) == 0
    monkeypatch.setattr(binding, "_direct", None)
    monkeypatch.setattr(binding, "_capture_workspace", lambda *a: given.append((a[0], real(*a))) or given[-1][1])
    side = torch.cuda.Stream()
    graphs, outs = [], []
    torch.cuda.synchronize()
    for args, kv in jobs:
        graph = torch.cuda.CUDAGraph()
        outs.append([torch.empty_like(args[9]) for _ in range(3)])
        with torch.cuda.graph(graph, stream=side):
            for out in outs[-1]:
                tv.tree_verify_attention_paged_fp8(*args[:9], out, kv_len=kv)
        graphs.append(graph)
    ids, at = [g[0] for g in given], [g[1].data_ptr() for g in given]
    assert len(ids) == 6 and len(set(ids[:3])) == len(set(ids[3:])) == 1 and ids[0] != ids[3]
    assert len(set(at[:3])) == len(set(at[3:])) == 1 and at[0] != at[3]
    streams = [torch.cuda.Stream() for _ in jobs]
    for turn in range(4):
        for o in outs[0] + outs[1]:
            o.zero_()
        torch.cuda.synchronize()
        for _ in range(6):
            for s, g in zip(streams, graphs):
                with torch.cuda.stream(s):
                    g.replay()
            with torch.cuda.stream(side):
                for args, kv in jobs:
                    tv.tree_verify_attention_paged_fp8(*args, kv_len=kv)
        torch.cuda.synchronize()
        for (args, _), o, w in zip(jobs, outs, want):
            for got in o + [args[9]]:
                assert np.array_equal(bits(got), w)


def test_far_pages():
    """Offsets beyond 32 bits: a pool of more than 4 GiB, whose last pages are the ones in use."""
    Hkv, D, bs = 8, 128, 1024
    nb = (5 << 30) // (Hkv * D * bs)
    k, v = (torch.zeros(nb, Hkv, bs, D, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
            for _ in range(2))
    ke, ve = (torch.zeros(nb, Hkv, bs // 32, dtype=torch.uint8, device="cuda") for _ in range(2))
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    new = [torch.randn(1, 1500, Hkv, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    q, kt, vt = (torch.randn(1, 3, h, D, generator=g, device="cuda").to(torch.bfloat16) for h in (16, 8, 8))
    outs = []
    for pages in ([nb - 1, nb - 2], [0, 5]):
        table, kv = dev_i32([pages]), dev_i32([0])
        tv.append_paged_fp8(*new, k, v, ke, ve, table, kv)
        out = torch.empty_like(q)
        tv.tree_verify_attention_paged_fp8(q, k, v, ke, ve, table, kt, vt, None, out, kv_len=kv)
        outs.append(bits(out))
        assert int(kv) == 1500
    assert np.array_equal(outs[0], outs[1])
    assert torch.equal(k[nb - 1].view(torch.uint8), k[0].view(torch.uint8)) and bool(k[0].view(torch.uint8).any())
    # and through the page calls
    tv.copy_pages(dev_i32([nb - 2]), dev_i32([nb - 3]), [k, v, ke, ve])
    assert torch.equal(v[nb - 3].view(torch.uint8), v[5].view(torch.uint8))


@pytest.mark.parametrize("native", [True, False])
def test_beside_a_graph_of_the_16_bit_call(native, monkeypatch):
    """A graph captured with the 16-bit call, which keeps its stream's workspace, replayed on another
    stream while that stream makes eager 8-bit calls: both split, neither sees the other's partials."""
    if native:
        binding.load_library()
        assert binding._direct is not None
    else:
        monkeypatch.setattr(binding, "_direct", None)
    args, kv = attention_args(10)
    q, table, kt, vt, parent, out = args[0], args[5], args[6], args[7], args[8], args[9]
    B, N, Hq, D = q.shape
    nb, Hkv, bs, _ = args[1].shape
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    pools = [torch.randn(nb, bs, Hkv, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2)]
    lib = binding.load_library()
    sizes = (B, N, Hq, Hkv, D, table.shape[1] * bs)
    assert lib.tv_tree_verify_attention_workspace(*sizes) > 1 << 15
    assert lib.tv_tree_verify_attention_paged_fp8_workspace(*sizes) > 1 << 15
    wide = torch.empty_like(out)

    def bf16_call():
        tv.tree_verify_attention_paged(q, *pools, table, kt, vt, parent, wide, kv_len=kv)

    def fp8_call():
        tv.tree_verify_attention_paged_fp8(*args, kv_len=kv)

    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        bf16_call()
        fp8_call()
    torch.cuda.synchronize()
    want = bits(wide), bits(out)
    held = {key[0]: ws.data_ptr() for key, ws in binding._workspaces.items() if key[2] == side.cuda_stream}
    assert held["attn"] != held["attn_fp8"]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        bf16_call()
    for _ in range(4):
        wide.zero_()
        out.zero_()
        torch.cuda.synchronize()
        for _ in range(10):
            with torch.cuda.stream(other):
                graph.replay()
            with torch.cuda.stream(side):
                fp8_call()
        torch.cuda.synchronize()
        assert np.array_equal(bits(wide), want[0]) and np.array_equal(bits(out), want[1])


def test_native_half_does_every_call(monkeypatch):
    """With the Python half's checks made to raise, every call that has a native half still goes
    through, and with the results that the Python half gives; a native half that declines does not."""
    def steps(cache, table, kv, ref, rows, tree):
        tv.tree_verify_attention_paged_fp8(*args, kv_len=lens)
        yield "attention", [args[9]]
        yield "reserve", [tv.reserve_pages(dev_i32([70, 40, 33, 5]), table, kv, ref, 32), table, ref]
        tv.append_paged_fp8(rows, rows, *cache, table, kv, n_new=dev_i32([70, 40, 33, 0]))
        yield "append", cache + [kv]
        tv.commit_path_paged_fp8(tree, tree, dev_i32([[0, 2, 3]] * 4), dev_i32([3, 2, 1, -1]), *cache, table, kv)
        yield "commit", cache + [kv]
        tv.free_pages(dev_i32([1, 3]), table, kv, ref)
        yield "free", [table, kv, ref]
        said = tv.fork_pages(dev_i32([0, 2]), dev_i32([1, 3]), table, kv, ref, 32, cache)
        yield "fork", list(said) + cache + [table, kv, ref]

    def state():
        cache, table, kv, ref, rows = serving_state(5)
        return cache, table, kv, ref, rows(70), rows(5)

    def run():
        return [(name, [x.view(torch.uint8).cpu().clone() for x in seen]) for name, seen in steps(*state())]

    args, lens = attention_args(8)
    binding.load_library()
    native = binding._direct
    assert native is not None
    monkeypatch.setattr(binding, "_direct", None)
    want = run()
    assert [name for name, _ in want] == ["attention", "reserve", "append", "commit", "free", "fork"]
    monkeypatch.setattr(binding, "_direct", native)

    def raises(*a, **k):
        raise AssertionError("the Python half was asked")

    monkeypatch.setattr(binding, "_need_all", raises)
    args[9].zero_()
    for (name, seen), (_, expect) in zip(run(), want):
        assert all(torch.equal(x, y) for x, y in zip(seen, expect)), name

    class Declines:
        def __init__(self, name):
            self.name = name

        def __getattr__(self, name):
            return (lambda *a: None) if name == self.name else getattr(native, name)

    for name, _ in want:
        monkeypatch.setattr(binding, "_direct", Declines(name))
        with pytest.raises(AssertionError, match="Python half"):
            run()


@pytest.mark.parametrize("error", [KeyboardInterrupt, SystemExit, ValueError])
def test_an_interrupt_is_not_lost_in_the_native_half(error):
    """What is raised while the native half asks for a workspace: an interrupt reaches the caller, and
    nothing is launched; an error of the call is left to the Python half, which meets it again."""
    args, kv = attention_args(4)
    native = binding._direct if binding.load_library() and binding._direct is not None else None
    assert native is not None

    def ask(*a):
        raise error("now")

    def connect(workspace):
        native.connect(binding.load_library()._handle, binding._raw_stream, torch._C._cuda_getDevice, workspace,
                       binding._capture_workspace)

    args[9].fill_(3.0)
    connect(ask)
    try:
        if error is ValueError:
            assert native.attention(*args, kv, None, None) is None
        else:
            with pytest.raises(error):
                native.attention(*args, kv, None, None)
            with pytest.raises(error):
                tv.tree_verify_attention_paged_fp8(*args, kv_len=kv)
    finally:
        connect(binding.workspace)
    torch.cuda.synchronize()
    assert bool((args[9] == 3.0).all())
    assert native.attention(*args, kv, None, None) is args[9]
