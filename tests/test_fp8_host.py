"""Host side of the 8-bit paged cache (no GPU): what its entry points refuse before anything is
launched, in C and in the binding."""
import ctypes

import pytest
import torch

from paper_2606_18394_amd import binding
from test_abi import FAKE, _lib

NULL, SHAPE, UNSUPPORTED, WORKSPACE, ALIGN = -1, -2, -4, -5, -7


def _attn(**kw):
    a = dict(q=FAKE, kp=FAKE, vp=FAKE, ke=FAKE + 1, ve=FAKE + 3, bt=FAKE, bs=64, mb=64, nb=500, kt=FAKE,
             vt=FAKE, parent=None, kv_len=None, out=FAKE, B=4, N=16, Hq=32, Hkv=8, D=128, ws=FAKE,
             wsb=1 << 40)
    assert not set(kw) - set(a)
    a.update(kw)
    return _lib().tv_tree_verify_attention_paged_fp8(
        a["q"], a["kp"], a["vp"], a["ke"], a["ve"], a["bt"], a["bs"], a["mb"], a["nb"], a["kt"], a["vt"],
        a["parent"], a["kv_len"], a["out"], a["B"], a["N"], a["Hq"], a["Hkv"], a["D"],
        ctypes.c_float(0), a["ws"], a["wsb"], None)


@pytest.mark.parametrize("code, bad", [
    (NULL, dict(q=None)), (NULL, dict(kp=None)), (NULL, dict(vp=None)), (NULL, dict(ke=None)),
    (NULL, dict(ve=None)), (NULL, dict(bt=None)), (NULL, dict(nb=0)), (NULL, dict(out=None)),
    (NULL, dict(kt=None)), (NULL, dict(vt=None)), (NULL, dict(kt=None, vt=None)),
    (SHAPE, dict(bs=16)), (SHAPE, dict(bs=48)), (SHAPE, dict(bs=1 << 21)), (SHAPE, dict(mb=-1)),
    (SHAPE, dict(nb=-1)), (SHAPE, dict(B=0)), (SHAPE, dict(N=0)), (SHAPE, dict(Hq=30)), (SHAPE, dict(Hkv=0)),
    (UNSUPPORTED, dict(D=96)), (UNSUPPORTED, dict(N=2049)), (UNSUPPORTED, dict(mb=1 << 25)),
    (UNSUPPORTED, dict(nb=1 << 28, bs=32)), (UNSUPPORTED, dict(nb=(1 << 31) - 1)),
    (ALIGN, dict(q=FAKE + 8)), (ALIGN, dict(kp=FAKE + 8)), (ALIGN, dict(vp=FAKE + 4)),
    (ALIGN, dict(kt=FAKE + 2)), (ALIGN, dict(vt=FAKE + 8)), (ALIGN, dict(out=FAKE + 8)),
    (ALIGN, dict(ws=FAKE + 8)), (WORKSPACE, dict(ws=None, B=1)), (WORKSPACE, dict(wsb=64, B=1)),
])
def test_attention_refuses(code, bad):
    assert _attn(**bad) == code


def test_attention_workspace_query():
    need = _lib().tv_tree_verify_attention_paged_fp8_workspace
    assert need(1, 1, 32, 8, 128, 4096) > 0 and need(1, 1, 32, 8, 128, 0) > 0
    for bad in [(0, 1, 32, 8, 128, 64), (1, 0, 32, 8, 128, 64), (1, 1, 30, 8, 128, 64),
                (1, 1, 32, 8, 96, 64), (1, 2049, 32, 8, 128, 64), (1, 1, 32, 8, 128, -1)]:
        assert need(*bad) == 0


def _tensors():
    f8, bf, i32 = torch.float8_e4m3fn, torch.bfloat16, torch.int32
    return dict(q=torch.zeros(2, 3, 8, 64, dtype=bf), k_pool=torch.zeros(5, 4, 64, 64, dtype=f8),
                v_pool=torch.zeros(5, 4, 64, 64, dtype=f8), k_exp=torch.zeros(5, 4, 2, dtype=torch.uint8),
                v_exp=torch.zeros(5, 4, 2, dtype=torch.uint8), block_table=torch.zeros(2, 2, dtype=i32),
                k_tree=torch.zeros(2, 3, 4, 64, dtype=bf), v_tree=torch.zeros(2, 3, 4, 64, dtype=bf),
                parent=torch.zeros(2, 3, dtype=i32), out=torch.zeros(2, 3, 8, 64, dtype=bf))


def test_binding_refuses_host_tensors_and_types():
    t = _tensors()
    with pytest.raises(ValueError, match="GPU tensor"):
        binding.tree_verify_attention_paged_fp8(**t)
    with pytest.raises(TypeError, match="q must be"):
        binding.tree_verify_attention_paged_fp8(**{**t, "q": t["q"].float()})


def _append(**kw):
    a = dict(k=FAKE, v=FAKE, n=None, kp=FAKE, vp=FAKE, ke=FAKE + 1, ve=FAKE + 3, bt=FAKE, bs=64, mb=64,
             nb=500, kv=FAKE, B=4, T=16, Hkv=8, D=128)
    assert not set(kw) - set(a)
    a.update(kw)
    return _lib().tv_append_paged_fp8(
        a["k"], a["v"], a["n"], a["kp"], a["vp"], a["ke"], a["ve"], a["bt"], a["bs"], a["mb"], a["nb"],
        a["kv"], a["B"], a["T"], a["Hkv"], a["D"], None)


def _commit(**kw):
    a = dict(k=FAKE, v=FAKE, path=FAKE, n=FAKE, kp=FAKE, vp=FAKE, ke=FAKE + 1, ve=FAKE + 3, bt=FAKE, bs=64,
             mb=64, nb=500, kv=FAKE, B=4, N=16, Hkv=8, D=128, Dmax=5)
    assert not set(kw) - set(a)
    a.update(kw)
    return _lib().tv_commit_path_paged_fp8(
        a["k"], a["v"], a["path"], a["n"], a["kp"], a["vp"], a["ke"], a["ve"], a["bt"], a["bs"], a["mb"],
        a["nb"], a["kv"], a["B"], a["N"], a["Hkv"], a["D"], a["Dmax"], None)


WRITE = [
    (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(kp=None)), (NULL, dict(vp=None)),
    (NULL, dict(ke=None)), (NULL, dict(ve=None)), (NULL, dict(bt=None)), (NULL, dict(kv=None)),
    (SHAPE, dict(B=0)), (SHAPE, dict(Hkv=0)), (SHAPE, dict(mb=0)), (SHAPE, dict(nb=0)), (SHAPE, dict(bs=33)),
    (SHAPE, dict(bs=16)), (UNSUPPORTED, dict(D=32)), (UNSUPPORTED, dict(mb=1 << 30)),
    (UNSUPPORTED, dict(nb=1 << 30)), (UNSUPPORTED, dict(B=(1 << 31) - 1)),
    (ALIGN, dict(k=FAKE + 8)), (ALIGN, dict(v=FAKE + 2)), (ALIGN, dict(kp=FAKE + 8)),
    (ALIGN, dict(vp=FAKE + 8)),
]


@pytest.mark.parametrize("code, bad", WRITE + [(SHAPE, dict(T=0))])
def test_append_refuses(code, bad):
    assert _append(**bad) == code


@pytest.mark.parametrize("code, bad", WRITE + [(SHAPE, dict(N=0)), (SHAPE, dict(Dmax=0)),
                                               (UNSUPPORTED, dict(N=2049)), (NULL, dict(path=None)),
                                               (NULL, dict(n=None))])
def test_commit_refuses(code, bad):
    assert _commit(**bad) == code


def _pools(n, size=64, base=FAKE):
    return (ctypes.c_void_p * n)(*[base] * n), (ctypes.c_int64 * n)(*[size] * n), n


def test_page_calls_refuse():
    lib = _lib()

    def reserve(n=FAKE, bt=FAKE, kv=FAKE, ref=FAKE, ok=FAKE, B=4, mb=8, bs=64, nb=100):
        return lib.tv_reserve_pages(n, bt, kv, ref, ok, B, mb, bs, nb, None)

    def fork(src=FAKE, dst=FAKE, n=3, bt=FAKE, kv=FAKE, ref=FAKE, B=4, mb=8, bs=64, nb=100, pools=_pools(2),
             ok=FAKE, cs=FAKE, cd=FAKE):
        return lib.tv_fork_pages(src, dst, n, bt, kv, ref, B, mb, bs, nb, *pools, ok, cs, cd, None)

    def free(seqs=FAKE, n=3, bt=FAKE, kv=FAKE, ref=FAKE, B=4, mb=8, nb=100):
        return lib.tv_free_pages(seqs, n, bt, kv, ref, B, mb, nb, None)

    def copy(src=FAKE, dst=FAKE, n=3, nb=100, pools=_pools(2)):
        return lib.tv_copy_pages(src, dst, n, nb, *pools, None)

    def compact(bt=FAKE, ref=FAKE, B=4, mb=8, nb=100, pools=_pools(2), live=FAKE, cs=FAKE, cd=FAKE, ws=FAKE,
                wsb=1 << 20):
        return lib.tv_compact_pages(bt, ref, B, mb, nb, *pools, live, cs, cd, ws, wsb, None)

    for call in (reserve, fork, free):
        assert call(bt=None) == call(kv=None) == call(ref=None) == NULL
        assert call(B=0) == call(mb=0) == call(nb=0) == SHAPE
        assert call(nb=(1 << 30) + 1) == call(B=1 << 20, mb=1 << 20) == UNSUPPORTED
    for call in (reserve, fork):
        assert call(bs=0) == call(bs=-64) == call(bs=48) == call(bs=16) == SHAPE
        assert call(mb=1 << 28) == UNSUPPORTED and call(ok=None) == NULL
    assert reserve(n=None) == NULL and reserve(B=4097) == UNSUPPORTED
    for call in (fork, copy):
        assert call(src=None) == call(dst=None) == NULL and call(n=0) == SHAPE
    assert fork(n=1025) == UNSUPPORTED and fork(cs=None) == fork(cd=None) == NULL
    assert free(seqs=None) == NULL and free(n=0) == SHAPE and free(n=4097) == UNSUPPORTED
    for call in (fork, copy, compact):
        assert call(pools=_pools(65)) == UNSUPPORTED and call(pools=(None, None, 2)) == NULL
        assert call(pools=_pools(2, base=None)) == NULL and call(pools=_pools(2, size=0)) == SHAPE
        assert call(pools=(*_pools(2)[:2], -1)) == SHAPE
        assert call(pools=_pools(2, size=1 << 35)) == UNSUPPORTED
    assert copy(nb=0) == copy(pools=_pools(0)) == SHAPE
    assert compact(bt=None) == compact(ref=None) == compact(live=None) == compact(cs=None) == NULL
    assert compact(ws=None) == compact(wsb=400) == WORKSPACE and compact(ws=FAKE + 8) == ALIGN
    need = lib.tv_compact_pages_workspace
    assert need(1) >= 4 and need(0) == need(-5) == need((1 << 30) + 1) == 0


def test_binding_checks_pages():
    i32 = torch.int32
    bt, kv, ref = torch.zeros(2, 3, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(5, dtype=i32)
    for call in (lambda: binding.reserve_pages(kv, bt, kv, ref, 64),
                 lambda: binding.fork_pages(kv, kv, bt, kv, ref, 64),
                 lambda: binding.free_pages(kv, bt, kv, ref),
                 lambda: binding.copy_pages(kv, kv, [torch.zeros(5, 4)]),
                 lambda: binding.compact_pages(bt, ref)):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()
    with pytest.raises(ValueError, match="at least one pool"):
        binding.copy_pages(kv, kv, [])
    with pytest.raises(ValueError, match="expected 5 pages"):
        binding._pool_arrays([torch.zeros(4, 2)], 5, torch.device("cpu"), -1)
    t = _tensors()
    with pytest.raises(ValueError, match="GPU tensor"):
        binding.append_paged_fp8(t["k_tree"], t["v_tree"], t["k_pool"], t["v_pool"], t["k_exp"],
                                 t["v_exp"], bt, kv)
    with pytest.raises(ValueError, match="GPU tensor"):
        binding.commit_path_paged_fp8(t["k_tree"], t["v_tree"], bt, kv, t["k_pool"], t["v_pool"],
                                      t["k_exp"], t["v_exp"], bt, kv)


def test_native_half_declines_what_is_not_ordinary():
    """The native half of the binding answers None for anything that it does not do: tensors of
    the host, other types, wrong numbers of arguments, things that are no tensors."""
    _lib()
    if binding._direct is None:
        from paper_2606_18394_amd import build
        build.build_direct()
        binding._connect(binding.load_library())
    d, t = binding._direct, _tensors()
    i32 = torch.int32
    bt, kv, ref = torch.zeros(2, 3, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(5, dtype=i32)
    cache = [t[k] for k in ("k_pool", "v_pool", "k_exp", "v_exp", "block_table")]
    calls = [(d.attention, [t["q"]] + cache + [t["k_tree"], t["v_tree"], t["parent"], t["out"], kv, None, None]),
             (d.append, [t["k_tree"], t["v_tree"]] + cache + [kv, None]),
             (d.commit, [t["k_tree"], t["v_tree"], bt, kv] + cache + [kv]),
             (d.reserve, [kv, bt, kv, ref, 64]), (d.fork, [kv, kv, bt, kv, ref, 64, ()]),
             (d.free, [kv, bt, kv, ref])]
    for call, args in calls:
        assert call(*args) is None
        assert call() is None and call(*args[:-1]) is None
        for i in range(len(args)):
            for other in (None, 7, "x", torch.zeros(3)):
                assert call(*args[:i], other, *args[i + 1:]) is None
