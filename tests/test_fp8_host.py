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
