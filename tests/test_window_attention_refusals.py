"""What aj_attention_fwd / _bwd refuse, on the host, before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2606_04484_amd import capi
from paper_2606_04484_amd.capi import AjError

P = C.c_void_p(16)


def raw(cfg=None, vl=None, ws_bytes=1 << 40, qkv=P, bwd=False):
    cfg = cfg or capi.AttnCfg(4, 2, 64, 16, 2, capi.AJ_BF16, 0.0)
    vl = vl or capi.Varlen(10, 1, 10, 0, P, None)
    L = capi.lib()
    if bwd:
        return L.aj_attention_bwd(C.byref(cfg), C.byref(vl), qkv, P, P, P, P, P, ws_bytes, None)
    return L.aj_attention_fwd(C.byref(cfg), C.byref(vl), qkv, P, P, P, ws_bytes, None)


@pytest.mark.parametrize("bwd", [False, True], ids=["fwd", "bwd"])
@pytest.mark.parametrize("fields, status", [
    ((4, 3, 64, 16, 2, 1, 0.0), 2), ((0, 1, 64, 16, 2, 1, 0.0), 2), ((4, 0, 64, 16, 2, 1, 0.0), 2),
    ((4, 2, 136, 16, 2, 1, 0.0), 3), ((4, 2, 12, 16, 2, 1, 0.0), 3), ((4, 2, 64, -1, 2, 1, 0.0), 2),
    ((4, 2, 64, 16, -1, 1, 0.0), 2), ((4, 2, 64, 16, 2, 7, 0.0), 3),
    ((4, 2, 64, 16, 2, 1, -1.0), 2), ((4, 2, 64, 16, 2, 1, float("nan")), 2),
    ((4, 2, 64, 16, 2, 1, float("inf")), 2)])
def test_configuration(fields, status, bwd):
    assert raw(cfg=capi.AttnCfg(*fields), bwd=bwd) == status


@pytest.mark.parametrize("bwd", [False, True], ids=["fwd", "bwd"])
def test_sizes_pointers_workspace(bwd):
    assert raw(vl=capi.Varlen(-1, 1, 10, 0, P, None), bwd=bwd) == 2
    assert raw(vl=capi.Varlen(10, 0, 10, 0, P, None), bwd=bwd) == 2
    assert raw(vl=capi.Varlen(10, 1, 10, 0, None, None), bwd=bwd) == 1
    assert raw(vl=capi.Varlen((1 << 30) + 1, 1, 10, 0, P, None), bwd=bwd) == 2
    assert raw(cfg=capi.AttnCfg(8, 2, 64, 16, 2, 1, 0.0), vl=capi.Varlen(1 << 30, 1, 10, 0, P, None),
               bwd=bwd) == 2
    assert raw(qkv=None, bwd=bwd) == 1
    assert raw(ws_bytes=8, bwd=bwd) == 4
    assert raw(vl=capi.Varlen(0, 0, 0, 0, None, None), bwd=bwd) == 0    # nothing to do


def test_block_refuses_negative_windows():
    cfg = capi.BlockCfg(128, 4, 4, 32, 512, 1e-6, 1e6, 0, -1, 0)
    w = capi.BlockWeights(*[P] * 6)
    vl = capi.Varlen(0, 0, 0, 0, None, None)
    assert capi.lib().aj_varlen_block_fwd(C.byref(cfg), C.byref(w), C.byref(vl), None, None, None,
                                          None, 0, None) == 2


def test_operands_must_fit():
    """The binding looks at types, shapes, order and place before it hands pointers on."""
    cfg = capi.attn_cfg(4, 2, 64, window=16, n_sink=2)
    n = 10
    ok = dict(qkv=torch.zeros(n, 512, dtype=torch.bfloat16), out=torch.zeros(n, 256, dtype=torch.bfloat16),
              lse=torch.zeros(4, n))
    cu, ws = torch.tensor([0, n], dtype=torch.int32), torch.zeros(1 << 20, dtype=torch.uint8)

    def call(**kw):
        a = {**ok, **kw}
        capi.aj_attention_fwd(cfg, kw.get("cu", cu), n, a["qkv"], a["out"], a["lse"], ws)

    with pytest.raises(AjError, match="current GPU"):
        call()                                              # host tensors
    with pytest.raises(AjError, match="out must be"):
        call(out=torch.zeros(n, 256))
    with pytest.raises(AjError, match="lse must be"):
        call(lse=torch.zeros(n, 4))
    with pytest.raises(AjError, match="qkv must be"):
        call(qkv=torch.zeros(n, 500, dtype=torch.bfloat16))
    with pytest.raises(AjError, match="contiguous"):
        call(qkv=torch.zeros(512, n, dtype=torch.bfloat16).t())
    with pytest.raises(AjError, match="cu_seqlens must be"):
        call(cu=torch.tensor([0, n]))
    with pytest.raises(AjError, match="unsupported dtype"):
        capi.attn_cfg(4, 2, 64, dtype=torch.float16)
