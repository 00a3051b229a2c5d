"""What the top-k and distillation calls refuse, on the host, before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2606_04484_amd import capi
from paper_2606_04484_amd.capi import AjError

P = C.c_void_p(16)
BIG = 1 << 40


def lg(rows=4, vocab=100, ld=100, dtype=0, inv_temp=1.0, logits=P):
    return capi.Logits(rows, vocab, ld, dtype, inv_temp, logits)


def teach(k=8, idx=P, logprob=P):
    return capi.Teacher(k, 1, idx, logprob, None, 1.0)


def status(x, t=None, k=8, ws=BIG, what="topk", d_dtype=0, ldd=100, dz=P):
    L = capi.lib()
    x, t = C.byref(x), C.byref(t or teach())
    if what == "topk":
        return L.aj_topk_logprob(x, k, P, P, P, P, ws, None)
    if what == "fwd":
        return L.aj_distill_loss_fwd(x, t, P, P, None, None, P, ws, None)
    if what == "bwd":
        return L.aj_distill_loss_bwd(x, t, P, dz, ldd, d_dtype, None)
    return L.aj_distill_loss_fwd_bwd(x, t, P, P, None, None, dz, ldd, d_dtype, P, ws, None)


ALL = pytest.mark.parametrize("what", ["topk", "fwd", "bwd", "fwd_bwd"])


@ALL
@pytest.mark.parametrize("kw, want", [
    (dict(dtype=3), 3), (dict(rows=-1), 2), (dict(vocab=0), 2), (dict(vocab=(1 << 24) + 1, ld=1 << 25), 2),
    (dict(ld=99), 2), (dict(inv_temp=0.0), 2), (dict(inv_temp=-1.0), 2), (dict(inv_temp=float("nan")), 2),
    (dict(inv_temp=float("inf")), 2), (dict(logits=None), 1), (dict(logits=C.c_void_p(18)), 2),
    (dict(rows=1 << 30), 2)])
def test_logits(kw, want, what):
    assert status(lg(**kw), what=what) == want


@ALL
def test_nothing_to_do(what):
    assert status(lg(rows=0, logits=None), what=what) == 0


@pytest.mark.parametrize("k", [0, -1, 257, 101])
def test_topk_k(k):
    assert status(lg(), k=k) == 2


@pytest.mark.parametrize("what", ["fwd", "bwd", "fwd_bwd"])
def test_teacher(what):
    assert status(lg(), teach(k=0), what=what) == 2
    assert status(lg(), teach(k=257), what=what) == 2
    assert status(lg(), teach(idx=None), what=what) == 1
    assert status(lg(), teach(logprob=None), what=what) == 1


@pytest.mark.parametrize("what", ["topk", "fwd", "fwd_bwd"])
def test_workspace(what):
    assert status(lg(), ws=4, what=what) == 4


@pytest.mark.parametrize("what", ["bwd", "fwd_bwd"])
def test_gradient(what):
    assert status(lg(), what=what, d_dtype=2) == 3
    assert status(lg(), what=what, ldd=99) == 2
    assert status(lg(), what=what, dz=None) == 1
    assert status(lg(), what=what, dz=C.c_void_p(33)) == 2
    # over the logits: only as they lie
    assert status(lg(), what=what, dz=P, d_dtype=1) == 2
    assert status(lg(), what=what, dz=P, ldd=104) == 2


def test_binding_looks_at_its_operands():
    z, i32 = torch.zeros(4, 100), torch.int32
    idx, lp = torch.zeros(4, 8, dtype=i32), torch.zeros(4, 8)
    loss, lse, ws = torch.zeros(4), torch.zeros(2, 4), torch.zeros(1 << 20, dtype=torch.uint8)
    with pytest.raises(AjError, match="current GPU"):
        capi.aj_topk_logprob(z, 1.0, idx, lp, loss, ws)
    with pytest.raises(AjError, match="logprob must be"):
        capi.aj_topk_logprob(z, 1.0, idx, lp[:, :7], loss, ws)
    with pytest.raises(AjError, match="rows of logits must be contiguous"):
        capi.aj_topk_logprob(torch.zeros(100, 4).t(), 1.0, idx, lp, loss, ws)
    with pytest.raises(AjError, match="unsupported dtype"):
        capi.aj_topk_logprob(z.half(), 1.0, idx, lp, loss, ws)
    with pytest.raises(AjError, match="must be a matrix"):
        capi.aj_topk_logprob(z[0], 1.0, idx, lp, loss, ws)
    t = capi.teacher(idx, lp)
    with pytest.raises(AjError, match="lse must be"):
        capi.aj_distill_loss_fwd(z, 1.0, t, loss, lse.t().contiguous(), ws)
    with pytest.raises(AjError, match="idx must be"):
        capi.aj_distill_loss_fwd(z, 1.0, capi.teacher(idx.long(), lp), loss, lse, ws)
    with pytest.raises(AjError, match="weight must be"):
        capi.aj_distill_loss_fwd(z, 1.0, capi.teacher(idx, lp, weight=loss[:3]), loss, lse, ws)
    with pytest.raises(AjError, match="loss must be"):
        capi.aj_distill_loss_fwd(z, 1.0, t, None, lse, ws)


def head(what, cfg=None, n_tok=10, n_tgt=4, targets=P, k=8, inv_temp=1.0, ws=BIG, w_t=None, dh=P, h=P):
    L = capi.lib()
    cfg = cfg or capi.LossCfg(64, 100, 128, 0.2, 1e-6, 1, 0)
    a = capi.LossIn(n_tok, n_tgt, 0, targets, None, None, None, 0.0, None, 0.0, w_t)
    if what == "topk":
        return L.aj_lm_head_topk(C.byref(cfg), C.byref(a), h, P, P, inv_temp, k, P, P, P, None, P, ws, None)
    return L.aj_lm_head_distill(C.byref(cfg), C.byref(a), h, P, P, inv_temp, C.byref(teach(k=k)), P, None, dh, P, P,
                                None, P, ws, None)


@pytest.mark.parametrize("what", ["topk", "distill"])
def test_lm_head(what):
    assert head(what, cfg=capi.LossCfg(60, 100, 128, 0.2, 1e-6, 1, 0)) == 2      # d_model % 8
    assert head(what, cfg=capi.LossCfg(64, 0, 128, 0.2, 1e-6, 1, 0)) == 2
    assert head(what, cfg=capi.LossCfg(64, 100, 128, 0.2, 0.0, 1, 0)) == 2
    assert head(what, cfg=capi.LossCfg(64, 100, 128, 0.2, 1e-6, 2, 0)) == 3
    assert head(what, n_tgt=11) == 2
    assert head(what, n_tgt=-1) == 2
    assert head(what, targets=None) == 1
    assert head(what, k=0) == 2 and head(what, k=257) == 2
    assert head(what, inv_temp=0.0) == 2 and head(what, inv_temp=float("nan")) == 2
    assert head(what, w_t=P) == 2                                                # vocab % 8
    assert head(what, h=None) == 1
    assert head(what, ws=64) == 4
    assert head(what, n_tok=0, n_tgt=0) == 0


def test_lm_head_own():
    assert head("topk", k=101) == 2          # more than the vocabulary
    assert head("distill", dh=None) == 1
