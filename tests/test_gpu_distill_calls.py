"""Calls of the teacher's and the student's operators that their documentation allows, or that
they refuse, beyond ordinary batches."""
import math

import pytest
import torch

from test_gpu_distill import E, LSE, definition, distill, lists
from test_gpu_distill import test_many_long_rows as many_long_rows
from test_gpu_distill_head import BASE, D, setup
from tests.gpu_cases import Case, workload
from workloads import get_config

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [0, 257, 5000])
def test_lists_of_a_length_that_is_refused(k):
    """Before any work, whatever the length."""
    from paper_2606_04484_amd import actor, capi
    case = Case(workload(get_config(0).model))
    L = actor.merge(actor.upload_timelines(case.tl, case.old))
    A = actor.ActorUpdate(case.m, case.device_weights())
    A.zero_grads()
    with pytest.raises(capi.AjError, match="lists of"):
        A.teacher_topk(L, k)
    idx = torch.zeros(L.n_mask, k, dtype=torch.int32, device="cuda")
    with pytest.raises(capi.AjError, match="lists of"):
        A.distill_step(L, idx, idx.float())
    torch.cuda.synchronize()
    assert all(not bool(g.any()) for g in A.G.values())


@pytest.mark.parametrize("tail", [False, True], ids=["listed", "tail"])
@pytest.mark.parametrize("dtype, grad", [("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("vocab, k, pad, offset", [(45056, 30, 0, 0), (73728, 9, 5, 3), (196592, 16, 0, 0),
                                                   (196593, 64, 1, 0), (262144, 33, 3, 5), (270320, 8, 0, 0),
                                                   (270321, 5, 0, 1)])
def test_ends_of_the_ranges_of_long_rows(vocab, k, pad, offset, dtype, grad, tail):
    """A workgroup's share of a row, at the sizes where the ways of forming its gradient change."""
    many_long_rows(vocab, k, pad, offset, dtype, grad, tail)


@pytest.mark.parametrize("part", ["step", "apart"])
@pytest.mark.parametrize("vocab, masked", [(40, False), (256, False), (3000, True), (20000, True)])
def test_a_list_of_all_that_the_student_can_say(vocab, masked, part):
    """What rounding leaves of the teacher's 1 is no class of its own where the student has
    nothing outside the list; a mass that is really missing there is."""
    g = torch.Generator().manual_seed(vocab)
    rows, k = 64, min(vocab, 200)
    z = torch.randn(rows, vocab, generator=g)
    if masked:
        z[:, k:] = -math.inf
    k = k if masked else vocab
    lp = torch.log_softmax(torch.randn(rows, k, generator=g) * 2, 1)
    idx = torch.stack([torch.randperm(k, generator=g) for _ in range(rows)]).to(torch.int32)
    left = 1 - lp.double().exp().sum(1)
    assert bool((left > 0).any()) and bool((left < 0).any()) and bool((left.abs() < 2 ** -14).all())
    loss, _, dz, stats, _ = distill(z.cuda(), 1.0, idx, lp, True, None, 1.0, "f32", part=part)
    want = definition(z, 1.0, idx, lp, False, torch.ones(rows).double())
    # the lists' own sum is 1 to within 2^-14, no more is known of the teacher
    assert bool(((loss - want[0]).abs() <= left.abs() * (2 + want[0]) + 3 * LSE + 8 * E * (40 + want[0])).all())
    assert bool(((dz - want[2]).abs() <= (left.abs()[:, None] + LSE + 300 * E) * want[3] + 1e-30).all())
    assert math.isfinite(float(stats[0]))
    # a token that the teacher gives a mass, and neither the list nor the student holds
    gone = idx[:, 3:4].long().clone()
    z.scatter_(1, gone, -math.inf)
    idx[:, 3] = -1
    loss = distill(z.cuda(), 1.0, idx, lp, True, None, 1.0, "f32", part=part)[0]
    missing = 1 - torch.where(idx >= 0, lp.double().exp(), 0.0).sum(1)
    assert torch.equal(loss == math.inf, missing > 2 ** -14) and bool((missing > 2 ** -14).any())


@pytest.mark.parametrize("part", ["step", "apart"])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab", [(7, 2000), (6, 70001), (513, 90000)])
def test_rows_of_weight_zero(rows, vocab, grad, part):
    """A row of weight 0 may hold anything: no gradient, no share of the sum; the others' as ever."""
    g = torch.Generator().manual_seed(rows)
    few = min(rows, 7)
    z = torch.randn(few, vocab, generator=g)
    idx, lp = lists(z, 20, 3, 1.0)
    w = torch.rand(few, generator=g) + 0.5
    w[1::2] = 0
    bad, blp = z.clone(), lp.clone()
    bad[1], bad[3, 5], bad[5, ::2] = math.nan, math.inf, -math.inf
    blp[1, 2] = blp[3] = math.nan
    if few > 5:
        blp[5, 0] = math.inf
    at = torch.arange(rows) % few
    a = distill(z[at].cuda(), 1.0, idx[at], lp[at], True, w[at], 0.5, grad, part=part)
    b = distill(bad[at].cuda(), 1.0, idx[at], blp[at], True, w[at], 0.5, grad, part=part)
    on = w[at] > 0
    assert bool((b[2][~on] == 0).all()) and torch.equal(a[2], b[2])
    assert torch.equal(a[0][on], b[0][on]) and torch.equal(a[3], b[3])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("n_tok, n_tgt", [(5, 3), (900, 700), (8600, 8400)])
def test_the_teacher_stays_in_its_workspace(n_tok, n_tgt, dtype):
    from paper_2606_04484_amd import capi
    cfg, h, gamma, w, rows, targets = setup(n_tok, n_tgt, dtype)
    res = []
    for query in (capi.aj_lm_head_topk_workspace_bytes, capi.aj_lm_head_workspace_bytes):
        size = query(cfg, n_tgt, 11)
        ws = torch.full((size + 4096,), 255, dtype=torch.uint8, device="cuda")
        idx = torch.zeros(n_tgt, 11, dtype=torch.int32, device="cuda")
        lp, lse = torch.zeros(n_tgt, 11, device="cuda"), torch.zeros(n_tgt, device="cuda")
        capi.aj_lm_head_topk(cfg, targets.cuda(), h.cuda(), gamma.cuda(), w.cuda(), 1.0, idx, lp, lse, ws[:size],
                             row_base=BASE)
        torch.cuda.synchronize()
        assert bool((ws[size:] == 255).all())
        res.append((idx, lp, lse))
    assert all(torch.equal(a, b) for a, b in zip(*res))


@pytest.mark.parametrize("vocab", [257, 1003])
@pytest.mark.parametrize("n_tok, n_tgt", [(70, 33), (700, 600)])
def test_head_of_an_odd_vocabulary_in_half_precision(n_tok, n_tgt, vocab):
    """bfloat16 weights of a vocabulary that is no multiple of 8: loss, d h, d W and d gamma
    against the definition on the same numbers, with what rounding the normalised rows and
    d logits to bfloat16 allows."""
    from paper_2606_04484_amd import capi
    g = torch.Generator().manual_seed(vocab)
    dt = torch.bfloat16
    h = (torch.randn(n_tok, D, generator=g) * 2).to(dt)
    gamma = (1 + 0.3 * torch.randn(D, generator=g)).to(dt)
    W = (torch.randn(vocab, D, generator=g) * 0.4).to(dt)
    rows = torch.randperm(n_tok, generator=g)[:n_tgt].sort().values
    cfg = capi.LossCfg(D, vocab, 1 << 14, 0.2, 1e-6, capi.AJ_BF16, 0)
    x, gm, w = h.double()[rows], gamma.double(), W.double()
    r = (x.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    exact = x * r * gm
    hn = exact.to(dt).double()            # a row is normalised in float32 and rounded once
    idx, lp = lists((hn @ w.T).float(), 9, 3, 1.0)
    loss, sw, dz, size = definition(hn @ w.T, 1.0, idx, lp, True, torch.ones(n_tgt))
    t = capi.teacher(idx.cuda(), lp.cuda(), tail=True)
    z = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    ws = torch.full((capi.aj_lm_head_workspace_bytes(cfg, n_tgt, 9),), 255, dtype=torch.uint8, device="cuda")
    out, dh, dg, dw = z(n_tgt), z(n_tok, D).fill_(7.0), z(D), z(vocab, D)
    capi.aj_lm_head_distill(cfg, (rows + 1 + BASE).to(torch.int32).cuda(), h.cuda(), gamma.cuda(), W.cuda(), 1.0, t, out,
                            dh, dg, dw, ws, row_base=BASE)
    torch.cuda.synchronize()
    # a normalised value next to the middle of two of its type may be rounded the other way: a
    # step of bfloat16, where its float32 value is within (D / 2 + 8) 2^-24 of the middle
    a = E * (D / 2 + 8)
    step = 2.0 ** (torch.floor(torch.log2(exact.abs())) - 7)
    flip = torch.where((exact - hn).abs() + a * exact.abs() >= step / 2, step, 0.0)
    assert float((flip > 0).double().mean()) < 0.01
    b = (flip @ w.abs().T + E * (D + 4) * (hn.abs() @ w.abs().T)).amax(1, keepdim=True)
    assert bool(((out.cpu() - loss).abs() <= 2.1 * b[:, 0] + 3 * LSE + 8 * E * (sw[0].abs() + loss.abs())).all())
    u = 2.0 ** -8
    ddz = (4.2 * b + LSE + 6 * E * (sw[0].abs()[:, None] + 40)) * size * 1.01 + 1e-37
    ddz = ddz + u * (dz.abs() + ddz)                                # d logits are rounded
    top = dz.abs() + ddz
    want = dz.T @ hn
    room = ddz.T @ (hn.abs() + flip) + dz.abs().T @ flip + E * (n_tgt + 8) * top.T @ hn.abs()
    assert bool(((dw.cpu() - want).abs() <= room + E * want.abs()).all())
    dhn, ddhn = dz @ w, ddz @ w.abs() + E * (vocab + 8) * top @ w.abs()
    back = lambda v, s: r * v + s * x.abs() * r ** 3 / D * (v * x.abs()).sum(1, keepdim=True)  # noqa: E731
    dx = r * gm * dhn - x * r ** 3 / D * (gm * dhn * x).sum(1, keepdim=True)
    mag = gm.abs() * (dhn.abs() + ddhn)
    assert bool(((dh.cpu()[rows] - dx).abs() <= back(gm.abs() * ddhn, 1) + E * (3 * D + 40) * back(mag, 1)).all())
    wg = (dhn * x * r).sum(0)
    room = (ddhn * x.abs() * r).sum(0) + E * (n_tgt + D + 24) * ((dhn.abs() + ddhn) * x.abs() * r).sum(0)
    assert bool(((dg.cpu() - wg).abs() <= room).all())
    rest = torch.ones(n_tok, dtype=torch.bool)
    rest[rows] = False
    assert bool((dh.cpu()[rest] == 0).all())


def test_lists_that_are_no_matrix():
    from paper_2606_04484_amd import actor, capi
    cfg, h, gamma, w, rows, targets = setup(50, 20, torch.float32)
    flat = torch.zeros(20, dtype=torch.int32, device="cuda")
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    with pytest.raises(capi.AjError, match="idx must be a matrix"):
        capi.aj_lm_head_topk(cfg, targets.cuda(), h.cuda(), gamma.cuda(), w.cuda(), 1.0, flat, flat.float(),
                             flat.float(), ws, row_base=BASE)
    case = Case(workload(get_config(0).model))
    L = actor.merge(actor.upload_timelines(case.tl, case.old))
    A = actor.ActorUpdate(case.m, case.device_weights())
    flat = torch.zeros(L.n_mask, dtype=torch.int32, device="cuda")
    with pytest.raises(capi.AjError, match="lists"):
        A.distill_step(L, flat, flat.float())


def test_teacher_and_student_of_one_object_keep_their_workspaces():
    """A graph of one call holds on to its workspace while the other is made."""
    from paper_2606_04484_amd import actor
    case = Case(workload(get_config(0).model))
    L = actor.merge(actor.upload_timelines(case.tl, case.old))
    A = actor.ActorUpdate(case.m, case.device_weights())
    A.zero_grads()
    idx, lp = A.teacher_topk(L, 8)
    at = A.tws.data_ptr()
    A.distill_step(L, idx, lp)
    own = A.hws.data_ptr()
    again = A.teacher_topk(L, 8)
    torch.cuda.synchronize()
    assert A.tws.data_ptr() == at and A.hws.data_ptr() == own != at
    assert torch.equal(again[0], idx) and torch.equal(again[1], lp)
