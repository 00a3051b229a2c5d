"""A teacher's top logits and the loss from them against their definitions in 64 bits, within
the error that float32 sums and the results' types allow."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
E = 2.0 ** -24      # half a step of float32, relative
# The log-sum-exp: a thread adds at most 512 terms in a row, waves and workgroups 14 more;
# the exponent of a term is off by 3 roundings of its distance from the maximum, whose
# mean under the probabilities is at most log(vocab) < 17 (in log2 units 25).
LSE = (512 + 14 + 3 * 25) * E
# ... and of sums that random signs of the roundings keep far below that: what is asserted
# is the bound, not the typical error.


def make(rows, vocab, dtype, pad, seed=0, std=2.5, offset=0):
    """Rows that start `offset` elements past a 16-byte boundary and lie vocab + pad apart."""
    g = torch.Generator().manual_seed(seed)
    z = (torch.randn(rows, vocab, generator=g) * std).to(DT[dtype])
    buf = torch.full((offset + rows * (vocab + pad) + 8,), float("nan"), dtype=DT[dtype], device="cuda")
    view = buf[offset:offset + rows * (vocab + pad)].view(rows, vocab + pad)[:, :vocab]
    view.copy_(z)
    return z, view


def place(z):
    """Indices in the documented order: larger first, NaN before all, equal ones by index."""
    key = torch.where(torch.isnan(z), math.inf, z.double())
    first = torch.isnan(z).to(torch.int8)
    at = torch.sort(key, dim=1, descending=True, stable=True).indices
    return at.gather(1, torch.sort(first.gather(1, at), dim=1, descending=True, stable=True).indices)


def topk(z, view, k, inv_temp=1.0, rows_ws=None):
    from paper_2606_04484_amd import capi
    rows, vocab = z.shape
    idx = torch.full((rows, k), -7, dtype=torch.int32, device="cuda")
    lp, lse = torch.full((rows, k), 9.0, device="cuda"), torch.full((rows,), 9.0, device="cuda")
    ws = torch.full((capi.aj_topk_workspace_bytes(rows_ws or rows, vocab, k),), 255, dtype=torch.uint8,
                    device="cuda")
    capi.aj_topk_logprob(view, inv_temp, idx, lp, lse, ws)
    torch.cuda.synchronize()
    return idx.cpu(), lp.cpu(), lse.cpu()


TOPK = [(1, 1, 1, 0, 0), (3, 5, 5, 0, 0), (2, 300, 256, 3, 1), (5, 1024, 8, 0, 0), (4, 2000, 1, 5, 3),
        (7, 4096, 64, 1, 1), (1, 151936, 64, 0, 0), (13, 20001, 100, 0, 5), (14, 20001, 256, 24, 0),
        (300, 16384, 20, 0, 0), (33, 65541, 256, 7, 2)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, vocab, k, pad, offset", TOPK)
def test_topk(rows, vocab, k, pad, offset, dtype):
    z, view = make(rows, vocab, dtype, pad, offset=offset)
    inv = 1 / 1.5
    idx, lp, lse = topk(z, view, k, inv)
    at = place(z)[:, :k]
    assert torch.equal(idx.long(), at)
    zz = z.double() * torch.tensor(inv, dtype=torch.float32).double()
    want = torch.logsumexp(zz, 1)
    assert bool(((lse - want).abs() <= LSE + 2 * E * want.abs()).all())
    lpw = zz.gather(1, at) - want[:, None]
    assert bool(((lp - lpw).abs() <= LSE + 2 * E * (lpw.abs() + want.abs()[:, None])).all())


@pytest.mark.parametrize("what", ["equal", "two values", "rising", "zeros of both signs", "masked",
                                  "all masked", "nan", "all nan", "+inf", "few finite"])
@pytest.mark.parametrize("vocab, k", [(900, 200), (40000, 64), (40000, 256)])
def test_topk_order(what, vocab, k):
    """Equal values, infinities and NaN: the order is the documented one, to the index."""
    z = torch.randn(4, vocab, generator=torch.Generator().manual_seed(1))
    if what == "equal":
        z[:] = 0.25
    elif what == "two values":
        z = (z > 1).float()
    elif what == "rising":
        z = torch.arange(vocab).float()[None].expand(4, -1).clone()
        z[1] = -z[1]
        z[2] = z[2] // 300
    elif what == "zeros of both signs":
        z = torch.where(z > 0, 0.0, -0.0)
    elif what == "masked":
        z[:, vocab // 3:] = -math.inf
    elif what == "all masked":
        z[1:3] = -math.inf
    elif what == "nan":
        z[0, 5], z[1, vocab - 1], z[1, 3], z[2, ::7] = math.nan, math.nan, -math.nan, math.nan
    elif what == "all nan":
        z[1] = math.nan
    elif what == "+inf":
        z[0, 9], z[2, ::5] = math.inf, math.inf
    elif what == "few finite":
        z[:] = -math.inf
        z[:, 17], z[:, vocab - 2] = 1.0, torch.finfo(torch.float32).min
    idx, lp, lse = topk(z, z.cuda(), k)
    at = place(z)[:, :k]
    assert torch.equal(idx.long(), at)
    want = torch.logsumexp(z.double(), 1)
    want = torch.where((z == math.inf).any(1), math.nan, want)      # documented: a row's lse is NaN
    bad = torch.isnan(want)
    assert torch.equal(torch.isnan(lse), bad)
    lpw = torch.where(want[:, None] == -math.inf, -math.inf, z.double().gather(1, at) - want[:, None])
    assert torch.equal(torch.isnan(lp), torch.isnan(lpw))
    fin = torch.isfinite(lpw)
    assert torch.equal(lp[~fin & ~torch.isnan(lpw)].double(), lpw[~fin & ~torch.isnan(lpw)])
    assert bool(((lp - lpw).abs()[fin] <= LSE + 3 * E * (lpw.abs() + want.abs()[:, None])[fin]).all())


def test_topk_workspace_serves_fewer_rows():
    from paper_2606_04484_amd import capi
    for vocab in (700, 20001, 151936):
        sizes = [capi.aj_topk_workspace_bytes(r, vocab, 64) for r in range(1, 700)]
        assert sizes == sorted(sizes)
        sizes = [capi.aj_distill_workspace_bytes(r, vocab, 64) for r in range(1, 3000)]
        assert sizes == sorted(sizes)
    z, view = make(13, 20001, "f32", 0)
    assert torch.equal(topk(z, view, 64, rows_ws=14)[0].long(), place(z)[:, :64])


# ------------------------------------------------------------------ distillation

def lists(z, k, seed, temp):
    """A teacher near the student: top of the logits with noise; some rows list less."""
    g = torch.Generator().manual_seed(seed + 1)
    t = z.float() / temp + torch.randn(z.shape, generator=g)
    top, at = torch.topk(t, k, dim=1)
    lp = top - torch.logsumexp(t, 1, keepdim=True)
    idx = at.to(torch.int32)
    if z.shape[0] > 1:
        idx[1::4, (k + 1) // 2:] = -1
    if z.shape[0] > 2:
        idx[2] = -5                              # nothing listed
    if k > 2:
        lp[0, k // 2] = -math.inf                # listed with probability 0
    return idx, lp


def definition(z, inv_temp, idx, lp, tail, w):
    """loss, lse [2], d logits in 64 bits (duplicate and out-of-range entries already out)."""
    z = z.double() * inv_temp
    rows, vocab = z.shape
    p, named = torch.zeros_like(z), torch.zeros_like(z, dtype=torch.bool)
    r, c = (idx >= 0).nonzero(as_tuple=True)
    named[r, idx[r, c].long()] = True
    p[r, idx[r, c].long()] = lp[r, c].double().exp()
    total = p.sum(1)
    rest = (1 - total).clamp(min=0) if tail else torch.zeros(rows, dtype=torch.float64)
    if not tail:
        p = torch.where(total[:, None] > 0, p / total[:, None], 0.0)
    lse = torch.logsumexp(z, 1)
    others = torch.logsumexp(z.masked_fill(named, -math.inf), 1)
    logq = z - lse[:, None]
    loss = torch.where(p > 0, p * (p.log() - logq), 0.0).sum(1)
    loss = loss + torch.where(rest > 0, rest * (rest.log() - (others - lse)), 0.0)
    share = torch.where(named, 0.0, (z - others[:, None]).exp()) * rest[:, None]
    full = p + torch.where(rest[:, None] > 0, share, 0.0)
    M = full.sum(1, keepdim=True) if not tail else (p.sum(1) + rest)[:, None]
    dz = (M * logq.exp() - full) * (w * inv_temp)[:, None]
    size = (M * logq.exp() + full) * (w * inv_temp).abs()[:, None]
    return loss, torch.stack([lse, others]), dz, size


def distill(view, inv_temp, idx, lp, tail, weight, coef, grad, part="step", inplace=False):
    from paper_2606_04484_amd import capi
    rows, vocab = view.shape
    dev = "cuda"
    t = capi.teacher(idx.to(dev), lp.to(dev), tail=tail, weight=None if weight is None else weight.to(dev),
                     coef=coef)
    loss, lse = torch.full((rows,), 9.0, device=dev), torch.full((2, rows), 9.0, device=dev)
    stats, err = torch.ones(2, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
    ws = torch.full((capi.aj_distill_workspace_bytes(rows, vocab, idx.shape[1]),), 255, dtype=torch.uint8,
                    device=dev)
    dz = view if inplace else torch.full((rows, vocab), 9.0, dtype=DT[grad], device=dev)
    if part == "step":
        capi.aj_distill_loss_fwd_bwd(view, inv_temp, t, loss, lse, dz, ws, stats=stats, err=err)
    else:
        capi.aj_distill_loss_fwd(view, inv_temp, t, loss, lse, ws, stats=stats, err=err)
        capi.aj_distill_loss_bwd(view, inv_temp, t, lse, dz)
    torch.cuda.synchronize()
    return loss.cpu(), lse.cpu(), dz.cpu(), stats.cpu(), int(err.item())


def check_distill(got, want, grad, inv_temp):
    (loss, lse, dz, _, _), (lw, sw, dw, size) = got, want
    fin = torch.isfinite(sw)
    assert torch.equal(lse[~fin].double(), sw[~fin])
    assert bool(((lse - sw).abs()[fin] <= LSE + 2 * E * sw.abs()[fin]).all())
    # infinite where the teacher has mass outside the list and the student none (the whole
    # vocabulary listed): then it has to be infinite
    off = torch.where(loss.double() == lw, 0.0, loss - lw).abs()
    assert bool((off <= 3 * LSE + 8 * E * (sw[0].abs() + lw.abs())).all()), off.max()
    # q is off by the log-sum-exp's error and 6 roundings of the exponent's terms
    rel = LSE + 6 * E * (sw[0].abs()[:, None] + 40)
    u = 2.0 ** -8 if grad == "bf16" else E
    err = (dz.double() - dw).abs()
    assert bool((err <= rel * size * 1.01 + u * (dw.abs() + rel * size) + 1e-37).all()), (err / (size + 1e-30)).max()


DISTILL = [(1, 1, 1, 0, 0), (1, 7, 7, 0, 0), (4, 40, 40, 1, 0), (5, 1024, 8, 0, 0), (9, 2003, 256, 5, 3),
           (3, 4099, 33, 0, 1), (1, 151936, 64, 0, 0), (6, 70001, 100, 3, 2), (40, 66000, 20, 0, 0)]


@pytest.mark.parametrize("tail", [False, True], ids=["listed", "tail"])
@pytest.mark.parametrize("dtype, grad", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("rows, vocab, k, pad, offset", DISTILL)
def test_distill(rows, vocab, k, pad, offset, dtype, grad, tail):
    z, view = make(rows, vocab, dtype, pad, seed=rows, offset=offset)
    inv = float(torch.tensor(1 / 1.3, dtype=torch.float32))
    idx, lp = lists(z, k, rows, 1.3)
    w = torch.rand(rows, generator=torch.Generator().manual_seed(3)) + 0.5
    coef = 0.25
    want = definition(z, inv, idx, lp, tail, w.double() * coef)
    got = distill(view, inv, idx, lp, tail, w, coef, grad)
    assert got[4] == 0
    check_distill(got, want, grad, inv)
    total = (want[0] * w.double() * coef).sum().item()
    assert got[3][0].item() == total or abs(got[3][0].item() - 1 - total) <= rows * 3 * LSE + 4 * E * (1 + abs(total)) * 2
    assert got[3][1].item() == 1 + rows
    apart = distill(view, inv, idx, lp, tail, w, coef, grad, part="apart")
    check_distill(apart, want, grad, inv)
    again = distill(view, inv, idx, lp, tail, w, coef, grad)
    for a, b, c in zip(got, apart, again):
        assert a == c if isinstance(a, int) else torch.equal(a, c)
        if vocab > 12280:     # few long rows: the same kernels (short ones sum in another order)
            assert a == b if isinstance(a, int) else torch.equal(a, b)


@pytest.mark.parametrize("tail", [False, True], ids=["listed", "tail"])
@pytest.mark.parametrize("dtype, grad", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("vocab, k, pad, offset", [(32768, 20, 0, 0), (40001, 256, 3, 1), (100003, 7, 0, 2),
                                                   (152064, 64, 0, 0)])
def test_many_long_rows(vocab, k, pad, offset, dtype, grad, tail):
    """Enough rows for a workgroup each: values kept on the chip, or read again, or both."""
    rows = 515
    z, view = make(rows, vocab, dtype, pad, seed=9, offset=offset)
    some = torch.cat([torch.arange(4), torch.arange(rows - 3, rows)])
    idx, lp = lists(z[some], k, 9, 1.0)
    idx = idx[torch.arange(rows) % 4].clone()
    lp = lp[torch.arange(rows) % 4].clone()
    idx[some], lp[some] = lists(z[some], k, 9, 1.0)
    w = torch.rand(rows, generator=torch.Generator().manual_seed(3)) + 0.5
    got = distill(view, 1.0, idx, lp, tail, w, 1.0, grad)
    want = definition(z[some], 1.0, idx[some], lp[some], tail, w[some].double())
    check_distill((got[0][some], got[1][:, some], got[2][some], None, None), want, grad, 1.0)
    apart = distill(view, 1.0, idx, lp, tail, w, 1.0, grad, part="apart")
    assert bool(((got[0] - apart[0]).abs() <= 3 * LSE + 8 * E * (apart[1][0].abs() + apart[0].abs())).all())
    u = 2.0 ** -7 if grad == "bf16" else 0.0
    # each is off by its q's error, and a named token's gradient w (M q - p) may be far
    # smaller than w q <= |gradient| + w p
    p = lp.double().exp() if tail else torch.softmax(torch.where(idx >= 0, lp, -math.inf).double(), 1).nan_to_num()
    at = torch.where(idx >= 0, idx, idx[:, :1].clamp(min=0)).long()
    size = apart[2].double().abs()
    size.scatter_add_(1, at, torch.where(idx >= 0, p, 0.0) * w[:, None].double() * 2)
    off = (got[2].double() - apart[2].double()).abs()
    assert bool((off <= u * apart[2].double().abs() + (2 * LSE + 300 * E) * size + 1e-37).all())
    if dtype == grad:
        assert torch.equal(distill(view, 1.0, idx, lp, tail, w, 1.0, grad, inplace=True)[2], got[2])


@pytest.mark.parametrize("part", ["step", "apart"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_in_the_logits_place(dtype, part):
    """d logits over the logits, whose rows lie apart: what is between them stays."""
    z, view = make(5, 9001, dtype, 7, seed=2, offset=3)
    idx, lp = lists(z, 50, 2, 1.0)
    want = distill(view, 1.0, idx, lp, True, None, 1.0, dtype, part=part)   # (the same calls)
    got = distill(view, 1.0, idx, lp, True, None, 1.0, dtype, part=part, inplace=True)
    assert torch.equal(got[2], want[2]) and torch.equal(got[0], want[0])
    rest = torch.as_strided(view, (4, 7), (9008, 1), view.storage_offset() + 9001)
    assert bool(torch.isnan(rest).all())


@pytest.mark.parametrize("tail", [False, True], ids=["listed", "tail"])
def test_repeated_and_foreign_entries(tail):
    """A token listed again, one past the vocabulary: reported, and as if not listed."""
    z, view = make(6, 3000, "f32", 0, seed=4)
    idx, lp = lists(z, 30, 4, 1.0)
    clean = idx.clone()
    bad = idx.clone()
    bad[0, 20] = bad[0, 3]
    clean[0, 20] = -1
    bad[3, 29], bad[3, 11] = bad[3, 0], bad[3, 0]
    clean[3, 29] = clean[3, 11] = -1
    a, b = (distill(view, 1.0, i, lp, tail, None, 1.0, "f32") for i in (clean, bad))
    assert a[4] == 0 and b[4] == 32
    assert all(torch.equal(x, y) for x, y in zip(a[:4], b[:4]))
    for v in (3000, 2 ** 31 - 1):
        far, none = clean.clone(), clean.clone()
        far[4, 2], none[4, 2] = v, -1
        a, b = (distill(view, 1.0, i, lp, tail, None, 1.0, "f32") for i in (none, far))
        assert b[4] == 1 and all(torch.equal(x, y) for x, y in zip(a[:4], b[:4]))


@pytest.mark.parametrize("tail", [False, True], ids=["listed", "tail"])
def test_masked_vocabulary_and_bad_rows(tail):
    """Logits of -inf outside the list take no gradient; a NaN or +inf stays in its row; the whole
    vocabulary listed leaves no others."""
    z = torch.randn(5, 5000, generator=torch.Generator().manual_seed(6))
    idx, lp = lists(z[:, :4000], 20, 6, 1.0)
    clean = z.clone()
    clean[:, 4000:] = -math.inf
    got = distill(clean.cuda(), 1.0, idx, lp, tail, None, 1.0, "f32")
    check_distill(got, definition(clean, 1.0, idx, lp, tail, torch.ones(5).double()), "f32", 1.0)
    assert bool((got[2][:, 4000:] == 0).all())
    bad = clean.clone()
    bad[1, 77], bad[3, 4999] = math.nan, math.inf
    worse = distill(bad.cuda(), 1.0, idx, lp, tail, None, 1.0, "f32")
    for r in range(5):
        same = r not in (1, 3)
        assert torch.equal(worse[2][r], got[2][r]) == same
        assert bool(torch.isnan(worse[0][r])) != same
    z = torch.randn(2, 40, generator=torch.Generator().manual_seed(7))
    lp = torch.log_softmax(torch.randn(2, 40, generator=torch.Generator().manual_seed(8)), 1)
    idx = torch.arange(40, dtype=torch.int32).flip(0).expand(2, -1).contiguous()
    got = distill(z.cuda(), 1.0, idx, lp, tail, None, 1.0, "f32")
    assert bool((got[1][1] == -math.inf).all()) and bool(torch.isfinite(got[2]).all())
    want = definition(z, 1.0, idx, lp, False, torch.ones(2).double())
    # with a tail the rounding of the given log-probs leaves 1 - sum p near 40 * 2^-24
    assert bool(((got[2] - want[2]).abs() <= 1e-5).all())


@pytest.mark.parametrize("tail", [False, True], ids=["listed", "tail"])
def test_gradient_against_differences(tail):
    z = torch.randn(3, 500, generator=torch.Generator().manual_seed(1))
    idx, lp = lists(z, 12, 1, 1.0)
    one = torch.ones(3).double()
    d = torch.randn(z.shape, generator=torch.Generator().manual_seed(2)).double()
    h = 1e-5
    f = [definition(z.double() + t * d, 0.5, idx, lp, tail, one)[0] for t in (h, -h)]
    want = (f[0] - f[1]) / (2 * h)
    got = distill(z.cuda(), 0.5, idx, lp, tail, None, 1.0, "f32")[2]
    have = (got.double() * d).sum(1)
    size = definition(z, 0.5, idx, lp, tail, one)[3]
    assert bool(((have - want).abs() <= ((LSE + 300 * E) * size * d.abs()).sum(1) + 1e-8).all())


def test_large_offsets():
    """Rows past 2^32 bytes, and past 2^31 elements, of one matrix."""
    rows, vocab = 8, 1000
    buf = torch.empty(7 * 340_000_000 + vocab, dtype=torch.bfloat16, device="cuda")
    view = torch.as_strided(buf, (rows, vocab), (340_000_000, 1))
    z = torch.randn(rows, vocab, generator=torch.Generator().manual_seed(1)).bfloat16()
    view.copy_(z)
    idx, lp, lse = topk(z, view, 10)
    assert torch.equal(idx.long(), place(z)[:, :10])
    ti, tl = lists(z, 10, 1, 1.0)
    got = distill(view, 1.0, ti, tl, True, None, 1.0, "bf16", inplace=True)
    check_distill(got, definition(z, 1.0, ti, tl, True, torch.ones(rows).double()), "bf16", 1.0)


def test_captured_replayed_and_other_stream():
    from paper_2606_04484_amd import capi
    rows, vocab, k = 9, 20000, 16
    z = torch.randn(rows, vocab, device="cuda")
    idx = torch.empty(rows, k, dtype=torch.int32, device="cuda")
    lp, lse1 = torch.empty(rows, k, device="cuda"), torch.empty(rows, device="cuda")
    loss, lse = torch.empty(rows, device="cuda"), torch.empty(2, rows, device="cuda")
    stats, dz = torch.zeros(2, device="cuda"), torch.empty_like(z)
    ws = torch.empty(max(capi.aj_topk_workspace_bytes(rows, vocab, k),
                         capi.aj_distill_workspace_bytes(rows, vocab, k)), dtype=torch.uint8, device="cuda")
    student = torch.randn(rows, vocab, device="cuda")
    t = capi.teacher(idx, lp, tail=True)

    def run():
        capi.aj_topk_logprob(z, 1.0, idx, lp, lse1, ws)
        capi.aj_distill_loss_fwd_bwd(student, 1.0, t, loss, lse, dz, ws, stats=stats)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        z.copy_(torch.randn(rows, vocab, device="cuda"))
        stats.zero_()
        run()
        torch.cuda.synchronize()
        want = [a.clone() for a in (idx, lp, loss, lse, dz, stats)]
        stats.zero_(), dz.zero_(), loss.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((idx, lp, loss, lse, dz, stats), want):
            assert torch.equal(a, b), i
