"""The teacher's lists and the distillation loss at the LM head, called directly: more targets
than one slab of logits holds, against the definition in 64 bits; what is reported."""
import math

import pytest
import torch

from test_gpu_distill import E, LSE, definition, lists

pytestmark = pytest.mark.gpu

D, V, BASE = 64, 72, 1000


def setup(n_tok, n_tgt, dtype, seed=0):
    from paper_2606_04484_amd import capi
    g = torch.Generator().manual_seed(seed)
    h = (torch.randn(n_tok, D, generator=g) * 2).to(dtype)
    gamma = (1 + 0.3 * torch.randn(D, generator=g)).to(dtype)
    w = (torch.randn(V, D, generator=g) * 0.4).to(dtype)
    rows = torch.randperm(n_tok, generator=g)[:n_tgt].sort().values
    cfg = capi.LossCfg(D, V, 1 << 14, 0.2, 1e-6, capi.AJ_BF16 if dtype == torch.bfloat16 else capi.AJ_F32, 0)
    return cfg, h, gamma, w, rows, (rows + 1 + BASE).to(torch.int32)


def step(cfg, h, gamma, w, targets, idx, lp, tail, frozen=False):
    from paper_2606_04484_amd import capi
    n, k = idx.shape
    z = lambda *s: torch.zeros(*s, device="cuda")  # noqa: E731
    t = capi.teacher(idx.cuda(), lp.cuda(), tail=tail)
    ws = torch.full((capi.aj_lm_head_workspace_bytes(cfg, n, k),), 255, dtype=torch.uint8, device="cuda")
    loss, dh, dg, dw = z(n), z(*h.shape).fill_(7.0), z(D), z(V, D)
    stats, err = z(2), torch.zeros(1, dtype=torch.int32, device="cuda")
    capi.aj_lm_head_distill(cfg, targets.cuda(), h.cuda(), gamma.cuda(), w.cuda(), 1.0, t, loss, dh,
                            None if frozen else dg, None if frozen else dw, ws, row_base=BASE, stats=stats,
                            err=err)
    torch.cuda.synchronize()
    return [x.cpu() for x in (loss, dh, dg, dw, stats)] + [int(err.item())]


@pytest.mark.parametrize("tail", [False, True], ids=["listed", "tail"])
@pytest.mark.parametrize("n_tok, n_tgt", [(1, 1), (90, 40), (8600, 8400)])
def test_loss_and_backward(n_tok, n_tgt, tail):
    cfg, h, gamma, w, rows, targets = setup(n_tok, n_tgt, torch.float32)
    x, g, W = h.double()[rows], gamma.double(), w.double()
    r = (x.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    hn = x * r * g
    z = hn @ W.T
    idx, lp = lists(z.float(), 9, 3, 1.0)
    loss, sw, dz, size = definition(z, 1.0, idx, lp, tail, torch.ones(n_tgt))
    got = step(cfg, h, gamma, w, targets, idx, lp, tail)
    assert got[5] == 0
    # a normalised row is off by a relatively (half a sum of D squares, and its factors), a
    # logit by b at most; a probability then by 2 b and a little, beyond what the loss's own
    # arithmetic allows for exact logits
    a = E * (D / 2 + 8)
    b = ((a + E * (D + 4)) * (hn.abs() @ W.abs().T)).amax(1, keepdim=True)
    assert bool(((got[0] - loss).abs() <= 2.1 * b[:, 0] + 3 * LSE + 8 * E * (sw[0].abs() + loss.abs())).all())
    assert abs(got[4][0] - loss.sum()) <= (2.1 * b.sum() + n_tgt * 3 * LSE + (n_tgt + 8) * E * loss.abs().sum()
                                           + 8 * E * (sw[0].abs() + loss.abs()).sum())
    assert got[4][1] == n_tgt
    ddz = (4.2 * b + LSE + 6 * E * (sw[0].abs()[:, None] + 40)) * size * 1.01 + E * dz.abs() + 1e-37
    top = dz.abs() + ddz
    dhn, ddhn = dz @ W, ddz @ W.abs() + E * (V + 8) * top @ W.abs()
    dw, ddw = dz.T @ hn, ddz.T @ hn.abs() + (a + E * (n_tgt + 8)) * top.T @ hn.abs()
    assert bool(((got[3] - dw).abs() <= ddw + E * dw.abs()).all())
    back = lambda v, s: r * v + s * x.abs() * r ** 3 / D * (v * x.abs()).sum(1, keepdim=True)  # noqa: E731
    dx = r * g * dhn - x * r ** 3 / D * (g * dhn * x).sum(1, keepdim=True)
    mag = g.abs() * (dhn.abs() + ddhn)
    ddx = back(g.abs() * ddhn, 1) + E * (3 * D + 40) * back(mag, 1)
    assert bool(((got[1][rows] - dx).abs() <= ddx).all())
    dg = (dhn * x * r).sum(0)
    ddg = (ddhn * x.abs() * r).sum(0) + E * (n_tgt + D + 24) * ((dhn.abs() + ddhn) * x.abs() * r).sum(0)
    assert bool(((got[2] - dg).abs() <= ddg).all())
    rest = torch.ones(n_tok, dtype=torch.bool)
    rest[rows] = False
    assert bool((got[1][rest] == 0).all())
    # frozen weights: the same loss and d hidden, nothing else written
    only = step(cfg, h, gamma, w, targets, idx, lp, tail, frozen=True)
    assert torch.equal(only[0], got[0]) and torch.equal(only[1], got[1]) and not only[2].any() and not only[3].any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_lists_beyond_a_slab(dtype):
    """The lists of all targets are those of any part of them; a target may be asked for twice."""
    from paper_2606_04484_amd import capi
    cfg, h, gamma, w, rows, targets = setup(8700, 8500, dtype, seed=1)
    k = 7

    def run(tg):
        n = tg.numel()
        idx, lp = torch.zeros(n, k, dtype=torch.int32, device="cuda"), torch.zeros(n, k, device="cuda")
        lse, err = torch.zeros(n, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        ws = torch.empty(capi.aj_lm_head_workspace_bytes(cfg, n, k), dtype=torch.uint8, device="cuda")
        capi.aj_lm_head_topk(cfg, tg.cuda(), h.cuda(), gamma.cuda(), w.cuda(), 1.0, idx, lp, lse, ws,
                             row_base=BASE, err=err)
        torch.cuda.synchronize()
        assert int(err.item()) == 0
        return idx.cpu(), lp.cpu(), lse.cpu()

    whole = run(targets)
    x = h.double()[rows]
    hn = x * (x.square().mean(1, keepdim=True) + 1e-6).rsqrt() * gamma.double()
    z, size = hn @ w.double().T, hn.abs() @ w.double().abs().T
    # a logit is off by the roundings of its normalised row (bfloat16: half a step of it) and of its sum
    b = ((2.0 ** -8 if dtype == torch.bfloat16 else 0.0) + E * (1.5 * D + 12)) * 1.01 * size.amax(1, keepdim=True)
    want = torch.logsumexp(z, 1, keepdim=True)
    assert bool(((whole[2][:, None] - want).abs() <= b + LSE + 2 * E * want.abs()).all())
    at = z.gather(1, whole[0].long())
    assert bool(((whole[1] - (at - want)).abs() <= 2 * b + LSE + 3 * E * (at.abs() + want.abs())).all())
    # a listed value is among the k largest to within two logits' errors
    assert bool((at >= torch.topk(z, k, dim=1).values[:, -1:] - 2 * b).all())
    twice = torch.cat([targets[8190:8195], targets[8190:8195].flip(0)])
    part = run(twice)
    pick = torch.cat([torch.arange(8190, 8195), torch.arange(8194, 8189, -1)])
    z_err = E * 2 * (D + 4) * size[pick].amax(1)       # another shape of product may add in another order
    assert bool(((part[2] - whole[2][pick]).abs() <= z_err + 2 * LSE + 4 * E * want[pick, 0].abs()).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_reported_targets(dtype):
    """A target twice, out of order, or outside the pack is reported; the others' losses stay."""
    cfg, h, gamma, w, rows, targets = setup(50, 20, dtype, seed=2)
    idx, lp = lists(torch.randn(20, V, generator=torch.Generator().manual_seed(5)), 5, 5, 1.0)
    want = step(cfg, h, gamma, w, targets, idx, lp, True)
    assert want[5] == 0
    for at, value in ((7, targets[6]), (7, targets[6] - 1), (19, BASE + 51), (0, BASE), (0, BASE - 5)):
        bad = targets.clone()
        bad[at] = value
        got = step(cfg, h, gamma, w, bad, idx, lp, True)
        keep = torch.arange(20) != at
        assert got[5] != 0 and torch.equal(got[0][keep], want[0][keep]), (at, int(value))
    assert math.isfinite(want[0].sum())


def test_operands_of_the_head():
    from paper_2606_04484_amd import capi
    cfg, h, gamma, w, rows, targets = setup(50, 20, torch.float32, seed=2)
    f = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")  # noqa: E731
    ws = f(capi.aj_lm_head_workspace_bytes(cfg, 20, 5), dt=torch.uint8)
    lists_ = f(20, 5, dt=torch.int32), f(20, 5)
    args = [targets.cuda(), h.cuda(), gamma.cuda(), w.cuda(), 1.0]
    t = capi.teacher(*lists_)
    for what, bad in (("err", f(1)), ("err", f(2, dt=torch.int32)), ("err", torch.zeros(1, dtype=torch.int32))):
        with pytest.raises(capi.AjError, match=what):
            capi.aj_lm_head_topk(cfg, *args, *lists_, f(20), ws, row_base=BASE, err=bad)
        with pytest.raises(capi.AjError, match=what):
            capi.aj_lm_head_distill(cfg, *args, t, f(20), f(50, D), None, None, ws, row_base=BASE, err=bad)
    with pytest.raises(capi.AjError, match="dh"):
        capi.aj_lm_head_distill(cfg, *args, t, f(20), f(49, D), None, None, ws, row_base=BASE)
    with pytest.raises(capi.AjError, match="weight"):
        capi.aj_lm_head_distill(cfg, *args, capi.teacher(*lists_, weight=f(19)), f(20), f(50, D), None, None, ws,
                                row_base=BASE)
