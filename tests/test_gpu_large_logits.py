"""Logits of the largest magnitudes that their type holds, finite ones: rows masked with the
lowest value, rows a long way from zero, low temperatures.  Top k and distillation against the
definition in 64 bits, every log-sum-exp relative to its largest value."""
import math

import pytest
import torch

from test_gpu_distill import DT, E, LSE, distill, lists, make, place, topk

pytestmark = pytest.mark.gpu
MAX = torch.finfo(torch.float32).max


def log_sum(z, inv, see):
    """(unit, log) of every row's log sum exp(z inv) over `see`; apart, as unit + log may be unit."""
    m = z.masked_fill(~see, -math.inf).amax(1)
    m = torch.where(m == -math.inf, 0.0, m)
    return m * inv, torch.where(see, ((z - m[:, None]) * inv).exp(), 0.0).sum(1).log()


def as_result(unit, log):
    return torch.where(log == -math.inf, -math.inf, (unit + log).clamp(-MAX, MAX))


def rows_of(what, rows, vocab, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, vocab, generator=g) * 2.5
    low, high = torch.finfo(DT[dtype]).min, torch.finfo(DT[dtype]).max
    if what == "lowest":
        z[:] = low
    elif what == "highest":
        z[:] = high
    elif what == "both ends":
        z = torch.where(z > 0, high, low)
    elif what == "mixed rows":        # the unit of a row is not its neighbour's
        z[::3] = low
        z[1::3, vocab // 2:] = low
    elif what == "far":
        z = z * 30 + 3e6
    elif what == "far below":
        z = z * 1e5 - 1e9
    return z.to(DT[dtype])


WHAT = ["lowest", "highest", "both ends", "mixed rows", "far", "far below"]


@pytest.mark.parametrize("inv_temp", [1.0, 1 / 0.7, 1e4, 1e30])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", WHAT)
@pytest.mark.parametrize("rows, vocab, k", [(4, 3000, 64), (1, 40001, 256), (1030, 9001, 20)])
def test_topk(rows, vocab, k, what, dtype, inv_temp):
    few = min(rows, 7)
    z = rows_of(what, few, vocab, dtype)
    at = torch.arange(rows) % few
    idx, lp, lse = topk(z[at], z[at].cuda(), k, inv_temp)
    inv = torch.tensor(inv_temp, dtype=torch.float32).double()
    order = place(z)[:, :k]
    assert torch.equal(idx.long(), order[at])
    d = z.double()
    unit, log = log_sum(d, inv, torch.ones_like(d, dtype=torch.bool))
    want = as_result(unit, log)[at]
    assert bool(((lse - want).abs() <= LSE + 2 * E * want.abs()).all())
    lpw = ((d.gather(1, order) * inv - unit[:, None]) - log[:, None])[at]
    # what is below float32's range is -inf as a log-prob (its lse is the lowest value)
    out = lpw < -MAX
    assert bool((lp[out] <= -MAX).all())
    assert bool(((lp - lpw).abs()[~out] <= LSE + 3 * E * lpw.abs()[~out]).all())


def definition(z, inv, idx, lp, tail, w):
    z = z.double()
    named = torch.zeros_like(z, dtype=torch.bool)
    p = torch.zeros_like(z)
    r, c = (idx >= 0).nonzero(as_tuple=True)
    named[r, idx[r, c].long()] = True
    p[r, idx[r, c].long()] = lp[r, c].double().exp()
    total = p.sum(1)
    rest = (1 - total).clamp(min=0) if tail else torch.zeros_like(total)
    if not tail:
        p = torch.where(total[:, None] > 0, p / total[:, None], 0.0)
    unit, log = log_sum(z, inv, torch.ones_like(named))
    runit, rlog = log_sum(z, inv, ~named)
    logq = (z * inv - unit[:, None]) - log[:, None]
    loss = torch.where(p > 0, p * (p.log() - logq), 0.0).sum(1)
    ratio = (runit - unit) + (rlog - log)
    loss = loss + torch.where(rest > 0, rest * (rest.log() - ratio), 0.0)
    share = torch.where(named, 0.0, ((z * inv - runit[:, None]) - rlog[:, None]).exp()) * rest[:, None]
    full = p + torch.where(rest[:, None] > 0, share, 0.0)
    M = (p.sum(1) + rest)[:, None]
    at = (w * inv)[:, None]
    return loss, torch.stack([as_result(unit, log), as_result(runit, rlog)]), (M * logq.exp() - full) * at, \
        (M * logq.exp() + full) * at


def check(got, want, grad):
    (loss, lse, dz), (lw, sw, dw, size) = got[:3], want
    none = sw == -math.inf
    assert torch.equal(lse == -math.inf, none)
    assert bool(((lse - sw).abs()[~none] <= LSE + 2 * E * sw.abs()[~none]).all())
    big = lw.abs() > MAX * (1 - 2 * E)          # the loss's own range
    assert bool((loss[big].abs() >= MAX * (1 - 4 * E)).all())
    assert bool(((loss - lw).abs()[~big] <= 3 * LSE + 8 * E * (1 + lw.abs()[~big])).all())
    # q is off by the log-sum-exp's error and 6 roundings of its exponent's terms, which are
    # distances from a unit and not the logits; below 16384 the gradient by itself may go by a
    # log-sum-exp in float32
    near = torch.where(sw.abs() < 16384, sw.abs(), 0.0).nan_to_num(0.0, 0.0, 0.0).amax(0)[:, None]
    rel = LSE + 6 * E * (near + 40)
    u = 2.0 ** -8 if grad == "bf16" else E
    err = (dz.double() - dw).abs()
    assert bool((err <= rel * size * 1.01 + u * (dw.abs() + rel * size) + 1e-37).all())


@pytest.mark.parametrize("tail", [False, True], ids=["listed", "tail"])
@pytest.mark.parametrize("part", ["step", "apart", "step in place", "apart in place"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", WHAT + ["listed alone", "unlisted alone"])
@pytest.mark.parametrize("rows, vocab, k, pad, offset", [(5, 2003, 20, 0, 1), (6, 70001, 100, 3, 0),
                                                        (515, 75001, 33, 0, 2)])
def test_distill(rows, vocab, k, pad, offset, what, dtype, part, tail):
    few = min(rows, 9)
    z = rows_of(what, few, vocab, dtype, seed=rows)
    idx, lp = lists(torch.randn(few, vocab, generator=torch.Generator().manual_seed(7)), k, rows, 1.0)
    if what in ("listed alone", "unlisted alone"):
        low = torch.finfo(DT[dtype]).min
        named = torch.zeros_like(z, dtype=torch.bool)
        r, c = (idx >= 0).nonzero(as_tuple=True)
        named[r, idx[r, c].long()] = True
        z[named != (what == "listed alone")] = low
    at = torch.arange(rows) % few
    _, view = make(rows, vocab, dtype, pad, offset=offset)
    view.copy_(z[at])
    inv = 1.0
    w = torch.rand(few, generator=torch.Generator().manual_seed(3)) + 0.5
    got = distill(view, inv, idx[at], lp[at], tail, w[at], 1.0, dtype, part=part.split()[0],
                  inplace="place" in part)
    assert got[4] == 0
    want = definition(z, inv, idx, lp, tail, w.double())
    for a in range(0, rows, few):
        n = min(few, rows - a)
        check((got[0][a:a + n], got[1][:, a:a + n], got[2][a:a + n]), [t[..., :n] if t.dim() == 1 or i == 1 else t[:n]
                                                                     for i, t in enumerate(want)], dtype)


@pytest.mark.parametrize("inv_temp", [1 / 0.7, 50.0])
@pytest.mark.parametrize("part", ["step", "apart"])
def test_lowest_values_at_a_low_temperature(part, inv_temp):
    """The product with the temperature leaves float32's range, the log-sum-exp is the lowest value."""
    z = rows_of("mixed rows", 9, 5000, "f32")
    idx, lp = lists(torch.randn(9, 5000, generator=torch.Generator().manual_seed(7)), 20, 3, 1.0)
    inv = float(torch.tensor(inv_temp, dtype=torch.float32))
    got = distill(z.cuda(), inv, idx, lp, True, None, 1.0, "f32", part=part)
    check(got, definition(z, inv, idx, lp, True, torch.ones(9).double()), "f32")


@pytest.mark.parametrize("inv_temp", [1e-30, 1e-38, 1e-44])
@pytest.mark.parametrize("what", ["random", "both ends"])
@pytest.mark.parametrize("part", ["step", "apart"])
def test_temperatures_at_which_all_tokens_are_alike(part, what, inv_temp):
    z = rows_of(what, 7, 4000, "f32")
    inv = float(torch.tensor(inv_temp, dtype=torch.float32))
    at = place(z)[:, :20]
    idx, lp, lse = topk(z, z.cuda(), 20, inv)
    unit, log = log_sum(z.double(), inv, torch.ones_like(z, dtype=torch.bool))
    assert torch.equal(idx.long(), at) and bool(((lse - unit - log).abs() <= LSE + 2 * E * lse.abs()).all())
    lpw = (z.double().gather(1, at) * inv - unit[:, None]) - log[:, None]
    assert bool(((lp - lpw).abs() <= LSE + 3 * E * lpw.abs()).all())
    ti, tl = lists(torch.randn(7, 4000, generator=torch.Generator().manual_seed(7)), 20, 3, 1.0)
    one = torch.ones(7).double()
    got = distill(z.cuda(), inv, ti, tl, True, None, 1.0 / inv if inv > 1e-37 else 1e30, "f32", part=part)
    want = definition(z, inv, ti, tl, True, one * (float(torch.tensor(1.0 / inv)) if inv > 1e-37 else
                                                   float(torch.tensor(1e30))))
    check(got, want, "f32")
