"""Top k where a workgroup walks a whole row (1024 rows and more) in many steps, with a threshold
that rises, lists that are cut on the way and values that do not fit them: the documented order to
the index, and the log-probs, as for few rows."""
import math

import pytest
import torch

from test_gpu_distill import DT, E, LSE, place, topk

pytestmark = pytest.mark.gpu
ROWS = 1030


def values(what, vocab, dtype):
    """A few distinct rows; all ROWS are these in turn."""
    z = torch.randn(7, vocab, generator=torch.Generator().manual_seed(vocab)) * 2.5
    if what == "equal":
        z[:] = 0.25
    elif what == "two values":
        z = (z > 3).float()
    elif what == "rising":
        z = torch.arange(vocab).float()[None].expand(7, -1).clone()
        z[1] = -z[1]
        z[2] = z[2] // 300
        z[3] = z[3] % 4096
        z[4] = (z[4] // 4096) + (z[4] % 2) * 100
    elif what == "late":                  # the largest ones in the last step
        z[:, -300:] += 50
    elif what == "zeros of both signs":
        z = torch.where(z > 0, 0.0, -0.0)
    elif what == "masked":
        z[:, vocab // 3:] = -math.inf
        z[3] = -math.inf
        z[4, :-5] = -math.inf
    elif what == "nan":
        z[0, 5], z[1, vocab - 1], z[1, 9000], z[2, ::7] = math.nan, math.nan, -math.nan, math.nan
        z[3] = math.nan
        z[4, 8192:] = math.nan
    elif what == "+inf":
        z[0, 9], z[2, ::5], z[3, -1] = math.inf, math.inf, math.inf
    elif what == "lowest":
        z[:, ::3] = torch.finfo(DT[dtype]).min
        z[2] = torch.finfo(DT[dtype]).min
    return z.to(DT[dtype])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", ["random", "equal", "two values", "rising", "late", "zeros of both signs", "masked",
                                  "nan", "+inf", "lowest"])
@pytest.mark.parametrize("vocab, k, pad, offset", [(40000, 1, 0, 0), (40000, 64, 3, 1), (40000, 256, 0, 0),
                                                   (20001, 256, 5, 7), (32768, 100, 0, 0)])
def test_order(vocab, k, pad, offset, what, dtype):
    z = values(what, vocab, dtype)
    at = torch.arange(ROWS) % len(z)
    buf = torch.full((offset + ROWS * (vocab + pad) + 8,), float("nan"), dtype=DT[dtype], device="cuda")
    view = buf[offset:offset + ROWS * (vocab + pad)].view(ROWS, vocab + pad)[:, :vocab]
    view.copy_(z.cuda()[at.cuda()])
    idx, lp, lse = topk(view, view, k)
    order = place(z)[:, :k]
    assert torch.equal(idx.long(), order[at])
    d = z.double()
    top = d.amax(1, keepdim=True)                    # (of NaN: NaN)
    unit = torch.where(torch.isinf(top), torch.where(top > 0, math.nan, 0.0), top)
    log = (d - unit).exp().sum(1, keepdim=True).log()
    want = (unit + log)[:, 0]
    bad = torch.isnan(want)[at]
    assert torch.equal(torch.isnan(lse), bad)
    want = want[at]
    same = lse.double() == want                      # -inf where it has to be
    assert bool((same | ((lse - want).abs() <= LSE + 2 * E * want.abs()))[~bad].all())
    lpw = torch.where(log == -math.inf, -math.inf, (d.gather(1, order) - unit) - log)[at]
    assert torch.equal(torch.isnan(lp), torch.isnan(lpw))
    fin = torch.isfinite(lpw)
    assert torch.equal(lp[~fin & ~torch.isnan(lpw)].double(), lpw[~fin & ~torch.isnan(lpw)])
    assert bool(((lp - lpw).abs()[fin] <= LSE + 3 * E * lpw.abs()[fin]).all())


def test_rows_at_the_change_from_parts_to_whole_rows():
    """1023 rows are cut into parts, 1024 are not: the same lists."""
    z = torch.randn(1024, 30011, generator=torch.Generator().manual_seed(3)).cuda()
    for dtype in (torch.float32, torch.bfloat16):
        x = z.to(dtype)
        a, b = topk(x, x, 200), topk(x[:1023], x[:1023], 200)
        assert torch.equal(a[0][:1023], b[0])
        assert bool(((a[1][:1023] - b[1]).abs() <= 2 * LSE + 4 * E * a[1][:1023].abs()).all())
        assert bool(((a[2][:1023] - b[2]).abs() <= 2 * LSE + 4 * E * a[2][:1023].abs()).all())
