"""Counts of rows at which a thread, or a wave, for each would be more than one launch takes
(2^32 threads): the same results as of a few of these rows."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, hq, hkv, hd, window, length", [
    (torch.float32, 64, 1, 8, 5, 32), (torch.bfloat16, 64, 1, 64, 0, 512), (torch.float32, 32, 1, 8, 20, 1024)])
def test_attention(dtype, hq, hkv, hd, window, length):
    """2^26 rows and more, counted with their heads (window 0: by the kernels of long segments)."""
    from paper_2606_04484_amd import capi
    n_seg = -(-((1 << 26) // hq + 3 * length) // length)
    n, dev = n_seg * length, "cuda"
    cfg = capi.attn_cfg(hq, hkv, hd, window=window, n_sink=2, dtype=dtype)
    g = torch.Generator(device=dev).manual_seed(1)
    width = (hq + 2 * hkv) * hd
    qkv = torch.randn(n, width, generator=g, device=dev, dtype=torch.float32 if hd == 8 else dtype).to(dtype)
    dout = torch.randn(n, hq * hd, generator=g, device=dev, dtype=torch.float32 if hd == 8 else dtype).to(dtype)

    def run(a, b):
        m = b - a
        cu = torch.arange(0, m + 1, length, dtype=torch.int32, device=dev)
        ws = torch.full((capi.aj_attention_workspace_bytes(cfg, m),), 255, dtype=torch.uint8, device=dev)
        out, lse = torch.empty(m, hq * hd, dtype=dtype, device=dev), torch.empty(hq, m, device=dev)
        dqkv = torch.full((m, width), float("nan"), dtype=dtype, device=dev)
        capi.aj_attention_fwd(cfg, cu, length, qkv[a:b], out, lse, ws)
        capi.aj_attention_bwd(cfg, cu, length, qkv[a:b], out, lse, dout[a:b], dqkv, ws)
        torch.cuda.synchronize()
        return out, lse, dqkv

    whole = run(0, n)
    for a in (0, n - 2 * length):
        part = run(a, a + 2 * length)
        assert torch.equal(whole[0][a:a + 2 * length], part[0])
        assert torch.equal(whole[1][:, a:a + 2 * length], part[1])
        x, y = whole[2][a:a + 2 * length].float(), part[2].float()
        # (the parts that a long pack's dK, dV are summed in may differ from a short one's)
        assert bool(torch.isfinite(x).all()) and bool(((x - y).norm() <= 1e-2 * y.norm()))


def test_rows_of_logits():
    from paper_2606_04484_amd import capi
    rows, dev = (1 << 24) - 1, "cuda"
    z = torch.randn(rows, 2, device=dev)
    idx, lp = torch.full((rows, 2), -1, dtype=torch.int32, device=dev), torch.zeros(rows, 2, device=dev)
    lse, ws = torch.zeros(rows, device=dev), torch.empty(capi.aj_topk_workspace_bytes(rows, 2, 2), dtype=torch.uint8,
                                                         device=dev)
    capi.aj_topk_logprob(z, 1.0, idx, lp, lse, ws)
    # two float32 terms, their exponents' and their sum's roundings: 3e-7; the result's, below 16: 4.8e-7
    want = torch.log_softmax(z.double(), 1)
    top, at = want.sort(dim=1, descending=True, stable=True)
    assert torch.equal(idx.long(), at) and bool(((lp - top).abs() <= 1e-6).all())
    loss, both, dz = torch.full((rows,), 9.0, device=dev), torch.zeros(2, rows, device=dev), torch.full_like(z, 9.0)
    ws = torch.empty(capi.aj_distill_workspace_bytes(rows, 2, 2), dtype=torch.uint8, device=dev)
    teacher = torch.log_softmax(torch.randn(rows, 2, device=dev), 1)
    t = capi.teacher(torch.tensor([[0, 1]], dtype=torch.int32, device=dev).expand(rows, 2).contiguous(), teacher)
    p = torch.softmax(teacher.double(), 1)
    kl = (p * (p.log() - want)).sum(1)
    for step in (True, False):
        if step:
            capi.aj_distill_loss_fwd_bwd(z, 1.0, t, loss, both, dz, ws)
        else:
            loss.fill_(9.0), dz.fill_(9.0)
            capi.aj_distill_loss_fwd(z, 1.0, t, loss, both, ws)
            capi.aj_distill_loss_bwd(z, 1.0, t, both, dz)
        torch.cuda.synchronize()
        assert bool(((loss - kl).abs() <= 2e-6).all())
        assert bool(((dz - (want.exp() - p)).abs() <= 2e-6).all())
