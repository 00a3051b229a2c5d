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


def test_hidden_gradient_past_a_launch():
    """d h of 2^32 elements and more is cleared to its end."""
    from paper_2606_04484_amd import capi
    D, V, n, dev = 8192, 64, (1 << 19) + 3, "cuda"
    cfg = capi.LossCfg(D, V, 1 << 14, 0.2, 1e-6, capi.AJ_BF16, 0)
    h = torch.zeros(n, D, dtype=torch.bfloat16, device=dev)
    rows = torch.tensor([5, n - 1], device=dev)
    h[rows] = torch.randn(2, D, device=dev).bfloat16()
    w = (torch.randn(V, D, device=dev) * 0.02).bfloat16()
    gamma = torch.ones(D, dtype=torch.bfloat16, device=dev)
    t = capi.teacher(torch.tensor([[1, 7], [9, 2]], dtype=torch.int32, device=dev),
                     torch.tensor([[-1.0, -2.0], [-0.5, -3.0]], device=dev), tail=True)
    ws = torch.empty(capi.aj_lm_head_workspace_bytes(cfg, 2, 2), dtype=torch.uint8, device=dev)

    def run(h, rows):
        dh = torch.full(h.shape, 7.0, device=dev)
        capi.aj_lm_head_distill(cfg, (rows + 1).to(torch.int32), h, gamma, w, 1.0, t, torch.empty(2, device=dev), dh,
                                None, None, ws)
        torch.cuda.synchronize()
        return dh

    dh = run(h, rows)
    few = run(h[rows].contiguous(), torch.arange(2, device=dev))
    assert torch.equal(dh[rows], few) and bool(few.any())
    dh[rows] = 0
    for a in range(0, n, 1 << 16):
        assert not bool(dh[a:a + (1 << 16)].any())
