"""Captured calls, every output cleared to NaN (lists to -7) before each replay, so that what a
replay does not write is seen; with the program's own eager calls between the replays."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def clear(tensors):
    for t in tensors:
        t.fill_(float("nan") if t.is_floating_point() else -7)


def check(run, inputs, outputs, keep=()):
    """keep: tensors that the calls add to, zero before each run."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    seen = None
    for i in range(4):
        for t in inputs:
            t.copy_(torch.randn(t.shape, device="cuda"))
        clear(outputs)
        [t.zero_() for t in keep]
        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in (*outputs, *keep)]
        assert seen is None or not any(torch.equal(a, b) for a, b in zip(want, seen))     # other inputs
        clear(outputs)
        [t.zero_() for t in keep]
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((*outputs, *keep), want):
            assert bool(torch.isfinite(b).all()) and torch.equal(a, b), i
        seen = want


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens, window", [([1500, 77], 200), ([1500, 1100], 0), ([40, 60, 3], 0), ([130, 90], 16)])
def test_attention(lens, window, dtype):
    from paper_2606_04484_amd import capi
    hq, hkv, hd, n = 4, 2, 64, sum(lens)
    cfg = capi.attn_cfg(hq, hkv, hd, window=window, n_sink=4, dtype=dtype)
    cu = torch.tensor([0] + lens).cumsum(0).to(torch.int32).cuda()
    ws = torch.empty(capi.aj_attention_workspace_bytes(cfg, n), dtype=torch.uint8, device="cuda")
    qkv = torch.randn(n, (hq + 2 * hkv) * hd, device="cuda").to(dtype)
    dout = torch.randn(n, hq * hd, device="cuda").to(dtype)
    out, dqkv, lse = torch.empty_like(dout), torch.empty_like(qkv), torch.empty(hq, n, device="cuda")

    def run():
        capi.aj_attention_fwd(cfg, cu, max(lens), qkv, out, lse, ws)
        capi.aj_attention_bwd(cfg, cu, max(lens), qkv, out, lse, dout, dqkv, ws)

    check(run, [qkv, dout], [out, lse, dqkv])


@pytest.mark.parametrize("rows, vocab", [(9, 20000), (600, 50000), (70, 1024), (1100, 9000)])
def test_lists_and_distillation(rows, vocab):
    from paper_2606_04484_amd import capi
    k, dev = 16, "cuda"
    z, student = torch.randn(rows, vocab, device=dev), torch.randn(rows, vocab, device=dev)
    idx = torch.empty(rows, k, dtype=torch.int32, device=dev)
    lp, lse1 = torch.empty(rows, k, device=dev), torch.empty(rows, device=dev)
    loss, lse, dz = torch.empty(rows, device=dev), torch.empty(2, rows, device=dev), torch.empty_like(z)
    lse2, loss2, dz2, stats = torch.empty_like(lse), torch.empty_like(loss), torch.empty_like(z), torch.zeros(2, device=dev)
    ws = torch.empty(max(capi.aj_topk_workspace_bytes(rows, vocab, k), capi.aj_distill_workspace_bytes(rows, vocab, k)),
                     dtype=torch.uint8, device=dev)
    t = capi.teacher(idx, lp, tail=True)

    def run():
        capi.aj_topk_logprob(z, 1.0, idx, lp, lse1, ws)
        capi.aj_distill_loss_fwd_bwd(student, 1.0, t, loss, lse, dz, ws, stats=stats)
        capi.aj_distill_loss_fwd(student, 1.0, t, loss2, lse2, ws)
        capi.aj_distill_loss_bwd(student, 1.0, t, lse2, dz2)

    check(run, [z, student], [idx, lp, lse1, loss, lse, dz, loss2, lse2, dz2])
    stats.zero_()
    run()
    torch.cuda.synchronize()
    assert stats[1] == rows
