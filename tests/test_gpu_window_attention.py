"""Windowed attention with sinks against its definition in 64 bits (tests/window_attention.py),
within the error that its roundings allow; what it leaves alone, and what it refuses."""
import math

import pytest
import torch

from window_attention import reference, visible

pytestmark = pytest.mark.gpu

#      lens, hq, hkv, hd, window, sinks
CASES = [
    ([1], 1, 1, 8, 1, 0),
    ([1, 1, 2, 1], 4, 2, 64, 1, 1),
    ([130], 2, 1, 64, 1, 0),                 # each row sees itself alone
    ([130, 67], 2, 1, 128, 1, 4),            # itself and the sinks
    ([64, 64, 64], 4, 4, 64, 64, 4),         # segments and windows on tile edges
    ([63, 65, 1, 129], 6, 2, 128, 63, 3),
    ([300, 41], 4, 1, 64, 65, 1),
    ([513], 3, 3, 128, 100, 70),             # more sinks than a tile holds
    ([200, 300], 4, 2, 64, 32, 1000),        # more sinks than tokens: full attention
    ([700], 2, 2, 32, 37, 5),                # the plain kernels' head dims
    ([90, 210], 3, 1, 40, 50, 9),
    ([257, 3, 140], 2, 1, 128, 130, 128),
    ([1100], 2, 1, 64, 300, 130),            # sinks over more than 128 keys
    ([2500, 1, 1400], 2, 1, 128, 200, 4),
    ([2300], 7, 1, 64, 1024, 4),
    ([40, 257, 600, 300, 1300], 4, 2, 32, 16, 128),    # (of 256 here)
    ([258, 5, 700], 2, 1, 96, 1, 70),
    ([40, 1025, 1100, 30, 2049], 4, 2, 64, 16, 128),   # sinks whose queries are taken in chunks
    ([1030, 5, 1027], 2, 1, 128, 1, 40),
    ([3, 4100], 6, 2, 128, 1500, 33),
    ([0, 130, 0, 0, 67, 0], 4, 2, 64, 20, 3),          # segments of no tokens
    ([0, 1300, 0, 0, 1100, 0], 2, 1, 128, 200, 6),
    ([0, 300, 0, 260, 0], 2, 1, 32, 30, 6),
    ([50, 60], 4, 2, 64, 4096, 4),           # a window that no row reaches past
]


def call(lens, hq, hkv, hd, window, n_sink, dtype, base=0, seed=0, scale=0.0, std=1.0, bad=None):
    from paper_2606_04484_amd import capi
    g = torch.Generator().manual_seed(seed)
    n = sum(lens)
    dev = "cuda"
    qkv = (torch.randn(n, (hq + 2 * hkv) * hd, generator=g) * std).to(dtype)
    dout = torch.randn(n, hq * hd, generator=g).to(dtype)
    cu = (torch.tensor([0] + lens).cumsum(0) + base).to(torch.int32).to(dev)
    cfg = capi.attn_cfg(hq, hkv, hd, window=window, n_sink=n_sink, dtype=dtype, scale=scale)
    ws = torch.full((capi.aj_attention_workspace_bytes(cfg, n),), 255, dtype=torch.uint8, device=dev)
    out = torch.full((n, hq * hd), float("nan"), dtype=dtype, device=dev)
    lse = torch.full((hq, n), float("nan"), device=dev)
    dqkv = torch.full((n, (hq + 2 * hkv) * hd), float("nan"), dtype=dtype, device=dev)
    x, dx = qkv.to(dev), dout.to(dev)
    if bad is not None:      # (rows, value): in the operands, not in what is returned
        x[bad[0]] = dx[bad[0]] = bad[1]
    capi.aj_attention_fwd(cfg, cu, max(lens), x, out, lse, ws, base=base)
    ws.fill_(255)
    capi.aj_attention_bwd(cfg, cu, max(lens), x, out, lse, dx, dqkv, ws, base=base)
    torch.cuda.synchronize()
    return qkv, dout, {"out": out.cpu(), "lse": lse.cpu(), "dqkv": dqkv.cpu()}


def check(got, want):
    for name, (val, err) in want.items():
        off = (got[name].double() - val).abs()
        assert bool(torch.isfinite(got[name]).all()), name
        worst = (off / (err + 1e-30)).max().item()
        assert worst <= 1.0, (name, worst, off.max().item())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(map(str, c[0])) + "-w%d-s%d-hd%d" % (c[4], c[5], c[3]))
def test_matches_definition(case, dtype):
    lens, hq, hkv, hd, window, n_sink = case
    qkv, dout, got = call(*case, dtype)
    check(got, reference(qkv, lens, hq, hkv, hd, window, n_sink, dout, bf16=dtype == torch.bfloat16))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_scale_base_and_large_scores(dtype):
    """Offsets of a slice of a larger batch, a scale of its own, scores of tens."""
    lens, hq, hkv, hd, window, n_sink = [311, 90], 4, 2, 64, 77, 4
    qkv, dout, got = call(lens, hq, hkv, hd, window, n_sink, dtype, base=123457, seed=3, scale=0.25,
                          std=2.0)
    check(got, reference(qkv, lens, hq, hkv, hd, window, n_sink, dout, scale=0.25,
                         bf16=dtype == torch.bfloat16))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_window_of_the_segment_is_full_attention(dtype):
    """The same numbers, bit for bit, whether no window is asked for or one that hides nothing."""
    a = call([333, 150], 4, 2, 64, 0, 0, dtype)[2]
    b = call([333, 150], 4, 2, 64, 483, 7, dtype)[2]
    for k in a:
        assert torch.equal(a[k], b[k]), k


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_same_bits_every_call(dtype):
    a = call([2100, 700], 4, 2, 128, 150, 4, dtype)[2]
    b = call([2100, 700], 4, 2, 128, 150, 4, dtype)[2]
    for k in a:
        assert torch.equal(a[k], b[k]), k


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_gradient_against_differences(dtype):
    """d qkv along a direction against the change of sum(dout * out) in 64 bits."""
    case = ([150, 60], 4, 2, 64, 40, 3)
    lens, hq, hkv, hd, window, n_sink = case
    qkv, dout, got = call(*case, dtype, seed=9)
    step = torch.randn(qkv.shape, generator=torch.Generator().manual_seed(1)).double()
    h = 1e-5
    f = [(reference(qkv.double() + t * step, lens, hq, hkv, hd, window, n_sink)["out"][0]
          * dout.double()).sum() for t in (h, -h)]
    want = ((f[0] - f[1]) / (2 * h)).item()
    err = reference(qkv, lens, hq, hkv, hd, window, n_sink, dout, bf16=dtype == torch.bfloat16)["dqkv"][1]
    have = (got["dqkv"].double() * step).sum().item()
    assert abs(have - want) <= (err * step.abs()).sum().item() + 1e-6 * abs(want)


@pytest.mark.parametrize("train", [False, True], ids=["fwd", "fwd+bwd"])
def test_captured_and_replayed(train):
    """A graph of the calls, replayed with the program's own eager calls in between."""
    from paper_2606_04484_amd import capi
    lens, hq, hkv, hd, window, n_sink = [1500, 77], 4, 2, 128, 200, 4
    n = sum(lens)
    cfg = capi.attn_cfg(hq, hkv, hd, window=window, n_sink=n_sink)
    cu = torch.tensor([0] + lens).cumsum(0).to(torch.int32).cuda()
    ws = torch.empty(capi.aj_attention_workspace_bytes(cfg, n), dtype=torch.uint8, device="cuda")
    qkv = torch.randn(n, (hq + 2 * hkv) * hd, device="cuda").bfloat16()
    dout = torch.randn(n, hq * hd, device="cuda").bfloat16()
    out, dqkv = torch.empty_like(dout), torch.empty_like(qkv)
    lse = torch.empty(hq, n, device="cuda")

    def run():
        capi.aj_attention_fwd(cfg, cu, max(lens), qkv, out, lse, ws)
        if train:
            capi.aj_attention_bwd(cfg, cu, max(lens), qkv, out, lse, dout, dqkv, ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        run()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        qkv.copy_(torch.randn(qkv.shape, device="cuda"))
        run()
        torch.cuda.synchronize()
        want = [t.clone() for t in (out, lse, dqkv)]
        out.zero_(), lse.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((out, lse) + ((dqkv,) if train else ()), want):
            assert torch.equal(a, b), i


def test_empty_pack_and_unaligned_rows():
    """No tokens: nothing is launched.  Views that start off a 16-byte boundary are right too."""
    from paper_2606_04484_amd import capi
    cfg = capi.attn_cfg(2, 1, 64, window=8, n_sink=1)
    e = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device="cuda")  # noqa: E731
    ws = e(capi.aj_attention_workspace_bytes(cfg, 0) + 1, dt=torch.uint8)
    cu = torch.zeros(1, dtype=torch.int32, device="cuda")
    capi.aj_attention_fwd(cfg, cu, 0, e(0, 256), e(0, 128), e(2, 0, dt=torch.float32), ws)
    lens, n = [90, 45], 135
    g = torch.Generator().manual_seed(5)
    qkv = torch.randn(n, 256, generator=g).bfloat16()
    dout = torch.randn(n, 128, generator=g).bfloat16()
    off = lambda t: torch.cat([t.new_zeros(1), t.reshape(-1)]).cuda()[1:].view(t.shape)  # noqa: E731
    ws = e(capi.aj_attention_workspace_bytes(cfg, n), dt=torch.uint8)
    cu = torch.tensor([0] + lens).cumsum(0).to(torch.int32).cuda()
    q, out, dq = off(qkv), off(torch.zeros(n, 128).bfloat16()), off(torch.zeros(n, 256).bfloat16())
    lse = e(2, n, dt=torch.float32)
    capi.aj_attention_fwd(cfg, cu, 90, q, out, lse, ws)
    capi.aj_attention_bwd(cfg, cu, 90, q, out, lse, off(dout), dq, ws)
    torch.cuda.synchronize()
    check({"out": out.cpu(), "lse": lse.cpu(), "dqkv": dq.cpu()},
          reference(qkv, lens, 2, 1, 64, 8, 1, dout, bf16=True))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_bad_rows_far_from_the_window_do_no_harm(dtype):
    """Infinities and NaN in a segment reach only rows of that segment's tiles: rows whose
    window starts well after them are what they are without them."""
    from paper_2606_04484_amd import capi
    n, hq, hkv, hd, window, n_sink = 1500, 2, 1, 64, 128, 2
    cfg = capi.attn_cfg(hq, hkv, hd, window=window, n_sink=n_sink, dtype=dtype)
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    ws = torch.empty(capi.aj_attention_workspace_bytes(cfg, n), dtype=torch.uint8, device="cuda")
    x = torch.randn(n, (hq + 2 * hkv) * hd, generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    res = []
    for bad in (False, True):
        y = x.clone()
        if bad:
            y[300], y[301, ::3] = float("nan"), float("inf")
        out, lse = torch.empty(n, hq * hd, dtype=dtype, device="cuda"), torch.empty(hq, n, device="cuda")
        capi.aj_attention_fwd(cfg, cu, n, y, out, lse, ws)
        torch.cuda.synchronize()
        res.append(out.cpu())
    # a tile of 64 keys that holds rows 300 and 301 is read by queries within the next
    # 64 + window rows, and by their neighbours in a workgroup of 256
    far = torch.cat([torch.arange(0, 44), torch.arange(301 + 64 + window + 256, n)])
    assert torch.equal(res[0][far], res[1][far])


def touched(lens, window, n_sink, bad):
    """Rows that see a bad one (themselves included), and rows that such a row sees."""
    n = sum(lens)
    see = torch.zeros(n, n, dtype=torch.bool)
    a = 0
    for L in lens:
        see[a:a + L, a:a + L] = visible(L, window, n_sink)
        a += L
    q = see[:, bad].any(1)
    return q, see[q].any(0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf], ids=["nan", "+inf", "-inf"])
@pytest.mark.parametrize("case", [
    # lens, hq, hkv, hd, window, sinks, bad rows
    ([200, 90, 150], 4, 2, 64, 20, 3, [70, 120, 289]),
    ([200, 90, 150], 2, 1, 128, 20, 3, list(range(200, 290))),     # a segment that nothing wrote
    ([31, 300], 7, 1, 128, 65, 0, [31, 32, 100, 330]),
    ([2500, 40], 2, 1, 128, 50, 4, [1300, 2499]),                  # far sinks' chunks
    ([1300, 33, 1100], 2, 2, 64, 30, 70, [1299, 1300, 1400]),
    ([300, 60], 2, 1, 32, 20, 3, [299, 310]),
], ids=lambda c: "x".join(map(str, c[0])) + "-hd%d" % c[3])
def test_bad_rows_stay_with_the_rows_that_see_them(case, value, dtype):
    """Infinities and NaN in a row, and in its output gradient, leave every result that does not
    depend on that row what its definition says, in the same tile too."""
    lens, hq, hkv, hd, window, n_sink, bad = case
    qkv, dout, got = call(*case[:6], dtype, seed=4, bad=(bad, value))
    q, k = touched(lens, window, n_sink, bad)
    assert not q.all() and not (q | k).all()
    for name, (val, err) in reference(qkv, lens, hq, hkv, hd, window, n_sink, dout,
                                      bf16=dtype == torch.bfloat16).items():
        rows = [(got[name], val, err, q)]
        if name == "lse":
            rows = [(got[name].T, val.T, err.T, q)]
        elif name == "dqkv":
            rows = [(t[0], t[1], t[2], m) for t, m in zip(
                zip(*(x.split([hq * hd, 2 * hkv * hd], 1) for x in (got[name], val, err))), (q, k))]
        for part, (have, want, room, skip) in enumerate(rows):
            have, want, room = have[~skip], want[~skip], room[~skip]
            assert bool(torch.isfinite(have).all()), (name, part)
            worst = ((have.double() - want).abs() / (room + 1e-30)).max().item()
            assert worst <= 1.0, (name, part, worst)


@pytest.mark.parametrize("case", [([130, 3], 4, 2, 64, 1, 0), ([300], 2, 1, 128, 1, 0), ([1], 4, 2, 128, 0, 0),
                                  ([1] * 70, 4, 2, 64, 0, 0), ([1] * 90, 7, 1, 128, 30, 4)],
                         ids=lambda c: "%dx%d-w%d-hd%d" % (len(c[0]), c[0][0], c[4], c[3]))
def test_rows_of_one_key_pass_no_gradient_to_scores(case):
    """p = 1 and dP = delta: d q and d k are what float32 leaves of their difference, not the
    rounding of a bfloat16 output."""
    lens, hq, hkv, hd, window, n_sink = case
    qkv, dout, got = call(*case, torch.bfloat16, seed=6)
    n, G, c = sum(lens), hq // hkv, 1.0 / math.sqrt(hd)
    q, k, v = (t.reshape(n, -1, hd).abs() for t in qkv.double().split([hq * hd, hkv * hd, hkv * hd], 1))
    k, v = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    d = dout.double().reshape(n, hq, hd).abs()
    # dP twice, hd products each; p, the exponential of a score less its log-sum-exp, by its own error
    size = c * (q * k).sum(2)
    ds = 2.0 ** -24 * (2 * (hd + 4) + 4 * (hd + 6) * size + 16) * (d * v).sum(2)
    room = torch.cat([(ds[..., None] * k * c).reshape(n, -1),
                      (ds[..., None] * q * c).reshape(n, hkv, G, hd).sum(2).reshape(n, -1)], 1) * (1 + 2.0 ** -7)
    assert bool((got["dqkv"][:, :(hq + hkv) * hd].double().abs() <= room).all())
