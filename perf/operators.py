"""The operators that turn a full-attention policy into a windowed one by distillation, as
cases that can be timed and compared.

  attn     attention over packed segments in which a query sees the last `window` keys of
           its segment and the segment's first `sink` keys (window 0: all keys up to its
           own); forward, or forward and backward as a training step runs them
  topk     the k largest logits of a row as log-probs under the row's whole softmax: what
           a teacher hands over
  distill  the loss of a student's logits against such a list, KL(teacher || student) with
           the teacher's listed tokens renormalised, or with all others as one more class;
           the loss alone, its gradient alone, or both in one call

Head counts, head dims, window-free lengths and vocabularies are those of
`workloads/configs.py`.  With `own` false every operator is computed from elementary torch
operations in float32; with `own` true by the library's entry points.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LOG2E = 1.4426950408889634


def listed():
    return [
        # a few short segments of the float32 policy, where launches weigh most
        dict(name="attn-tiny-f32", kind="attn", tokens=91, segs=3, hq=4, hkv=4, hd=32, window=24,
             sink=2, dtype="f32", train=True),
        # one batch of the float32 policy's merged episodes
        dict(name="attn-f32", kind="attn", tokens=3443, segs=13, hq=4, hkv=4, hd=32, window=128,
             sink=4, dtype="f32", train=True),
        # scoring two short episodes (reference or rollout log-probs): forward only
        dict(name="attn-fwd-1.5b-short", kind="attn", tokens=2347, segs=2, hq=12, hkv=2, hd=128,
             window=512, sink=4, dtype="bf16", train=False),
        # scoring a pack of agent episodes with narrow heads
        dict(name="attn-fwd-hd64", kind="attn", tokens=14511, segs=4, hq=28, hkv=4, hd=64,
             window=1024, sink=16, dtype="bf16", train=False),
        # a training pack of agent episodes
        dict(name="attn-train-7b", kind="attn", tokens=19437, segs=5, hq=28, hkv=4, hd=128,
             window=1024, sink=4, dtype="bf16", train=True),
        # one long-horizon episode, where the sinks see queries of the whole segment
        dict(name="attn-train-32b-long", kind="attn", tokens=32771, segs=1, hq=40, hkv=8, hd=128,
             window=2048, sink=4, dtype="bf16", train=True),
        # the teacher's list for one position of a response
        dict(name="topk-one", kind="topk", rows=1, vocab=151936, k=64, dtype="f32", pad=0, temp=1.0),
        # half-precision logits (many equal ones) of an episode's targets
        dict(name="topk-bf16", kind="topk", rows=1531, vocab=151936, k=20, dtype="bf16", pad=0,
             temp=2.0),
        # a slab of the 7B vocabulary, rows padded apart
        dict(name="topk-slab", kind="topk", rows=4096, vocab=152064, k=128, dtype="f32", pad=8,
             temp=1.0),
        # the float32 policy's loss: few rows of a small vocabulary
        dict(name="distill-tiny", kind="distill", rows=67, vocab=1024, k=8, dtype="f32",
             grad="f32", pad=0, temp=1.0, tail=True, part="step"),
        # scoring a student held in half precision: the loss alone
        dict(name="distill-fwd", kind="distill", rows=2751, vocab=151936, k=64, dtype="bf16",
             grad="bf16", pad=0, temp=1.5, tail=False, part="loss"),
        # a training slab of the 7B vocabulary: loss and half-precision gradient
        dict(name="distill-slab", kind="distill", rows=8192, vocab=152064, k=64, dtype="f32",
             grad="bf16", pad=0, temp=1.0, tail=True, part="step"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attn", "attn", "topk", "distill"])
    if kind == "attn":
        hq, hkv, hd = rng.choice([(4, 4, 32), (12, 2, 128), (28, 4, 128), (28, 4, 64), (8, 8, 64),
                                  (40, 8, 128)])
        f32 = hd == 32 or rng.random() < 0.15
        window = rng.choice([0, 1, 2]) and _log(rng, 8, 256 if f32 else 2048)
        top = 3500 if f32 else 20000 if window else 6000
        tokens = _log(rng, 1, top)
        return dict(kind="attn", tokens=tokens, segs=rng.randint(1, min(9, tokens)), hq=hq, hkv=hkv,
                    hd=hd, window=window, sink=rng.choice([0, 1, 4, _log(rng, 1, 100)]),
                    dtype="f32" if f32 else "bf16", train=rng.random() < 0.7)
    vocab = rng.choice([1024, 2000, 151936, 152064, _log(rng, 300, 160000)])
    rows = _log(rng, 1, min(20000, 4096 * 152064 // vocab))
    dtype = rng.choice(["f32", "bf16"])
    pad = rng.choice([0, 0, 1, 24])
    temp = rng.choice([1.0, 0.7, 2.0])
    if kind == "topk":
        return dict(kind="topk", rows=rows, vocab=vocab, k=_log(rng, 1, 256), dtype=dtype, pad=pad,
                    temp=temp)
    return dict(kind="distill", rows=rows, vocab=vocab, k=_log(rng, 1, 256), dtype=dtype,
                grad=dtype if dtype == "bf16" else rng.choice(["f32", "bf16"]), pad=pad, temp=temp,
                tail=rng.random() < 0.5, part=rng.choice(["loss", "grad", "step"]))


def _lengths(case):
    """The case's segment lengths: uneven, at least one token each."""
    r = random.Random(1000003 * case["tokens"] + case["segs"])
    cuts = sorted(r.sample(range(1, case["tokens"]), case["segs"] - 1))
    return [b - a for a, b in zip([0] + cuts, cuts + [case["tokens"]])]


# ------------------------------------------------------------------ attention

def _band(case, lens):
    """The pack cut into blocks of queries, each with the keys that any of them sees: token
    numbers of queries [blocks, B] and keys [blocks, K] (0 where there is none), and
    their positions in the segment (-1 where there is none)."""
    W = case["window"] or max(lens)
    S = case["sink"] if case["window"] else 0
    B = min(max(W, 64), max(lens), 2048)
    n = torch.tensor(lens)
    nb = (n + B - 1) // B
    seg = torch.repeat_interleave(torch.arange(len(lens)), nb)
    first = torch.cumsum(nb, 0) - nb
    p0 = (torch.arange(len(seg)) - first[seg]) * B            # first query of the block
    t0 = (torch.cumsum(n, 0) - n)[seg]                        # first token of its segment
    qpos = p0[:, None] + torch.arange(B)
    qpos = torch.where(qpos < n[seg][:, None], qpos, -1)
    back = min(W - 1, max(lens) - 1)
    low = (p0 - back)[:, None]
    band = low + torch.arange(back + B)
    band = torch.where((band >= 0) & (band < n[seg][:, None]), band, -1)
    sinks = torch.arange(min(S, max(lens)))[None].expand(len(seg), -1)
    sinks = torch.where(sinks < low, sinks, -1)               # those that the band has not
    kpos = torch.cat([sinks, band], 1)
    token = lambda p: torch.where(p >= 0, p + t0[:, None], 0)  # noqa: E731
    return [t.to(DEV) for t in (token(qpos), qpos, token(kpos), kpos)]


def _attn_prepare(case, g):
    lens = _lengths(case)
    n, hq, hkv, hd = case["tokens"], case["hq"], case["hkv"], case["hd"]
    dt = DTYPES[case["dtype"]]
    rnd = lambda *s: torch.randn(*s, generator=g, device=DEV, dtype=torch.float32)  # noqa: E731
    cu = torch.tensor([0] + lens).cumsum(0)
    st = {"case": case, "qkv": rnd(n, (hq + 2 * hkv) * hd).to(dt),
          "cu": cu.to(device=DEV, dtype=torch.int32), "longest": max(lens), "band": _band(case, lens)}
    if case["train"]:
        st["dout"] = rnd(n, hq * hd).to(dt)
    return st


def _attn_plain(st):
    c = st["case"]
    n, hq, hkv, hd = c["tokens"], c["hq"], c["hkv"], c["hd"]
    G, dt = hq // hkv, DTYPES[c["dtype"]]
    scale = 1.0 / math.sqrt(hd)
    qt, qp, kt, kp = st["band"]
    nb, B = qt.shape
    K = kt.shape[1]
    x = st["qkv"].float()
    q, k, v = x.split([hq * hd, hkv * hd, hkv * hd], 1)
    # [blocks, kv heads, G * B, hd] and [blocks, kv heads, K, hd]
    rows = lambda t: t.view(n, hkv, G, hd)[qt].permute(0, 2, 3, 1, 4).reshape(nb, hkv, G * B, hd)  # noqa: E731
    cols = lambda t: t.view(n, hkv, hd)[kt].permute(0, 2, 1, 3).contiguous()  # noqa: E731
    qb, kb, vb = rows(q), cols(k), cols(v)
    a, b = qp[:, :, None], kp[:, None, :]
    see = (a >= 0) & (b >= 0) & (b <= a)
    if c["window"]:
        see &= (b > a - c["window"]) | (b < c["sink"])
    see = see[:, None, None].expand(nb, 1, G, B, K).reshape(nb, 1, G * B, K)
    s = torch.matmul(qb, kb.transpose(2, 3).contiguous()).mul_(scale).masked_fill_(~see, -math.inf)
    m = s.amax(3, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)                   # the places past a segment's end
    p = s.sub_(m).exp_()
    l = p.sum(3, keepdim=True)
    p = p.div_(l.clamp(min=1e-30))
    ob = torch.matmul(p, vb)
    lseb = (m + l.log()).squeeze(3) * LOG2E
    put = qp.reshape(-1) >= 0
    at = qt.reshape(-1)[put]
    back = lambda t, w: t.view(nb, hkv, G, B, w).permute(0, 3, 1, 2, 4).reshape(nb * B, hkv * G * w)[put]  # noqa: E731
    out = torch.empty(n, hq * hd, device=DEV)
    out[at] = back(ob, hd)
    lse = torch.empty(n, hq, device=DEV)
    lse[at] = back(lseb, 1)
    res = {"out": out.to(dt), "lse": lse.t().contiguous()}
    if not c["train"]:
        return res
    do = rows(st["dout"].float())
    do = do * (qp >= 0)[:, None, None, :, None].expand(nb, 1, G, B, 1).reshape(nb, 1, G * B, 1)
    dp = torch.matmul(do, vb.transpose(2, 3).contiguous())
    ds = dp.sub_((do * ob).sum(3, keepdim=True)).mul_(p).mul_(scale)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    del p, s
    dq = torch.matmul(ds, kb)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), qb)
    dx = torch.zeros(n, (hq + 2 * hkv) * hd, device=DEV)
    dx[at, :hq * hd] = back(dq, hd)
    to = kt.reshape(-1)
    flat = lambda t: t.permute(0, 2, 1, 3).reshape(nb * K, hkv * hd)  # noqa: E731
    dx[:, hq * hd:].index_add_(0, to, torch.cat([flat(dk), flat(dv)], 1))
    return {**res, "dqkv": dx.to(dt)}


def _attn_own(st):
    from paper_2606_04484_amd import capi
    c = st["case"]
    n, hq, hd = c["tokens"], c["hq"], c["hd"]
    if "cfg" not in st:
        st["cfg"] = capi.attn_cfg(c["hq"], c["hkv"], c["hd"], window=c["window"], n_sink=c["sink"],
                                  dtype=DTYPES[c["dtype"]])
        st["ws"] = torch.empty(capi.aj_attention_workspace_bytes(st["cfg"], n), dtype=torch.uint8,
                               device=DEV)
    out = torch.empty(n, hq * hd, dtype=st["qkv"].dtype, device=DEV)
    lse = torch.empty(hq, n, dtype=torch.float32, device=DEV)
    capi.aj_attention_fwd(st["cfg"], st["cu"], st["longest"], st["qkv"], out, lse, st["ws"])
    res = {"out": out, "lse": lse}
    if c["train"]:
        res["dqkv"] = torch.empty_like(st["qkv"])
        capi.aj_attention_bwd(st["cfg"], st["cu"], st["longest"], st["qkv"], out, lse, st["dout"],
                              res["dqkv"], st["ws"])
    return res


def _attn_exact(case, st):
    """Segment by segment and 512 queries at a time, in 64 bits."""
    n, hq, hkv, hd = case["tokens"], case["hq"], case["hkv"], case["hd"]
    G, scale = hq // hkv, 1.0 / math.sqrt(hd)
    q, k, v = st["qkv"].double().split([hq * hd, hkv * hd, hkv * hd], 1)
    heads = lambda t, h: t.reshape(n, h, hd).transpose(0, 1).contiguous()  # noqa: E731
    q, k, v = heads(q, hq).view(hkv, G, n, hd), heads(k, hkv), heads(v, hkv)
    train = case["train"]
    do = heads(st["dout"].double(), hq).view(hkv, G, n, hd) if train else None
    out, lse = torch.empty_like(q), torch.empty(hkv, G, n, dtype=torch.float64, device=DEV)
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    start = 0
    for length in _lengths(case):
        for a in range(0, length, 512):
            b = min(a + 512, length)
            low = max(0, a - case["window"] + 1) if case["window"] else 0
            pos = torch.cat([torch.arange(min(case["sink"], low)), torch.arange(low, b)]).to(DEV)
            at = torch.arange(a, b, device=DEV)[:, None]
            hidden = pos > at
            if case["window"]:
                hidden |= (at - pos >= case["window"]) & (pos >= case["sink"])
            t, r = start + pos, slice(start + a, start + b)
            kk, vv = k[:, t], v[:, t]
            w = len(at)
            sc = (q[:, :, r].reshape(hkv, G * w, hd) @ kk.mT.contiguous() * scale).view(hkv, G, w, -1)
            sc = sc.masked_fill(hidden, -math.inf)
            ls = torch.logsumexp(sc, 3)
            p = torch.exp(sc - ls[..., None]).view(hkv, G * w, -1)
            o = p @ vv
            lse[:, :, r], out[:, :, r] = ls, o.view(hkv, G, w, hd)
            if not train:
                continue
            d = do[:, :, r].reshape(hkv, G * w, hd)
            ds = p * (d @ vv.mT.contiguous() - (d * o).sum(2, keepdim=True)) * scale
            dq[:, :, r] = (ds @ kk).view(hkv, G, w, hd)
            dk.index_add_(1, t, ds.mT.contiguous() @ q[:, :, r].reshape(hkv, G * w, hd))
            dv.index_add_(1, t, p.mT.contiguous() @ d)
        start += length
    flat = lambda t: t.reshape(-1, n, hd).transpose(0, 1).reshape(n, -1)  # noqa: E731
    res = {"out": flat(out), "lse": lse.view(hq, n) * LOG2E}
    if train:
        res["dqkv"] = torch.cat([flat(dq), flat(dk), flat(dv)], 1)
    return res


def _pairs(case):
    """Query-key pairs that are seen, over all segments."""
    W, S, total = case["window"], case["sink"], 0
    for n in _lengths(case):
        if not W or W >= n:
            total += n * (n + 1) // 2
            continue
        total += W * (W + 1) // 2 + (n - W) * W
        # query i >= W sees min(S, i - W + 1) sinks before its window
        full = max(0, n - W - S)
        part = n - W - full
        total += full * S + part * (part + 1) // 2
    return total


# ------------------------------------------------------------------ logits

def _logits(case, g):
    """Rows of logits as a trained head gives them: most of the mass on a few tokens."""
    z = torch.empty(case["rows"], case["vocab"] + case["pad"], device=DEV, dtype=torch.float32)
    z.normal_(0.0, 2.5, generator=g)
    z = z.to(DTYPES[case["dtype"]])
    return z[:, :case["vocab"]] if case["pad"] else z


def _k(case):
    return min(case["k"], case["vocab"])


def _topk_prepare(case, g):
    return {"case": case, "logits": _logits(case, g)}


def _lse(z):
    m = z.amax(1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    return m + (z - m).exp_().sum(1, keepdim=True).log_()


def _topk_plain(st):
    c, z = st["case"], st["logits"].float()
    top, at = torch.sort(z, dim=1, descending=True, stable=True)   # equal ones: lowest index first
    top, at = top[:, :_k(c)].clone(), at[:, :_k(c)].to(torch.int32)
    lse = _lse(z * (1.0 / c["temp"]))
    return {"idx": at, "logprob": top * (1.0 / c["temp"]) - lse, "lse": lse[:, 0]}


def _topk_own(st):
    from paper_2606_04484_amd import capi
    c, z = st["case"], st["logits"]
    k = _k(c)
    if "ws" not in st:
        st["ws"] = torch.empty(capi.aj_topk_workspace_bytes(c["rows"], c["vocab"], k),
                               dtype=torch.uint8, device=DEV)
    idx = torch.empty(c["rows"], k, dtype=torch.int32, device=DEV)
    logprob = torch.empty(c["rows"], k, dtype=torch.float32, device=DEV)
    lse = torch.empty(c["rows"], dtype=torch.float32, device=DEV)
    capi.aj_topk_logprob(z, 1.0 / c["temp"], idx, logprob, lse, st["ws"])
    return {"idx": idx, "logprob": logprob, "lse": lse}


def _topk_exact(case, st):
    k, lp, ls = _k(case), [], []
    for z in st["logits"].split(256):
        z = z.double() / case["temp"]
        ls.append(torch.logsumexp(z, 1))
        lp.append(torch.topk(z, k, dim=1).values - ls[-1][:, None])
    return {"idx": None, "logprob": torch.cat(lp), "lse": torch.cat(ls)}


def _distill_prepare(case, g):
    """The student's logits, and a teacher that agrees with them in part: its list is the
    top of the student's logits with noise.  Some positions list fewer tokens."""
    z = _logits(case, g)
    rows, k = case["rows"], _k(case)
    idx = torch.empty(rows, k, dtype=torch.int32, device=DEV)
    lp = torch.empty(rows, k, dtype=torch.float32, device=DEV)
    for a in range(0, rows, 1024):
        t = z[a:a + 1024].float()
        t = t + torch.empty_like(t).normal_(0.0, 1.0, generator=g)
        top, at = torch.topk(t, k, dim=1)
        idx[a:a + 1024], lp[a:a + 1024] = at, top - torch.logsumexp(t, 1, keepdim=True)
    short = torch.rand(rows, 1, generator=g, device=DEV) < 0.1
    idx[short & (torch.arange(k, device=DEV) >= (k + 1) // 2)] = -1
    weight = torch.rand(rows, generator=g, device=DEV) + 0.5
    st = {"case": case, "logits": z, "idx": idx, "logprob": lp, "weight": weight}
    if case["part"] == "grad":
        # what the forward pass has left for the gradient: the log-sum-exp of every
        # row, and that of the tokens outside its list
        s = torch.empty(2, rows, dtype=torch.float32, device=DEV)
        for a in range(0, rows, 512):
            r = slice(a, a + 512)
            t = z[r].double() / case["temp"]
            s[0, r] = torch.logsumexp(t, 1)
            at = torch.where(idx[r] >= 0, idx[r].long(), idx[r, :1].long())
            s[1, r] = torch.logsumexp(t.scatter(1, at, -math.inf), 1)
        st["lse"] = s
    return st


def _distill_plain(st):
    c = st["case"]
    inv = 1.0 / c["temp"]
    z = st["logits"].float() * inv
    on = st["idx"] >= 0
    at = torch.where(on, st["idx"], st["idx"][:, :1]).long()   # the first one is always there
    t = torch.where(on, st["logprob"], -math.inf)
    p = t.exp()
    if c["tail"]:
        rest = (1.0 - p.double().sum(1, keepdim=True)).clamp(min=0.0).float()
        mass = p.sum(1, keepdim=True) + rest
    else:
        t = t - _lse(t)
        p = t.exp()
        rest, mass = torch.zeros_like(p[:, :1]), torch.ones_like(p[:, :1])
    zt = z.gather(1, at)
    if c["part"] == "grad":
        lse, lse_rest = st["lse"][0][:, None], st["lse"][1][:, None]
    else:
        lse, lse_rest = _lse(z), _lse(z.scatter(1, at, -math.inf))
    res = {}
    if c["part"] != "grad":
        kl = torch.where(p > 0, p * (t - (zt - lse)), 0.0).sum(1, keepdim=True)
        if c["tail"]:
            kl = kl + torch.where(rest > 0, rest * (rest.log() - (lse_rest - lse)), 0.0)
        res = {"loss": kl[:, 0], "lse": torch.cat([lse, lse_rest], 1).t().contiguous()}
    if c["part"] != "loss":
        w = (st["weight"] * (inv / c["rows"]))[:, None]
        listed_dz = w * (mass * (zt - lse).exp() - p)
        if c["tail"]:
            dz = (z - torch.where(lse_rest == -math.inf, 0.0, lse_rest)).exp_()
            dz.mul_(w * (mass * (lse_rest - lse).exp() - rest))
        else:
            dz = (z - lse).exp_().mul_(w * mass)
        src = torch.where(on, listed_dz, listed_dz[:, :1])
        res["dlogits"] = dz.scatter_(1, at, src).to(DTYPES[c["grad"]])
    return res


def _distill_own(st):
    from paper_2606_04484_amd import capi
    c, z = st["case"], st["logits"]
    rows, k = c["rows"], _k(c)
    if "ws" not in st:
        st["ws"] = torch.empty(capi.aj_distill_workspace_bytes(rows, c["vocab"], k),
                               dtype=torch.uint8, device=DEV)
    teacher = capi.teacher(st["idx"], st["logprob"], tail=c["tail"], weight=st["weight"],
                           coef=1.0 / rows)
    res = {}
    if c["part"] != "grad":
        res = {"loss": torch.empty(rows, dtype=torch.float32, device=DEV),
               "lse": torch.empty(2, rows, dtype=torch.float32, device=DEV)}
    if c["part"] != "loss":
        res["dlogits"] = torch.empty(rows, c["vocab"], dtype=DTYPES[c["grad"]], device=DEV)
    inv = 1.0 / c["temp"]
    if c["part"] == "loss":
        capi.aj_distill_loss_fwd(z, inv, teacher, res["loss"], res["lse"], ws=st["ws"])
    elif c["part"] == "grad":
        capi.aj_distill_loss_bwd(z, inv, teacher, st["lse"], res["dlogits"])
    else:
        capi.aj_distill_loss_fwd_bwd(z, inv, teacher, res["loss"], res["lse"], res["dlogits"],
                                     ws=st["ws"])
    return res


def _distill_exact(case, st):
    parts = []
    for a in range(0, case["rows"], 256):
        r = slice(a, min(a + 256, case["rows"]))
        z = st["logits"][r].double() / case["temp"]
        on = st["idx"][r] >= 0
        row, col = on.nonzero()[:, 0], st["idx"][r][on].long()
        teach = torch.zeros_like(z)                 # the teacher's distribution over all tokens
        teach[row, col] = st["logprob"][r][on].double().exp()
        named = torch.zeros_like(z, dtype=torch.bool)
        named[row, col] = True
        logq = torch.log_softmax(z, 1)
        lse = torch.logsumexp(z, 1)
        lse_rest = torch.logsumexp(z.masked_fill(named, -math.inf), 1)
        rest = torch.zeros_like(lse)
        if case["tail"]:
            rest = (1.0 - teach.sum(1)).clamp(min=0.0)
        else:
            teach /= teach.sum(1, keepdim=True)
        loss = (torch.xlogy(teach, teach) - torch.where(teach > 0, teach * logq, 0.0)).sum(1)
        loss += torch.where(rest > 0, torch.xlogy(rest, rest) - rest * (lse_rest - lse), 0.0)
        # the rest of the teacher's mass, shared out as the student shares its own
        teach += torch.where(named, 0.0, rest[:, None] * (z - lse_rest[:, None]).exp())
        mass = teach.sum(1, keepdim=True)
        dz = (mass * logq.exp() - teach) * (st["weight"][r].double() / case["temp"] / case["rows"])[:, None]
        parts.append((loss, torch.stack([lse, lse_rest]), dz.float() if case["grad"] == "bf16" else dz))
    res = {}
    if case["part"] != "grad":
        res = {"loss": torch.cat([p[0] for p in parts]), "lse": torch.cat([p[1] for p in parts], 1)}
    if case["part"] != "loss":
        res["dlogits"] = torch.cat([p[2] for p in parts])
    return res


# ------------------------------------------------------------------ the calls

PREPARE = {"attn": _attn_prepare, "topk": _topk_prepare, "distill": _distill_prepare}
PLAIN = {"attn": _attn_plain, "topk": _topk_plain, "distill": _distill_plain}
OWN = {"attn": _attn_own, "topk": _topk_own, "distill": _distill_own}
EXACT = {"attn": _attn_exact, "topk": _topk_exact, "distill": _distill_exact}


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return PREPARE[case["kind"]](case, g)


def run(state):
    return (OWN if own else PLAIN)[state["case"]["kind"]](state)


def exact(case, seed):
    return EXACT[case["kind"]](case, prepare(case, seed))


def work(case):
    es = {"f32": 4, "bf16": 2}
    if case["kind"] == "attn":
        n, hq, hkv, hd, e = (case[k] for k in ("tokens", "hq", "hkv", "hd", "dtype"))
        e = es[e]
        width, pairs = (hq + 2 * hkv) * hd, _pairs(case) * hq
        nbytes, flops = n * (width + hq * hd) * e + 4 * n * hq, 4.0 * pairs * hd
        if case["train"]:   # d out read, d qkv written; scores again, dP, dQ, dK, dV
            nbytes, flops = nbytes + n * (width + hq * hd) * e, flops + 10.0 * pairs * hd
        return {"bytes": float(nbytes), "flops": flops}
    rows, vocab, k = case["rows"], case["vocab"], _k(case)
    nbytes = rows * vocab * es[case["dtype"]] + 8 * rows * k
    if case["kind"] == "topk":
        return {"bytes": float(nbytes + 4 * rows), "flops": 4.0 * rows * vocab}
    nbytes += 16 * rows
    if case["part"] != "loss":
        nbytes += rows * vocab * es[case["grad"]]
    return {"bytes": float(nbytes), "flops": 4.0 * rows * vocab}
