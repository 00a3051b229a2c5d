"""Pins of the oracle's windowed attention and distillation loss against library ops and torch
autograd in float64, and of their limits."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import merge as om
from oracle import model as M
from tests.gpu_cases import workload, bf16_case_model, episodes
from workloads import make_timelines, make_weights_numpy


@pytest.mark.parametrize("window, n_sink", [(0, 0), (1, 0), (1, 2), (7, 0), (7, 3), (40, 5), (3, 40)])
def test_window_attention_against_autograd(window, n_sink):
    g = torch.Generator().manual_seed(1)
    L, hq, hkv, hd = 33, 4, 2, 8
    q, k, v, do = (torch.randn(L, h, hd, generator=g, dtype=torch.float64, requires_grad=True)
                   for h in (hq, hkv, hkv, hq))
    see = torch.zeros(L, L, dtype=torch.bool)
    for i in range(L):
        for j in range(i + 1):
            see[i, j] = window == 0 or j > i - window or j < n_sink
    rep = lambda t: t.repeat_interleave(hq // hkv, 1).transpose(0, 1)  # noqa: E731
    o = torch.nn.functional.scaled_dot_product_attention(q.transpose(0, 1)[None], rep(k)[None], rep(v)[None],
                                                         attn_mask=see)[0].transpose(0, 1)
    o.backward(do)
    a = [t.detach().numpy() for t in (q, k, v)]
    mine, lse = M.attention_segment(*a, hd ** -0.5, window, n_sink)
    np.testing.assert_allclose(mine, o.detach().numpy(), rtol=0, atol=1e-12)
    grads = M.attention_segment_bwd(*a, mine, lse, do.detach().numpy(), hd ** -0.5, window, n_sink)
    for got, t in zip(grads, (q, k, v)):
        np.testing.assert_allclose(got, t.grad.numpy(), rtol=0, atol=1e-12)


@pytest.mark.parametrize("tail", [False, True])
def test_distill_terms_against_autograd(tail):
    g = torch.Generator().manual_seed(2)
    z = torch.randn(5, 30, generator=g, dtype=torch.float64, requires_grad=True)
    t = torch.log_softmax(2 * torch.randn(5, 30, generator=g, dtype=torch.float64), 1)
    lp, idx = torch.topk(t, 6, dim=1)
    idx[3, 4:] = -1
    loss, dz = M.distill_terms(z.detach().numpy(), idx.numpy(), lp.numpy(), tail)
    logq = torch.log_softmax(z, 1)
    for i in range(5):
        on = idx[i] >= 0
        a, l = idx[i][on], lp[i][on]
        if tail:
            others = torch.ones(30, dtype=torch.bool)
            others[a] = False
            p = torch.cat([l.exp(), 1 - l.exp().sum()[None]])
            lq = torch.cat([logq[i][a], torch.logsumexp(logq[i][others], 0)[None]])
        else:
            p, lq = torch.softmax(l, 0), logq[i][a]
        want = torch.nn.functional.kl_div(lq, p, reduction="sum")
        assert abs(loss[i] - want.item()) < 1e-12
        grad, = torch.autograd.grad(want, z, retain_graph=True)
        np.testing.assert_allclose(dz[i], grad[i].numpy(), rtol=0, atol=1e-12)


def test_distill_limits():
    """A teacher that is the student: no loss, no gradient, whatever is listed (with a tail); the
    whole vocabulary listed: the plain KL; nothing listed: nothing."""
    z = np.random.default_rng(0).normal(size=(3, 20))
    q = np.log(np.exp(z) / np.exp(z).sum(1, keepdims=True))
    idx = np.argsort(-z, axis=1)[:, :5]
    loss, dz = M.distill_terms(z, idx, np.take_along_axis(q, idx, 1), True)
    assert np.abs(loss).max() < 1e-14 and np.abs(dz).max() < 1e-14
    every = np.tile(np.arange(20), (3, 1))
    t = np.random.default_rng(1).normal(size=(3, 20))
    t -= np.log(np.exp(t).sum(1, keepdims=True))
    loss, dz = M.distill_terms(z, every, t, False)
    np.testing.assert_allclose(loss, (np.exp(t) * (t - q)).sum(1), rtol=0, atol=1e-13)
    np.testing.assert_allclose(dz, np.exp(q) - np.exp(t), rtol=0, atol=1e-13)
    for tail in (False, True):
        loss, dz = M.distill_terms(z, np.full((3, 2), -1), np.zeros((3, 2)), tail)
        assert np.abs(loss).max() < 1e-15 and np.abs(dz).max() < 1e-15   # (log of a sum of 20: 2^-53 each)


def test_distill_update_against_differences():
    m = dataclasses.replace(bf16_case_model(hd=8, d=16, hq=2, hkv=1, ff=24, vocab=40), dtype="f32", n_layers=2,
                            window=9, n_sink=2)
    cfg = workload(m, n_traj=2, turns=(2, 2), prompt=(6, 6), resp=(3, 5), obs=(2, 4))
    tl = make_timelines(cfg)
    packed = om.merge_batch(episodes(tl, np.zeros(tl.n_tok, np.float32)))[0]
    W = {k: v.astype(np.float64) for k, v in make_weights_numpy(m, gain_std=0.1).items()}
    n = len(M.masked_targets(packed))
    rng = np.random.default_rng(3)
    idx = np.stack([rng.permutation(40)[:6] for _ in range(n)])
    lp = np.log(rng.dirichlet(np.ones(8), n)[:, :6])
    w = rng.uniform(0.5, 1.5, n)
    got = M.distill_update(packed, W, m, idx, lp, True, 0.7, w)
    for name in ("w_qkv", "w_down.1", "w_vocab", "final_norm", "emb"):
        d = rng.normal(size=W[name].shape)
        h = 1e-5
        f = [M.distill_update(packed, {**W, name: W[name] + s * d}, m, idx, lp, True, 0.7, w)["loss"] for s in (h, -h)]
        want = (f[0] - f[1]) / (2 * h)
        assert abs((got["grads"][name] * d).sum() - want) < 1e-7 * max(1, abs(want)), name
