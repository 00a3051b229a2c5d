"""A full-attention teacher's lists and a windowed student's update from them, through
actor.ActorUpdate, against the float64 oracle on the same merged timelines.

Tolerances are those of the actor update: float32 1e-4 (log-probs absolute, loss relative,
gradients relative L2), bfloat16 2e-2, 1e-2 and 1e-2 with cosine >= 0.999."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle import model as M
from tests.gpu_cases import Case, bf16_case_model, workload, rel_l2, cosine
from workloads import get_config, make_lora_numpy

pytestmark = pytest.mark.gpu

TINY = get_config(0).model


def policies(case, window, n_sink, seed=2000):
    """(teacher model, its weights), (student model, its weights: the case's)."""
    from workloads import bf16_round, make_weights_numpy
    Wt = make_weights_numpy(case.m, seed=seed, gain_std=0.1)
    if case.m.dtype == "bf16":
        Wt = {k: bf16_round(v) for k, v in Wt.items()}
    return (case.m, Wt), (dataclasses.replace(case.m, window=window, n_sink=n_sink), case.W)


CASES = {
    "f32": (TINY, dict(), 24, 2),
    "f32-2-layers": (dataclasses.replace(TINY, n_layers=2), dict(), 100, 4),
    "bf16-hd64": (bf16_case_model(hd=64), dict(), 70, 4),
    "bf16-hd128-2-layers": (dataclasses.replace(bf16_case_model(hd=128, d=256, hq=4, hkv=2, vocab=3000), n_layers=2),
                            dict(n_traj=4), 33, 1),
    # segments whose sinks see past their window for more than a chunk of queries
    "bf16-long": (bf16_case_model(hd=64, hq=2, hkv=1), dict(n_traj=2, prompt=(900, 1100), resp=(64, 128), obs=(64, 128)),
                  128, 4),
}


@pytest.mark.parametrize("pack_tokens", [131072, 700], ids=["one-pack", "packs"])
@pytest.mark.parametrize("tail", [True, False], ids=["tail", "listed"])
@pytest.mark.parametrize("name", list(CASES))
def test_teacher_and_student(name, tail, pack_tokens):
    from paper_2606_04484_amd import actor
    m, recipe, window, n_sink = CASES[name]
    case = Case(workload(m, **recipe))
    (mt, Wt), (ms, Ws) = policies(case, window, n_sink)
    f32, temp, k = m.dtype == "f32", 1.25, 24
    dev = actor.upload_timelines(case.tl, case.old)
    L = actor.merge(dev, pack_tokens=pack_tokens)
    T = actor.ActorUpdate(mt, case.device_weights(which=Wt))
    idx, lp = T.teacher_topk(L, k, temperature=temp)
    S = actor.ActorUpdate(ms, case.device_weights())
    S.zero_grads()
    w = torch.rand(L.n_mask, generator=torch.Generator().manual_seed(1)) + 0.5
    stats = S.distill_step(L, idx, lp, temperature=temp, tail=tail, weight=w.cuda())
    torch.cuda.synchronize()
    assert int(T.err.cpu()[0]) == 0 and int(S.err.cpu()[0]) == 0
    idx, lp, stats = idx.cpu().numpy(), lp.cpu().numpy(), stats.cpu().numpy()
    # the teacher: log-probs in descending order, each that of its token, none larger left out
    z = M.target_logits(case.merged, Wt, mt) / temp
    ref = z - np.log(np.exp(z - z.max(1, keepdims=True)).sum(1, keepdims=True)) - z.max(1, keepdims=True)
    tol = 1e-4 if f32 else 2e-2
    assert (np.diff(lp, axis=1) <= 0).all()
    assert np.abs(lp - np.take_along_axis(ref, idx.astype(np.int64), 1)).max() < tol
    rest = ref.copy()
    np.put_along_axis(rest, idx.astype(np.int64), -np.inf, 1)
    assert (rest.max(1) <= lp[:, -1] + tol).all()
    assert all(len(set(r)) == k for r in idx)
    # the student on the same lists
    want = M.distill_update(case.merged, Ws, ms, idx, lp, tail, 1.0 / temp, w.numpy())
    assert stats[1] == L.n_mask
    assert abs(stats[0] - want["loss"]) <= (1e-4 if f32 else 1e-2) * abs(want["loss"])
    for key, ref_g in want["grads"].items():
        got = S.G[key].cpu().numpy()
        assert rel_l2(got, ref_g) < (1e-4 if f32 else 1e-2), (key, rel_l2(got, ref_g))
        if not f32:
            assert cosine(got, ref_g) >= 0.999, key


def test_teacher_is_the_student():
    """Full attention on both sides and a tail: the loss is the rounding of the lists, and the
    gradient against that of another teacher next to nothing."""
    from paper_2606_04484_amd import actor
    case = Case(workload(TINY))
    L = actor.merge(actor.upload_timelines(case.tl, case.old))
    A = actor.ActorUpdate(case.m, case.device_weights())
    idx, lp = A.teacher_topk(L, 16)
    A.zero_grads()
    loss = A.distill_step(L, idx, lp)
    small = {k: g.clone() for k, g in A.G.items()}
    A.zero_grads()
    other = A.distill_step(L, idx.roll(1, 0).contiguous(), lp.roll(1, 0).contiguous())
    torch.cuda.synchronize()
    # (random weights are near uniform: other rows' lists cost 0.004.)  Sums of float32
    # probabilities: 16 roundings of 2^-24 each, in the loss twice (p and 1 - sum p)
    assert abs(float(loss[0])) < 1e-5 and float(other[0]) > 1e-3
    for k, g in A.G.items():
        assert float(small[k].norm()) < 1e-3 * float(g.norm()), k


def test_update_with_adapters_and_after_a_step():
    """LoRA on a windowed student: only the adapters get a gradient, that of the merged weights'
    chain rule; and policy-gradient and distillation steps of one object do not disturb each other."""
    from paper_2606_04484_amd import actor
    m = dataclasses.replace(TINY, window=24, n_sink=2)
    case = Case(workload(TINY))
    lora = make_lora_numpy(m, rank=8, seed=5, b_std=0.05)
    L = actor.merge(actor.upload_timelines(case.tl, case.old))
    T = actor.ActorUpdate(case.m, case.device_weights())
    idx, lp = T.teacher_topk(L, 12)
    A = actor.ActorUpdate(m, case.device_weights(), lora=case.device_weights(which=lora), lora_rank=8, lora_scale=0.5)
    A.zero_grads()
    A.step(L)
    torch.cuda.synchronize()
    first = {k: g.clone() for k, g in A.G.items()}
    A.zero_grads()
    A.distill_step(L, idx, lp)
    torch.cuda.synchronize()
    W = M.lora_effective(case.W, lora, 0.5, m)
    want = M.distill_update(case.merged, W, m, idx.cpu().numpy(), lp.cpu().numpy(), True)["grads"]
    for proj in ("w_qkv", "w_o", "w_gate_up", "w_down"):
        a, b = lora[f"lora_a.{proj}"].astype(np.float64), lora[f"lora_b.{proj}"].astype(np.float64)
        dw = want[proj]
        assert rel_l2(A.G[f"lora_a.{proj}"].cpu().numpy(), 0.5 * b.T @ dw) < 1e-4, proj
        assert rel_l2(A.G[f"lora_b.{proj}"].cpu().numpy(), 0.5 * dw @ a.T) < 1e-4, proj
    A.zero_grads()
    A.step(L)
    torch.cuda.synchronize()
    for k, g in A.G.items():
        assert torch.equal(g, first[k]), k


def test_weights_of_another_layout_are_refused_before_any_work():
    from paper_2606_04484_amd import actor, capi
    case = Case(workload(TINY))
    L = actor.merge(actor.upload_timelines(case.tl, case.old), pack_tokens=700)
    A = actor.ActorUpdate(case.m, case.device_weights())
    A.zero_grads()
    idx, lp = A.teacher_topk(L, 8)
    with pytest.raises(capi.AjError, match="weight"):
        A.distill_step(L, idx, lp, weight=torch.ones(L.n_mask - 1, device="cuda"))
    with pytest.raises(capi.AjError, match="lists"):
        A.distill_step(L, idx[1:], lp[1:])
    torch.cuda.synchronize()
    assert all(not bool(g.any()) for g in A.G.values())
