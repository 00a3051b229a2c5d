"""Calls of the teacher's and the student's operators that their documentation allows, or that
they refuse, beyond ordinary batches."""
import pytest
import torch

from tests.gpu_cases import Case, workload
from workloads import get_config

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [0, 257, 5000])
def test_lists_of_a_length_that_is_refused(k):
    """Before any work, whatever the length."""
    from paper_2606_04484_amd import actor, capi
    case = Case(workload(get_config(0).model))
    L = actor.merge(actor.upload_timelines(case.tl, case.old))
    A = actor.ActorUpdate(case.m, case.device_weights())
    A.zero_grads()
    with pytest.raises(capi.AjError, match="lists of"):
        A.teacher_topk(L, k)
    idx = torch.zeros(L.n_mask, k, dtype=torch.int32, device="cuda")
    with pytest.raises(capi.AjError, match="lists of"):
        A.distill_step(L, idx, idx.float())
    torch.cuda.synchronize()
    assert all(not bool(g.any()) for g in A.G.values())
