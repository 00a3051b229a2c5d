"""Calls of the teacher's and the student's operators that their documentation allows, or that
they refuse, beyond ordinary batches."""
import pytest
import torch

from test_gpu_distill import test_many_long_rows as many_long_rows
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


@pytest.mark.parametrize("tail", [False, True], ids=["listed", "tail"])
@pytest.mark.parametrize("dtype, grad", [("f32", "bf16"), ("bf16", "bf16")])
@pytest.mark.parametrize("vocab, k, pad, offset", [(45056, 30, 0, 0), (73728, 9, 5, 3), (196592, 16, 0, 0),
                                                   (196593, 64, 1, 0), (262144, 33, 3, 5), (270320, 8, 0, 0),
                                                   (270321, 5, 0, 1)])
def test_ends_of_the_ranges_of_long_rows(vocab, k, pad, offset, dtype, grad, tail):
    """A workgroup's share of a row, at the sizes where the ways of forming its gradient change."""
    many_long_rows(vocab, k, pad, offset, dtype, grad, tail)
