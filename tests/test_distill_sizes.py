"""The sizes that the top-k and distillation calls answer and take, at their ends; on the host."""
import ctypes as C

import pytest

from paper_2606_04484_amd import capi

CFG = capi.LossCfg(64, 151936, 1 << 14, 0.2, 1e-6, 1, 0)


@pytest.mark.parametrize("k", [257, 4096, 4097, 5000, 2 ** 31 - 1])
@pytest.mark.parametrize("rows", [0, 1, 4, 1023, 1024, 100000])
def test_workspace_of_a_list_too_long(rows, k):
    """No size, and no end of the process, for a k that the calls refuse."""
    assert capi.aj_topk_workspace_bytes(rows, 151936, k) == 0
    assert capi.aj_distill_workspace_bytes(rows, 151936, k) == 0
    assert capi.aj_lm_head_workspace_bytes(CFG, rows, k) == 0


@pytest.mark.parametrize("rows", [1, 4, 1023, 1024, 100000])
@pytest.mark.parametrize("vocab", [1, 300, 151936, 1 << 24])
def test_workspace_of_the_longest_list(rows, vocab):
    assert capi.aj_topk_workspace_bytes(rows, vocab, 256) >= capi.aj_topk_workspace_bytes(rows, vocab, 1) > 0
    assert capi.aj_distill_workspace_bytes(rows, vocab, 256) > 0
