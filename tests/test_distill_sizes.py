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


P16 = C.c_void_p(16)


@pytest.mark.parametrize("rows, vocab", [(1 << 24, 1), ((1 << 24) - 1, 65530), (1 << 16, 1 << 24), ((1 << 31) - 1, 100)])
def test_rows_past_a_launch(rows, vocab):
    """Rows for which a launch has not threads enough are refused before any work."""
    L = capi.lib()
    lg = C.byref(capi.Logits(rows, vocab, vocab, 0, 1.0, P16))
    t = C.byref(capi.Teacher(1, 1, P16, P16, None, 1.0))
    big = 1 << 60
    assert L.aj_topk_logprob(lg, 1, P16, P16, P16, P16, big, None) == 2
    assert L.aj_distill_loss_fwd(lg, t, P16, P16, None, None, P16, big, None) == 2
    assert L.aj_distill_loss_bwd(lg, t, P16, P16, vocab, 0, None) == 2
    assert L.aj_distill_loss_fwd_bwd(lg, t, P16, P16, None, None, P16, vocab, 0, P16, big, None) == 2


@pytest.mark.parametrize("d, v, dtype", [(64, 72, 0), (1536, 151936, 1), (3584, 152064, 1), (128, 1024, 0), (64, 8, 1)])
def test_workspace_of_the_teacher_alone(d, v, dtype):
    """Less than the student's, and as that one enough for fewer targets."""
    cfg = capi.LossCfg(d, v, 1 << 14, 0.2, 1e-6, dtype, 0)
    for k in (1, 8, min(v, 256)):
        sizes = [capi.aj_lm_head_topk_workspace_bytes(cfg, n, k) for n in range(1, 9000, 7)]
        assert sizes == sorted(sizes) and sizes[0] > 0
        both = [capi.aj_lm_head_workspace_bytes(cfg, n, k) for n in range(1, 9000, 7)]
        assert both == sorted(both) and all(a <= b for a, b in zip(sizes, both))
    for n in (1, 8192, 20000):
        teacher, student = (q(cfg, n, 8) for q in (capi.aj_lm_head_topk_workspace_bytes,
                                                   capi.aj_lm_head_workspace_bytes))
        # no d hidden, and with bfloat16 no d logits
        assert student - teacher >= 4 * n * d + (2 * min(n, 8192) * v if dtype else 0) - (1 << 20)
    assert capi.aj_lm_head_topk_workspace_bytes(cfg, 4, 257) == 0
