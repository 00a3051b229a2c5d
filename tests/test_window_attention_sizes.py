"""Sizes past what a launch takes, refused on the host before any work."""
import ctypes as C

import pytest

from paper_2606_04484_amd import capi

P16 = C.c_void_p(16)


@pytest.mark.parametrize("n_tok, heads", [((1 << 30) - 1023, 1), (1 << 30, 1), (1 << 28, 16)])
def test_tokens_past_a_launch(n_tok, heads):
    L = capi.lib()
    cfg, vl = C.byref(capi.AttnCfg(heads, 1, 8, 16, 2, 0, 0.0)), C.byref(capi.Varlen(n_tok, 1, 10, 0, P16, None))
    assert L.aj_attention_fwd(cfg, vl, P16, P16, P16, P16, 1 << 60, None) == 2
    assert L.aj_attention_bwd(cfg, vl, P16, P16, P16, P16, P16, P16, 1 << 60, None) == 2
