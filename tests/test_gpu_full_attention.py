"""aj_attention_fwd / _bwd without a window on packs of long segments (256 rows and more on
average, where the causal kernels run with the entry point's own scratch and parts) against the
definition in 64 bits, and on both sides of that size."""
import pytest
import torch

from test_gpu_window_attention import call, check
from window_attention import reference

pytestmark = pytest.mark.gpu

CASES = [
    # lens, hq, hkv, hd
    ([600, 300], 4, 2, 64),
    ([600, 300], 4, 2, 128),
    ([257], 2, 1, 64),
    ([1500], 7, 1, 128),                  # parts of a group's heads
    ([1111, 1, 900], 6, 1, 64),
    ([0, 1300, 0, 700], 2, 2, 128),       # segments of no tokens
    ([256, 256], 4, 1, 64),               # the last size of short segments
    ([257, 257], 4, 1, 64),               # the first of long ones
    ([900, 1200], 2, 1, 32),
    ([700], 3, 3, 96),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("lens, hq, hkv, hd", CASES)
def test_matches_definition(lens, hq, hkv, hd, dtype):
    qkv, dout, got = call(lens, hq, hkv, hd, 0, 0, dtype, seed=5)
    check(got, reference(qkv, lens, hq, hkv, hd, 0, 0, dout, bf16=dtype == torch.bfloat16))


def test_a_long_segment_among_empty_ones():
    """The average counts segments of no tokens: another kernel, the same definition."""
    lens = [0] * 20 + [1200] + [0] * 20
    qkv, dout, got = call(lens, 4, 2, 64, 0, 0, torch.bfloat16, seed=5)
    check(got, reference(qkv, lens, 4, 2, 64, 0, 0, dout, bf16=True))
