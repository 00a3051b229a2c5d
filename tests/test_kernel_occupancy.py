"""A windowed attention kernel keeps as many waves on a SIMD as its causal twin: what it has
besides (masks, the way over rows that are not finite) is not to cost registers in the main
loop.  Read from the compiler's resource remarks for the library's own build options."""
import os
import re
import subprocess

import pytest

from paper_2606_04484_amd import build

SRC = "attention_mfma.hip"


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="hipcc not installed")
def test_windowed_kernels_keep_their_waves(tmp_path):
    r = subprocess.run([build.HIPCC, *build.FLAGS, *build.FILE_FLAGS[SRC], "-x", "hip",
                        "--offload-device-only", "-Rpass-analysis=kernel-resource-usage", "-c",
                        os.path.join(build.CSRC, SRC), "-o", str(tmp_path / "x.o")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    waves = {k: int(v) for k, v in re.findall(r"Function Name: (\S+).*?Occupancy \[waves/SIMD\]: (\d+)", r.stderr, re.S)}
    pairs = 0
    for name, n in waves.items():
        if "ELi4ELb1E" in name:          # <head_dim, 4 waves, window>
            twin = waves[name.replace("ELi4ELb1E", "ELi4ELb0E")]
            assert n >= twin, (name, n, twin)
            pairs += 1
    assert pairs == 6                    # forward, dQ, dK/dV at head_dim 64 and 128
