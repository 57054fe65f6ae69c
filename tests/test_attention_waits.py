"""Results of matrix instructions are waited for on every way through the attention kernels (no GPU needed)."""
import os
import subprocess

import pytest

import mfma_waits
from paper_2605_00422_amd import build

FILES = ["attention_split.hip", "attention_tile.hip", "attention_tile_f32.hip", "attention_weights.hip"]


@pytest.mark.parametrize("name", FILES)
def test_results_of_matrix_instructions_are_waited_for(tmp_path, name):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    out = str(tmp_path / "kernels.s")
    subprocess.run([build.HIPCC, *build.FLAGS, "-w", "-S", "--cuda-device-only", "-o", out, os.path.join(build.CSRC, name)], check=True,
                   stderr=subprocess.DEVNULL)
    found = 0
    for kernel, body in mfma_waits.kernels(open(out).read().split("\n")):
        found += 1
        early = mfma_waits.early_reads(body)
        assert not early, (kernel, early[:3])
    assert found
