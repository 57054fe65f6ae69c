"""Results of matrix instructions are waited for on every way through the kernels, with ways told apart at each branch (no GPU needed): the
follower itself, and the rotations' kernels."""
import os
import subprocess

import pytest

import mfma_waits
from paper_2605_00422_amd import build

# What lies between a product and the reading of its result may be another product here, which waits for the unit.  (The attention's kernels are
# followed in test_attention_waits.py and test_attention8_asm.py, by the compiler's rule.)
FILES = ["rotate_quant.hip", "rotate_terms.hip", "rotate_terms_many.hip", "rotate_terms_f32.hip"]


def test_what_a_branch_skips_does_not_count_as_waiting():
    """With a label in front of it or without: a block that is entered from above alone has none."""
    ahead = ["v_mfma_f32_32x32x16_f16 v[0:15], v[16:19], v[20:23], 0", "s_cbranch_scc0 .LBB0_2"]
    long, read = ["v_add_f32_e32 v30, v31, v31"] * 20, [".LBB0_2:", "v_max_f32_e32 v30, v3, v3", "s_endpgm"]
    for label in (".LBB0_1:", "; %bb.1:"):
        assert mfma_waits.early_reads(ahead + [label] + long + read)
        assert not mfma_waits.early_reads(ahead[:1] + ["s_nop 11"] + ahead[1:] + [label] + long + read)


def test_a_product_that_reads_another_ones_result_as_an_operand():
    ahead, nops = ["v_mfma_f32_16x16x32_f16 v[0:3], v[16:19], v[20:23], 0"], ["s_nop 7"]
    for operands, early in (("v[0:3], v[20:23], v[4:7]", True), ("v[20:23], v[0:3], v[4:7]", True), ("v[16:19], v[20:23], v[0:3]", False)):
        last = [f"v_mfma_f32_16x16x32_f16 v[0:3], {operands}", "s_endpgm"]
        assert bool(mfma_waits.early_reads(ahead + last)) == early and not mfma_waits.early_reads(ahead + nops + last)


def test_a_product_in_between_waits_for_the_unit():
    two = ["v_mfma_f32_16x16x32_f16 v[0:3], v[16:19], v[20:23], 0", "v_mfma_f32_16x16x32_f16 v[4:7], v[16:19], v[20:23], 0"]
    read = ["v_max_f32_e32 v30, v3, v3", "s_endpgm"]
    for n, early in ((3, False), (2, True)):           # 8 states: 4 passes, n + 1 others
        assert bool(mfma_waits.early_reads(two + [f"s_nop {n}"] + read, busy=True)) == early
    assert mfma_waits.early_reads(two + ["s_nop 3"] + read) and not mfma_waits.early_reads(two + ["s_nop 6"] + read)


@pytest.mark.parametrize("name", FILES)
def test_results_of_matrix_instructions_are_waited_for(tmp_path, name):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    out = str(tmp_path / "kernels.s")
    subprocess.run([build.HIPCC, *build.FLAGS, *build.FILE_FLAGS.get(name, []), "-w", "-S", "--cuda-device-only", "-o", out,
                    os.path.join(build.CSRC, name)], check=True, stderr=subprocess.DEVNULL)
    found = 0
    for kernel, body in mfma_waits.kernels(open(out).read().split("\n")):
        found += 1
        early = mfma_waits.early_reads(body, busy=True)
        assert not early, (kernel, early[:3])
    assert found
