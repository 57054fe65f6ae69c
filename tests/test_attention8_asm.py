"""Structural checks of the compiled kernels of the 8-bit cache (no GPU needed): MFMA takes no notice of the execution mask, so none may lie
in a region that the compiler entered by narrowing the mask without a jump around it; and what becomes of codes is counted."""
import os
import re
import subprocess

import pytest

import mfma_waits
from paper_2605_00422_amd import build

FILES = ["attention8_split.hip", "attention8_split_f32.hip", "attention8_tile.hip", "attention8_tile_e4m3.hip", "attention8_tile_f32.hip",
         "attention8_tile_f32_e4m3.hip"]


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not available")
    tmp = tmp_path_factory.mktemp("asm")
    jobs = [(f, str(tmp / (f + ".s"))) for f in FILES]
    runs = [subprocess.Popen([build.HIPCC, *build.FLAGS, "-w", "-S", "--cuda-device-only", "-o", out, os.path.join(build.CSRC, f)],
                             stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL) for f, out in jobs]
    assert all(r.wait() == 0 for r in runs)
    return {f: open(out).read().split("\n") for f, out in jobs}


@pytest.mark.parametrize("name", FILES)
def test_no_mfma_under_a_narrowed_mask(asm, name):
    lines = [l.split(";")[0].strip() for l in asm[name]]
    lines = [l for l in lines if l and not l.startswith(".") or re.match(r"\.LBB", l)]
    assert any(l.startswith("v_mfma") for l in lines)
    for i, l in enumerate(lines):
        if "saveexec" not in l or any("s_cbranch_execz" in x for x in lines[i + 1:i + 4]):
            continue
        for x in lines[i + 1:]:
            if re.match(r"s_(or|mov|andn2|xor)_b64 exec", x) or x.startswith("s_endpgm"):
                break
            assert not x.startswith("v_mfma"), (name, i, l, x)


@pytest.mark.parametrize("name", FILES)
def test_results_of_matrix_instructions_are_waited_for(asm, name):
    found = 0
    for kernel, body in mfma_waits.kernels(asm[name]):
        found += 1
        early = mfma_waits.early_reads(body)
        assert not early, (kernel, early[:3])
    assert found >= 12


def test_an_early_read_is_found():
    """The way around a branch that may be skipped counts, and so does a loop's way back."""
    ahead = ["v_mfma_f32_32x32x16_f16 v[0:15], v[16:19], v[20:23], 0", "s_cbranch_scc0 .LBB0_2"]
    long = [".LBB0_1:"] + ["v_add_f32_e32 v30, v31, v31"] * 20
    assert mfma_waits.early_reads(ahead + long + [".LBB0_2:", "v_max_f32_e32 v30, v3, v3", "s_endpgm"])
    assert not mfma_waits.early_reads(ahead + long + [".LBB0_2:", "s_nop 11", "v_max_f32_e32 v30, v3, v3", "s_endpgm"])
    assert not mfma_waits.early_reads(ahead[:1] + long + [".LBB0_2:", "v_max_f32_e32 v30, v3, v3", "s_endpgm"])
    loop = [".LBB0_1:", "v_add_f32_e32 v30, v4, v4", "v_mfma_f32_16x16x32_f16 v[4:7], v[16:19], v[20:23], v[4:7]", "s_cbranch_scc0 .LBB0_1", "s_endpgm"]
    assert mfma_waits.early_reads(loop) and not mfma_waits.early_reads(loop[:3] + ["s_nop 6"] + loop[3:])


@pytest.mark.parametrize("name", FILES)
def test_codes_become_halves_without_a_detour(asm, name):
    """e4m3 codes by the conversion of pairs, integers by permutes and a packed addition: no conversions of single codes to fp32."""
    text = "\n".join(asm[name])
    both = "split" in name
    assert ("v_cvt_scalef32_pk_f16_fp8" in text) == (both or "e4m3" in name) and ("v_pk_add_f16" in text) == (both or "e4m3" not in name)
    assert "v_cvt_f32_fp8" not in text
    assert "v_pk_fma_f32" not in text and "v_pk_mul_f32" not in text and "v_pk_add_f32" not in text
