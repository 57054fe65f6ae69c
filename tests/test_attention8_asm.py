"""Structural checks of the compiled kernels of the 8-bit cache (no GPU needed): MFMA takes no notice of the execution mask, so none may lie
in a region that the compiler entered by narrowing the mask without a jump around it; and what becomes of codes is counted."""
import os
import re
import subprocess

import pytest

from paper_2605_00422_amd import build

FILES = ["attention8_split.hip", "attention8_split_f32.hip", "attention8_tile.hip", "attention8_tile_f32.hip"]


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
def test_codes_become_halves_without_a_detour(asm, name):
    """e4m3 codes by the conversion of pairs, integers by permutes and a packed addition: no conversions of single codes to fp32."""
    text = "\n".join(asm[name])
    assert "v_cvt_scalef32_pk_f16_fp8" in text and "v_pk_add_f16" in text
    assert "v_cvt_f32_fp8" not in text
    assert "v_pk_fma_f32" not in text and "v_pk_mul_f32" not in text and "v_pk_add_f32" not in text
