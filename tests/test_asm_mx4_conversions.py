"""Static check of the 6-bit conversions of queries (CPU only).

v_cvt_scalef32_2xpk16_fp6_f32 and v_cvt_scalef32_pk32_f32_fp6 work in several passes: where the
result lies in the registers of an operand, later passes read what earlier ones wrote (a low half of
a query whose scale was overwritten was wrong).  The compiler does not keep them apart by itself, so
in the gfx950 assembly of every kernel that uses them none may overlap.
"""
import os
import re
import shutil
import subprocess

import pytest

from tests.test_asm_lds_reads import CSRC, HIPCC, ROOT


def _registers(text):
    """The vector registers of each operand."""
    spans = []
    for m in re.finditer(r"\bv(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
        lo = int(m[1] or m[3])
        spans.append(set(range(lo, int(m[2] or lo) + 1)))
    return spans


def _overlaps(lines):
    bad, seen = [], 0
    for line in lines:
        line = line.split(";")[0].strip()
        if not re.match(r"v_cvt_scalef32_(2xpk16_fp6_f32|pk32_f32_fp6)\b", line):
            continue
        seen += 1
        result, *operands = _registers(line.split(None, 1)[1])
        if any(result & x for x in operands):
            bad.append(line)
    return seen, bad


def test_the_scan_sees_an_overlap():
    good = "\tv_cvt_scalef32_2xpk16_fp6_f32 v[134:139], v[2:17], v[34:49], v18"
    bad = "\tv_cvt_scalef32_2xpk16_fp6_f32 v[18:23], v[2:17], v[34:49], v18"
    also = "\tv_cvt_scalef32_pk32_f32_fp6 v[2:33], v[30:35], v83"
    assert _overlaps([good, "\tv_mov_b32_e32 v1, v1"]) == (1, [])
    assert _overlaps([good, bad, also]) == (3, [bad.strip(), also.strip()])


@pytest.mark.parametrize("name", ["attn_mx4", "attn_mx4_rows"])
def test_no_conversion_overwrites_its_operands(tmp_path, name):
    if not os.path.exists(HIPCC) and not shutil.which("hipcc"):
        pytest.skip("hipcc not available")
    out = tmp_path / f"{name}.s"
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC",
                    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    f"-I{os.path.join(ROOT, 'include')}", "--cuda-device-only", "-S",
                    os.path.join(CSRC, f"{name}.hip"), "-o", str(out)], check=True, capture_output=True)
    seen, bad = _overlaps(open(out))
    assert seen >= 36 and not bad, (seen, bad)
