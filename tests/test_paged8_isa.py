"""Checks on the gfx950 assembly of the 8-bit paged cache's kernels: no registers spilled, no
packed float32 instruction, no load that the compiler could only address generically (whose
wait holds up all others), and e4m3 pairs widened by the conversion that keeps them exact."""

import os
import re
import shutil
import subprocess

import pytest

from paper_2511_14694_amd import build as B

KERNELS = {"paged_attend.hip": 17, "paged_append.hip": 14, "paged_extend.hip": 3}


@pytest.mark.parametrize("source", sorted(KERNELS))
def test_kernels_as_compiled(source, tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc is not available")
    out = tmp_path / "k.s"
    subprocess.run([hipcc, *B.HIPCC_FLAGS, *B.EXTRA_FLAGS.get(source, []), "--cuda-device-only", "-S",
                    os.path.join(B.CSRC, source), "-o", str(out)], check=True, capture_output=True)
    text = out.read_text()
    scratch = re.findall(r"^; ScratchSize: (\d+)", text, re.M)
    assert len(scratch) >= KERNELS[source] and set(scratch) == {"0"}
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text)
    assert not re.search(r"\bflat_load", text)
    if source == "paged_attend.hip":
        assert "v_cvt_scalef32_pk_bf16_fp8" in text
        for m in re.finditer(r"v_cvt_scalef32_pk_bf16_fp8 \S+ \S+ (\S+)", text):
            assert m.group(1) == "1.0"
