"""The same distances as in test_mfma_hazards, around the inline-asm MFMAs of the
video kernel's forms for 8-bit pages and token windows."""
import os
import subprocess

from paper_2607_04443_amd import _build
from test_mfma_hazards import hazards


def test_no_hazard_around_the_inline_asm_mfmas(tmp_path):
    out = tmp_path / "video_paths.asm"
    subprocess.run([_build._hipcc()] + _build.HIP_FLAGS + ["-x", "hip", "--offload-device-only", "-S",
                   os.path.join(_build.CSRC, "video_paths.hip"), "-o", str(out)], check=True, capture_output=True)
    n, found = hazards(out.read_text())
    assert n > 1000, n  # (three wave widths in three kernels)
    assert not found, found[:5]
