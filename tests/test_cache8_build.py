"""The generated gfx950 code of the 8-bit cache's kernels (CPU only: hipcc cross-compiles the device code to assembly)."""
import os
import re
import subprocess

import pytest

from paper_2503_16257_amd import build as B


@pytest.mark.parametrize("src,kernels", [("cache8_attn.hip", 18), ("cache8.hip", 14), ("rotary.hip", 6)])
def test_no_kernel_spills_vector_registers(src, kernels, tmp_path):
    """(The many-query kernel's 48 rows a wave take all but two of the 256 that two waves a SIMD leave it.)"""
    flags = [f for f in B.FLAGS if f not in ("-fPIC", "-Wall", "-Wno-unused-function")]
    out = tmp_path / "k.s"
    r = subprocess.run([B._hipcc(), *flags, "-w", "-S", "--cuda-device-only", os.path.join(B.CSRC, src), "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    found = re.findall(r"\.name:\s+(\S+).*?\.private_segment_fixed_size:\s+(\d+).*?\.vgpr_spill_count:\s+(\d+)", out.read_text(), re.S)
    assert len(found) == kernels and all(f[1:] == ("0", "0") for f in found), found
