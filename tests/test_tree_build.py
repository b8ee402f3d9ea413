"""The generated gfx950 code of the kernels for drafted trees (CPU only: hipcc cross-compiles the device code to assembly)."""
import os
import re
import subprocess

import pytest

from paper_2503_16257_amd import build as B


@pytest.mark.parametrize("src,kernels", [("cache8_tree.hip", 36), ("cache8_append.hip", 4), ("tree.hip", 13)])
def test_no_kernel_spills_vector_registers(src, kernels, tmp_path):
    """Nor touches scratch memory (scalar registers that are spilled go to lanes of a vector register)."""
    flags = [f for f in B.FLAGS if f not in ("-fPIC", "-Wall", "-Wno-unused-function")]
    out = tmp_path / "k.s"
    r = subprocess.run([B._hipcc(), *flags, "-w", "-S", "--cuda-device-only", os.path.join(B.CSRC, src), "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    text = out.read_text()
    found = re.findall(r"\.name:\s+(\S+).*?\.vgpr_spill_count:\s+(\d+)", text, re.S)
    assert len(found) == kernels and all(f[1] == "0" for f in found), found
    assert not re.search(r"^\s+scratch_", text, re.M)
