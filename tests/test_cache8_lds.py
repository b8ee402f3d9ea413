"""LDS of the attention's kernels (CPU only: hipcc cross-compiles the device code to assembly)."""
import os
import re
import subprocess

from paper_2503_16257_amd import build as B


def lds(src, out):
    flags = [f for f in B.FLAGS if f not in ("-fPIC", "-Wall", "-Wno-unused-function")]
    r = subprocess.run([B._hipcc(), *flags, "-w", "-S", "--cuda-device-only", os.path.join(B.CSRC, src), "-o", str(out)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    return {n: int(b) for b, n in re.findall(r"\.group_segment_fixed_size:\s+(\d+).*?\.name:\s+(\S+)", out.read_text(), re.S)}


def test_without_a_tree_there_is_no_room_for_one(tmp_path):
    """Many queries: two blocks' operands, 32 KB; a tree's first block 16 KB more and its masks, where it waits in LDS."""
    got = {n: b for n, b in lds("cache8_attn.hip", tmp_path / "a.s").items() if "c8_many_kernel" in n}
    assert len(got) == 6 and set(got.values()) == {32768}, got
    tree = lds("cache8_tree.hip", tmp_path / "t.s")
    for nt, want in ((1, 49152 + 2 * 4 * 1 * 64), (2, 49152 + 2 * 4 * 2 * 64), (3, 32768 + 2 * 4 * 3 * 64)):
        got = {n: b for n, b in tree.items() if f"c8_tree_many_kernelILi{nt}E" in n}
        assert len(got) == 4 and set(got.values()) == {want}, got
