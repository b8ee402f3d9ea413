"""LDS and scratch memory of the 8-bit cache's and the trees' kernels (CPU only: hipcc cross-compiles the device code to assembly)."""
import concurrent.futures as cf
import os
import re
import subprocess

import pytest

from paper_2503_16257_amd import build as B

SOURCES = {"cache8_attn.hip": 18, "cache8_tree.hip": 36, "cache8_append.hip": 4, "tree.hip": 13}


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """Of each source: kernel -> (bytes of LDS, bytes of a thread's private segment)."""
    d = tmp_path_factory.mktemp("isa")
    flags = [f for f in B.FLAGS if f not in ("-fPIC", "-Wall", "-Wno-unused-function")]

    def one(src):
        out = d / (src + ".s")
        r = subprocess.run([B._hipcc(), *flags, "-w", "-S", "--cuda-device-only", os.path.join(B.CSRC, src), "-o", str(out)],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-2000:]
        return {n: (int(b), int(p)) for b, n, p in re.findall(
            r"\.group_segment_fixed_size:\s+(\d+).*?\.name:\s+(\S+).*?\.private_segment_fixed_size:\s+(\d+)", out.read_text(), re.S)}
    with cf.ThreadPoolExecutor(max_workers=4) as ex:
        return dict(zip(SOURCES, ex.map(one, SOURCES)))


def test_without_a_tree_there_is_no_room_for_one(kernels):
    """Many queries: two blocks' operands, 32 KB; a tree's first block 16 KB more and its masks, where it waits in LDS."""
    got = {n: b[0] for n, b in kernels["cache8_attn.hip"].items() if "c8_many_kernel" in n}
    assert len(got) == 6 and set(got.values()) == {32768}, got
    for nt, want in ((1, 49152 + 2 * 4 * 1 * 64), (2, 49152 + 2 * 4 * 2 * 64), (3, 32768 + 2 * 4 * 3 * 64)):
        got = {n: b[0] for n, b in kernels["cache8_tree.hip"].items() if f"c8_tree_many_kernelILi{nt}E" in n}
        assert len(got) == 4 and set(got.values()) == {want}, got


@pytest.mark.parametrize("src", SOURCES)
def test_no_kernel_has_scratch_memory_set_up(kernels, src):
    """Not even where nothing touches it: a dispatch with a private segment makes the runtime provide for it."""
    assert len(kernels[src]) == SOURCES[src]
    assert {n: b[1] for n, b in kernels[src].items() if b[1]} == {}
