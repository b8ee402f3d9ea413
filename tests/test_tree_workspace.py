"""The tree attention's workspace: what the size query says is taken, and a call's sums have one order whatever more there is."""
import ctypes as C
import random

import pytest
import torch

from paper_2503_16257_amd import binding as vk

A = 0x10000                                                # a 256-aligned address


def refused_for_space(p, n, size):
    """Whether a tree of n nodes finds `size` bytes too few (else it goes on to a launch, which ends without a device)."""
    v = C.byref(vk.VidkvView(A, 1 << 20, 128, 1 << 16, 0))
    st = vk.lib().vidkv_cache8_tree_attention(C.byref(p), 0, n, v, v, v, A, A, 1 << 62, A, None, v, A, size, None)
    assert st in (vk.ENOSPACE, vk.EHIP), st
    return st == vk.ENOSPACE


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls would launch")
def test_every_tree_fits_what_was_asked_for():
    r = random.Random(9)
    for _ in range(3000):
        shape = (r.choice([1, 2, 3, 4, 8, 9, 16, 33, 64]), r.choice([1, 2, 4, 8]), r.choice([1, 2, 4, 7, 8, 13]), 32 * int(2 ** r.uniform(0, 12.5)))
        p, n = vk.make_cache8(shape[0], *shape[:2], shape[1] * shape[2], shape[3]), r.randint(1, 256)
        size = vk.cache8_workspace_bytes(p, n)
        assert not refused_for_space(p, n, size), (shape, n)
        assert not refused_for_space(p, n, vk.cache8_workspace_bytes(p, 256)), (shape, n)


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls would launch")
def test_a_tree_with_more_splits_than_the_attention_has_refuses_less_than_its_own():
    """Such a plan does not shrink to what there is: its sums would have another order.  (4 sequences of 4 x 7 heads over 8192 tokens,
    33 nodes: 17 splits where the attention of as many queries has 9.)"""
    for shape, n in (((4, 4, 28, 8192), 33), ((1, 4, 28, 16384), 33)):
        p = vk.make_cache8(1, *shape)
        size, row = vk.cache8_workspace_bytes(p, n), shape[0] * shape[2] * n * 130 * 4
        lo, hi = 0, size                                   # the least that is taken
        while hi - lo > 1:
            mid = (lo + hi) // 2
            lo, hi = (mid, hi) if refused_for_space(p, n, mid) else (lo, mid)
        splits = (hi - 256) // row
        assert splits > 1 and hi == -(-splits * row // 256) * 256 + 256 and hi <= size
        v = C.byref(vk.VidkvView(A, 1 << 20, 128, 1 << 16, 0))
        attention = vk.lib().vidkv_cache8_attention(C.byref(p), 0, n, 0, v, A, 1 << 62, A, None, v, A, hi - 1, None)
        assert attention == vk.EHIP and refused_for_space(p, n, hi - 1)


@pytest.mark.gpu
@pytest.mark.parametrize("code,dtype", [(0, torch.float16), (1, torch.bfloat16)])
@pytest.mark.parametrize("B,H,rep,n,cap,lens,counts", [
    (4, 4, 7, 33, 8192, [8192, 5000, 0, 33], [33, 20, 33, 0]), (1, 4, 7, 33, 16384, [16000], None), (3, 2, 2, 150, 8192, [8000, 1, 4100], None)])
def test_a_larger_workspace_leaves_the_bits_as_they_are(B, H, rep, n, cap, lens, counts, code, dtype):
    """Sizes where more splits would be cheaper than the size query has room for; each result against the oracle."""
    from test_gpu_tree import Case, trees, words
    print(f"[case] workspace B={B} H={H} rep={rep} n={n} cap={cap} code={code}", flush=True)
    c = Case(B, H, rep, n, cap, lens, code, dtype, n + cap)
    sees = trees(B, n, n)
    masks, first = words(sees), None
    size = vk.cache8_workspace_bytes(c.p, n)
    for more in (0, 4096, vk.cache8_workspace_bytes(c.p, 256) - size, size, 1 << 28):
        c.ws = torch.full((size + more,), 0xFF, dtype=torch.uint8, device="cuda:0")
        out = c.run(masks, counts)
        if first is None:
            first = out
            c.check(out, sees, counts, rows=(0, 17, n - 1))
        assert torch.equal(out, first), more
        assert (c.ws[size:] == 0xFF).all()
