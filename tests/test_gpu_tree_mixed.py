"""Attention of trees whose rows are some tiles of 192 and a rest of up to 128: the workgroups of the rest have tiles and splits of
their own.  For 256 compute units these shapes are shared out so: rests of 39, 116, 64 and 120 rows, one or two tiles a wave.
Tolerance: that of test_gpu_tree.py."""
import pytest
import torch

from test_gpu_tree import Case, trees, words

pytestmark = pytest.mark.gpu
F16, BF16 = torch.float16, torch.bfloat16

# counts that end in the whole tile, in the rest, just in front of it and behind its first node, at none
SHAPES = [
    (4, 4, 7, 33, 4096, [4096, 3000, 0, 17], [33, 20, 29, 0], (0, 19, 26, 27, 28, 32)),
    (4, 4, 7, 33, 4096, [32, 4096, 4095, 2000], None, (0, 27, 28, 32)),
    (4, 4, 7, 44, 4096, [1, 4096, 0, 3333], [44, 27, 0, 30], (0, 26, 27, 28, 29, 43)),
    (4, 4, 7, 44, 4096, [4096, 100, 4064, 0], [28, 44, 44, 44], (0, 27, 28, 43)),
    (1, 1, 7, 256, 8192, [8000], None, (0, 27, 28, 246, 247, 255)),
    (1, 1, 7, 256, 8192, [8191], [130], (0, 54, 55, 128, 129)),
    (1, 2, 7, 72, 16384, [16384], None, (0, 54, 55, 71)),
    (1, 2, 7, 72, 16384, [9999], [40], (0, 27, 39)),
]


@pytest.mark.parametrize("code,dtype", [(0, F16), (1, F16), (0, BF16), (1, BF16)])
@pytest.mark.parametrize("B,H,rep,n,cap,lens,counts,rows", SHAPES)
def test_whole_tiles_and_a_rest(B, H, rep, n, cap, lens, counts, rows, code, dtype):
    print(f"[case] tiles and a rest B={B} H={H} n={n} cap={cap} lens={lens} counts={counts} code={code} {dtype}", flush=True)
    c = Case(B, H, rep, n, cap, lens, code, dtype, n + cap + code, strided=bool(n % 2))
    sees = trees(B, n, n + 1)
    masks = words(sees)
    first = c.run(masks, counts)
    c.check(first, sees, counts, rows=rows)
    c.ws.fill_(0x11)                                             # (partials of splits that the rest does not have are written too)
    assert torch.equal(c.run(masks, counts), first)


@pytest.mark.parametrize("code,dtype", [(0, F16), (1, BF16)])
def test_any_mask_over_tiles_and_a_rest(code, dtype):
    """Masks that are no tree's, rows of nothing among them, over caches of nothing and of much."""
    import numpy as np
    r = np.random.default_rng(8)
    c = Case(4, 4, 7, 44, 4096, [0, 4000, 0, 50], code, dtype, 77, L=2, layer=1)
    sees = [r.random((44, 44)) < 0.3 for _ in range(4)]
    for s in sees:
        s[::3] = False
    c.check(c.run(words(sees), [44, 44, 30, 44]), sees, [44, 44, 30, 44], rows=(0, 1, 26, 27, 28, 42, 43))
