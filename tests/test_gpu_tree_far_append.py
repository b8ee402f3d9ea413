"""Appending to a cache of more than 2^33 bytes writes the blocks that the path reaches, and nothing else."""
import pytest
import torch

from paper_2503_16257_amd import binding as vk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("code,dtype", [(0, torch.float16), (1, torch.bfloat16)])
def test_nothing_but_the_paths_blocks_is_written(code, dtype):
    """4 layers of 8 heads x 2^20 tokens, 8.6 GB; the path's five nodes go into the last block, and into two blocks far from both ends."""
    L, H, cap, n = 4, 8, 1 << 20, 9
    p = vk.make_cache8(L, 1, H, H, cap, code)
    heads, nbc = L * H, cap // 32
    buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
    buf.fill_(0x21)
    assert buf.numel() > 1 << 33
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    K, V = (torch.randn((L, 1, H, n, 128), generator=g, device=DEV).to(dtype) for _ in range(2))
    path = torch.tensor([[8, 0, 3, 3, 7, -1, -1, -1, -1]], dtype=torch.int32, device=DEV)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    codes = heads * nbc * 4096
    parts = [buf[:codes].view(heads, nbc, 4096), buf[codes:2 * codes].view(heads, nbc, 4096),
             buf[2 * codes:2 * codes + heads * nbc * 4].view(heads, nbc, 4), buf[2 * codes + heads * nbc * 4:].view(heads, nbc, 4)]
    reached = set()
    for start, blocks in ((cap - 5, {nbc - 1}), (700030, {700030 // 32, 700030 // 32 + 1}), (cap, set()), (-1, set())):
        vk.cache8_append_path(p, buf, K, V, path, i32(5), i32(start))
        reached |= blocks
        other = torch.ones(nbc, dtype=torch.bool, device=DEV)
        other[list(reached)] = False
        for part in parts:
            changed = torch.zeros(nbc, dtype=torch.bool, device=DEV)
            for h in range(heads):
                changed |= (part[h] != 0x21).any(dim=1)
            assert not changed[other].any(), start
            assert not reached or changed[~other].all()
    # and the tokens are there, in every layer
    back = torch.empty((1, H, 5, 128), device=DEV)
    for layer in range(L):
        for x, at in ((K, 0), (V, 1)):
            vk.cache8_read(p, layer, buf, i32(700030), *([None] * at), back, *([None] * (1 - at)))
            want = x[layer][:, :, [8, 0, 3, 3, 7]].float()
            # each block's magnitude is at most that of the tokens in it; 0x21212121 as a float, 5e-19, holds none of them up
            a = torch.stack([want[:, :, :2].abs().amax(dim=(2, 3)), want[:, :, 2:].abs().amax(dim=(2, 3))])
            a = a.repeat_interleave(torch.tensor([2, 3], device=DEV), dim=0).permute(1, 2, 0)[..., None]
            step = a * (0.5 / 127) if code == 0 else want.abs() * 2.0 ** -4 + a * 2.0 ** -10 / 448
            assert ((back - want).abs() <= step * 1.0001).all(), layer
