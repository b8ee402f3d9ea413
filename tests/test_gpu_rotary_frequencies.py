"""Frequencies of the caller's own: an image encoder's, which begin anew with each axis, and any others.

Tolerance as for the library's own frequencies: cos and sin to 5 u (u = 2^-24), y = x1 cos - x2 sin to 8 u (|x1| + |x2|), half a
step of the type; the frequency's own 2^-64 of a turn times the position are beyond all that."""
import numpy as np
import pytest
import torch

from oracle import cache8 as O
from paper_2503_16257_amd import binding as vk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("d,dtype,n", [(80, torch.float32, 257), (64, torch.bfloat16, 1), (128, torch.float16, 333)])
def test_frequencies_that_begin_anew_with_each_axis(d, dtype, n, inverse):
    print(f"[case] own frequencies d={d} n={n} {dtype} inverse={inverse}", flush=True)
    r = np.random.default_rng(91)
    pairs = d // 2
    each = pairs // 2
    freq = [10000.0 ** (-i / each) for i in range(each)] * 2
    freq[1], freq[2] = -3.0, 0.0                          # backwards; not at all
    plan = vk.make_rotary((each, pairs - each), head_dim=d, freq=freq)
    pos = r.integers(0, 5000, (2, 2, n)).astype(np.int32)
    x = torch.from_numpy(r.standard_normal((2, 6, n, d))).to(dtype).to(DEV)
    y = torch.empty_like(x)
    vk.rotary(plan, torch.from_numpy(pos).to(DEV), x, y, inverse=inverse)
    x64 = x.double().cpu().numpy()
    ref = O.rotary(x64, pos, (each, pairs - each), rot_dim=d, inverse=inverse, freq=freq)
    s = np.abs(x64[..., :pairs]) + np.abs(x64[..., pairs:])
    tol = 8 * 2.0 ** -24 * np.concatenate([s, s], -1) + 1.0001 * torch.finfo(dtype).eps / 2 * np.abs(ref) + (2.0 ** -25 if dtype == torch.float16 else 1e-37)
    err = np.abs(y.double().cpu().numpy() - ref)
    assert (err <= tol).all(), (err / tol).max()
