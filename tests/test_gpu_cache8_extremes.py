"""What large and non-finite numbers become in the 8-bit cache, byte for byte against the float64 oracle."""
import numpy as np
import pytest
import torch

from oracle import cache8 as O
from paper_2503_16257_amd import binding as vk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16 = torch.float16, torch.bfloat16


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def as_held(t):
    """The numbers that a tensor's elements enter a block as: an infinity as the type's largest, a NaN as zero."""
    big = torch.finfo(t.dtype).max
    return torch.nan_to_num(t.double(), nan=0.0, posinf=big, neginf=-big).cpu().numpy()


class Pair:
    """A cache and the oracle's."""

    def __init__(self, H, cap, code):
        self.p = vk.make_cache8(1, 1, H, H, cap, code)
        self.buf = vk.alloc_bytes(vk.cache8_bytes(self.p), DEV)
        self.buf.fill_(0xFF)
        self.geom, self.code = (1, 1, H, cap), code
        self.want = [a.copy() for a in O.unpack(self.buf.cpu().numpy(), *self.geom)]

    def write(self, K, V, start, **kw):
        vk.cache8_write(self.p, 0, self.buf, K, V, i32([start]), **kw)
        for x, c, m in ((K, self.want[0], self.want[2]), (V, self.want[1], self.want[3])):
            O.write(as_held(x)[0], start, x.shape[2], c[0, 0], m[0, 0], self.code)

    def check(self):
        for name, g, w in zip(("K codes", "V codes", "K magnitudes", "V magnitudes"), O.unpack(self.buf.cpu().numpy(), *self.geom),
                              self.want):
            np.testing.assert_array_equal(g.view(np.uint8), w.view(np.uint8), err_msg=name)


def with_some(r, shape, dtype, numbers, every=97):
    x = torch.from_numpy(r.standard_normal(shape)).to(dtype)
    flat = x.view(-1)
    at = torch.arange(3, flat.numel(), every)
    flat[at] = torch.tensor(numbers, dtype=dtype).repeat(len(at))[:len(at)]
    return x.to(DEV)


@pytest.mark.parametrize("code", [0, 1])
def test_the_largest_bfloat16(code):
    """Beyond 2^40, where the magnitude is held, and beyond 2^128 / 127, whose product with the level leaves float's range:
    the largest codes, with their signs."""
    r = np.random.default_rng(81)
    big = torch.finfo(BF16).max
    numbers = [3e38, -3e38, 2.0 ** 40, -2.0 ** 41, 2.7e36, -2.8e36, 7e35, -8e35, big, -big, 1e12]
    c = Pair(3, 160, code)
    for start, n in ((0, 1), (1, 70), (71, 33), (104, 1)):
        print(f"[case] largest {n} at {start}, code {code}", flush=True)
        c.write(with_some(r, (1, 3, n, 128), BF16, numbers), with_some(r, (1, 3, n, 128), BF16, numbers[::-1], every=311), start)
    c.check()
