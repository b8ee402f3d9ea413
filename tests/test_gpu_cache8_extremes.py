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


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_what_is_not_finite(dtype, code):
    """Infinities as the type's largest number, NaN as zero: a NaN leaves its block's other tokens as they are."""
    r = np.random.default_rng(82)
    inf, nan = float("inf"), float("nan")
    for numbers in ([nan, -nan], [inf, -inf], [nan, inf, -inf, 65504.0]):
        c = Pair(2, 192, code)
        for start, n in ((0, 40), (40, 1), (41, 1), (42, 100)):
            print(f"[case] not finite {numbers} {n} at {start}", flush=True)
            clean = torch.from_numpy(r.standard_normal((1, 2, n, 128))).to(dtype).to(DEV)
            some = with_some(r, (1, 2, n, 128), dtype, numbers)
            c.write(some, clean, start)
        c.check()
        c = Pair(2, 192, code)
        for start, n in ((0, 40), (40, 1), (41, 100)):
            c.write(torch.zeros((1, 2, n, 128), dtype=dtype, device=DEV), with_some(r, (1, 2, n, 128), dtype, numbers), start)
        c.check()
        c.write(torch.full((1, 2, 32, 128), nan, dtype=dtype, device=DEV), torch.full((1, 2, 32, 128), nan, dtype=dtype, device=DEV), 160)
        c.check()


@pytest.mark.parametrize("n,every", [(3, 1), (70, 1), (70, 5)])
def test_keys_that_overflow_when_they_are_turned(n, every):
    """A pair of 65504 turned by an eighth is beyond fp16: the rotation by itself leaves infinities (no pair has both where
    every fifth element is so large), and the cache is the same as after it."""
    plan = vk.make_rotary((64,), freq=[0.7853981633974483] * 64)
    r = np.random.default_rng(83)
    K, V = (with_some(r, (1, 2, n, 128), F16, [65504.0], every=every) for _ in range(2))
    pos = torch.arange(n, device=DEV, dtype=torch.int32)[None, None]
    Kt = torch.empty_like(K)
    vk.rotary(plan, pos, K, Kt)
    assert torch.isinf(Kt).any() == (every == 1)
    a, b = Pair(2, 128, 1), Pair(2, 128, 1)
    a.write(Kt, V, 0)
    a.check()
    vk.cache8_write(b.p, 0, b.buf, K, V, i32([0]), rotary=plan, positions=pos)
    assert torch.equal(a.buf, b.buf)


@pytest.mark.parametrize("rep,n", [(2, 20), (7, 40)])
def test_a_token_that_is_not_finite_stays_with_the_queries_that_see_it(rep, n):
    """Causal queries before it give the same bits as without it."""
    r = np.random.default_rng(84)
    for cap, T in ((96, 90), (4096, 4090)):
        for dtype in (F16, BF16):
            outs = []
            at = T - n + 12                                # the token of query 12
            K, V = (torch.from_numpy(r.standard_normal((1, 1, T, 128))).to(dtype).to(DEV) for _ in range(2))
            q = torch.from_numpy(r.standard_normal((1, rep, n, 128))).to(dtype).to(DEV)
            for bad in (0.0, float("nan")):
                p = vk.make_cache8(1, 1, 1, rep, cap, 1)
                buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
                K[:, :, at, ::3] = bad
                V[:, :, at, ::3] = bad
                vk.cache8_write(p, 0, buf, K, V, i32([0]))
                out = torch.empty_like(q)
                vk.cache8_attention(p, 0, buf, q, out, i32([T]), vk.alloc_bytes(vk.cache8_workspace_bytes(p, n), DEV))
                outs.append(out)
            assert torch.isfinite(outs[1]).all() and torch.equal(*outs)
