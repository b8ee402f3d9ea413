"""Rotary positions on the GPU against the float64 oracle.

Tolerance (u = 2^-24).  The angle's turn is exact to 2^-33 (position times a 64-bit turn, top 32 bits of what is left of
the nearest quarter); as a float, times the constant, it is off by 3 u of at most pi/4, and the Taylor sums by what they
leave out (1.8e-9) and two roundings of numbers of at most 1: cos and sin to 5 u.  y = x1 cos - x2 sin adds two roundings:
8 u (|x1| + |x2|), then half a step of the result's type (of fp16 at least half of its smallest, 2^-25)."""
import numpy as np
import pytest
import torch

from oracle import cache8 as O
from paper_2503_16257_amd import binding as vk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def bound(x, y, dtype, rot_dim, adjacent):
    z = np.abs(x[..., :rot_dim])
    if adjacent:
        s = np.repeat(z[..., 0::2] + z[..., 1::2], 2, axis=-1)
    else:
        s = np.concatenate([z[..., :rot_dim // 2] + z[..., rot_dim // 2:]] * 2, axis=-1)
    b = np.zeros(x.shape)
    b[..., :rot_dim] = 8 * 2.0 ** -24 * s + torch.finfo(dtype).eps / 2 * np.abs(y[..., :rot_dim]) * 1.0001
    return b + (2.0 ** -25 if dtype == F16 else 1e-37)


def tokens(r, shape, dtype, strided=False):
    x = torch.from_numpy(r.standard_normal(shape)).to(dtype).to(DEV)
    return x.transpose(1, 2).contiguous().transpose(1, 2) if strided else x


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("B,Hq,Hk,n,d,rot,sections,adjacent,dtype,strided,far", [
    (1, 28, 4, 1, 128, 128, (16, 24, 24), False, F16, False, 0),
    (2, 28, 4, 197, 128, 128, (16, 24, 24), False, BF16, True, 0),
    (3, 7, 1, 333, 128, 128, (16, 24, 24), True, F16, False, 0),
    (64, 4, 4, 1, 128, 96, (48,), False, BF16, False, 100000),
    (2, 16, 16, 129, 80, 80, (20, 20), False, F32, False, 0),
    (1, 3, 2, 70, 80, 64, (10, 10, 12), True, F32, True, 0),
    (2, 2, 1, 33, 256, 256, (32, 32, 32, 32), False, F16, True, 0),
    (1, 1, 1, 5, 16, 16, (8,), False, F32, False, 2 ** 31 - 5),
    (1, 2, 1, 4, 128, 16, (0, 8), True, BF16, False, -2 ** 31),
    (1, 28, 4, 9000, 128, 128, (16, 24, 24), False, F16, True, 196000),
])
@pytest.mark.parametrize("inverse", [False, True])
def test_matches_oracle(B, Hq, Hk, n, d, rot, sections, adjacent, dtype, strided, far, inverse):
    print(f"[case] rotary B={B} Hq={Hq} n={n} d={d} rot={rot} {dtype} inverse={inverse}", flush=True)
    r = np.random.default_rng(B * 1000 + n)
    plan = vk.make_rotary(sections, theta=1.0e6, head_dim=d, rot_dim=rot, adjacent=adjacent)
    pos = (far + r.integers(0, 5 if far else 3000, (len(sections), B, n))).astype(np.int32)
    q, k = tokens(r, (B, Hq, n, d), dtype, strided), tokens(r, (B, Hk, n, d), dtype, strided)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    vk.rotary(plan, torch.from_numpy(pos).to(DEV), q, qo, k, ko, inverse=inverse)
    for x, y in ((q, qo), (k, ko)):
        hs = sorted({0, x.shape[1] // 2, x.shape[1] - 1})               # (first, middle and last head; extended precision is slow)
        ref = O.rotary(f64(x[:, hs]), pos, sections, 1.0e6, rot, adjacent, inverse)
        err = np.abs(f64(y[:, hs]) - ref)
        b = bound(f64(x[:, hs]), ref, dtype, rot, adjacent)
        assert (err <= b).all(), (err / b).max()
        assert torch.isfinite(y).all()
        np.testing.assert_array_equal(f64(y)[..., rot:], f64(x)[..., rot:])
    # in place: the same bits; and queries or keys alone
    q2, k2 = q.clone(), k.clone()
    p = torch.from_numpy(pos).to(DEV)
    vk.rotary(plan, p, q2, q2, inverse=inverse)
    vk.rotary(plan, p, None, None, k2, k2, inverse=inverse)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)


def test_broadcast_and_backward_strides():
    """Inputs may repeat an axis (stride 0) or run backwards."""
    r = np.random.default_rng(3)
    plan = vk.make_rotary((16, 24, 24))
    base = tokens(r, (1, 1, 6, 128), F16)
    pos = torch.from_numpy(r.integers(0, 99, (3, 2, 6)).astype(np.int32)).to(DEV)
    x = base.expand(2, 5, 6, 128)
    y, z = torch.empty((2, 5, 6, 128), dtype=F16, device=DEV), torch.empty((2, 5, 6, 128), dtype=F16, device=DEV)
    vk.rotary(plan, pos, x, y)
    vk.rotary(plan, pos, x.contiguous(), z)
    assert torch.equal(y, z)


def test_gradient():
    """y = R x is linear: <g, R(x + h e) - R(x - h e)> / 2h = (R^T g)_e, and R^T g is the inverse rotation of g.  In float32,
    with x, g of N(0, 1) and h = 1: a difference of two sums that the rotation's own error, 8 u (|x1| + |x2|) an element,
    and one rounding of each product enter."""
    r = np.random.default_rng(4)
    plan = vk.make_rotary((4, 6, 6), head_dim=32)
    pos = torch.from_numpy(r.integers(0, 5000, (3, 1, 4)).astype(np.int32)).to(DEV)
    x, g = tokens(r, (1, 2, 4, 32), F32), tokens(r, (1, 2, 4, 32), F32)
    back = torch.empty_like(g)
    vk.rotary(plan, pos, g, back, inverse=True)

    def f(v):
        y = torch.empty_like(v)
        vk.rotary(plan, pos, v, y)
        return y.double()
    for h, t, c in ((0, 0, 0), (1, 3, 31), (0, 2, 15), (1, 1, 16), (0, 3, 7)):
        e = torch.zeros_like(x)
        e[0, h, t, c] = 1.0
        diff = (g.double() * (f(x + e) - f(x - e))).sum().item() / 2
        tol = 2 * 8 * 2.0 ** -24 * (g.abs()[0, h, t].sum().item() * (x.abs()[0, h, t].max().item() + 1) * 2)
        assert abs(diff - back[0, h, t, c].item()) <= tol, (diff, back[0, h, t, c].item())
    ref = O.rotary(f64(g), pos.cpu().numpy(), (4, 6, 6), inverse=True)
    assert (np.abs(f64(back) - ref) <= bound(f64(g), ref, F32, 32, False)).all()


def test_refusals_of_the_binding():
    r = np.random.default_rng(5)
    plan = vk.make_rotary((16, 24, 24))
    x = tokens(r, (2, 3, 4, 128), F16)
    pos = torch.zeros((3, 2, 4), dtype=torch.int32, device=DEV)
    for bad in (pos[:2], pos.long(), pos[:, :, :3], pos.cpu()):
        with pytest.raises((TypeError, ValueError)):
            vk.rotary(plan, bad, x, x.clone())
    for bad in (x.double(), x[0], x[..., :64], x.transpose(2, 3), x[..., ::2]):
        with pytest.raises((TypeError, ValueError)):
            vk.rotary(plan, pos, bad, bad)
    with pytest.raises(ValueError):                          # written to where elements overlap
        vk.rotary(plan, pos, x, x[:, :1].expand(2, 3, 4, 128))
    with pytest.raises(vk.VidkvError):                       # not 16-byte aligned
        y = torch.empty(2 * 3 * 4 * 128 + 8, dtype=F16, device=DEV)[1:1 + 2 * 3 * 4 * 128].view(2, 3, 4, 128)
        vk.rotary(plan, pos, x, y)
    with pytest.raises(vk.VidkvError):
        vk.rotary(plan, pos, x, torch.empty((2, 3, 4, 128), dtype=BF16, device=DEV))
    vk.rotary(plan, pos[:, :, :0].contiguous(), x[:, :, :0], x[:, :, :0])                # nothing to do
