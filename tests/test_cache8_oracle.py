"""CPU: the oracle of the rotary positions and the 8-bit cache against other arithmetic, and the entry points' refusals
and size functions (host checks; the pointers are addresses that nothing follows)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import cache8 as O
from paper_2503_16257_amd import binding as vk

A = 0x10000                                                # a 256-aligned address


def test_e4m3_codes_against_torch():
    t = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(np.isnan(t), np.isnan(O.e4m3_values()))
    ok = ~np.isnan(t)
    np.testing.assert_array_equal(t[ok], O.e4m3_values()[ok])
    r = np.concatenate([np.linspace(-448, 448, 20001), t[ok], 2.0 ** -10 * np.arange(-40, 41)])
    got = O.byte_of(r, 1)
    want = torch.from_numpy(r).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(O.value_of(got, 1), O.value_of(want, 1))


def test_int8_codes_round_half_to_even():
    np.testing.assert_array_equal(O.value_of(O.byte_of(np.array([0.5, 1.5, -0.5, -2.5, 126.5, 200, -200]), 0), 0),
                                  [0, 2, 0, -2, 126, 127, -127])


def test_rotary_is_a_rotation():
    r = np.random.default_rng(1)
    x = r.standard_normal((2, 3, 5, 32))
    pos = r.integers(0, 100, (3, 2, 5))
    for adjacent in (False, True):
        y = O.rotary(x, pos, [4, 6, 6], adjacent=adjacent)
        np.testing.assert_allclose((y ** 2).sum(-1), (x ** 2).sum(-1), rtol=1e-13)
        np.testing.assert_allclose(O.rotary(y, pos, [4, 6, 6], adjacent=adjacent, inverse=True), x, atol=1e-13)
    z = x[..., :16] + 1j * x[..., 16:]
    f = 10000.0 ** (-np.arange(16) / 16)
    axis = np.repeat([0, 1, 2], [4, 6, 6])
    z = z * np.exp(1j * pos[axis].transpose(1, 2, 0)[:, None] * f)
    np.testing.assert_allclose(O.rotary(x, pos, [4, 6, 6]), np.concatenate([z.real, z.imag], -1), atol=1e-12)


@pytest.mark.parametrize("code", [0, 1])
def test_write_in_pieces(code):
    """Error of a value: half a step of its block's last magnitude, and of each smaller one that it was coded under."""
    r = np.random.default_rng(2)
    x = r.standard_normal((2, 70, 128)) * np.exp(r.standard_normal((2, 70, 1)))
    b, m = np.full((2, 96, 128), 0x5A, np.uint8), np.ones((2, 3))
    at = 0
    for n in (1, 1, 30, 5, 33):
        O.write(x[:, at:], at, n, b, m, code)
        at += n
    assert (b[:, 70:] == 0x5A).all()                        # behind the last token: as it was
    got = O.values(b, m, code)[:, :70]
    big = np.repeat(np.abs(np.pad(x, ((0, 0), (0, 26), (0, 0)))).reshape(2, 3, -1).max(-1), 32, 1)[:, :70, None]
    # int8: at most four codings of a token (pieces 1, 1, 30 share a block; the second block is written twice)
    step = big / 127 if code == 0 else np.maximum(np.abs(x) * 2.0 ** -3, big * 2.0 ** -9 / 448 * 2)
    assert (np.abs(got - x) <= 3 * 0.5 * step * 1.1).all()


def test_turns_are_the_frequencies():
    rot = vk.make_rotary((16, 24, 24), theta=1.0e6)
    for i in range(64):
        f = np.longdouble(1.0e6) ** (-np.longdouble(i) / 64) / (2 * np.arccos(np.longdouble(-1)))
        assert abs(int(rot.turn[i]) - int(f * np.longdouble(2) ** 64)) <= 2 ** 4, i        # a long double's last bits
    assert list(rot.axis[:64]) == [0] * 16 + [1] * 24 + [2] * 24
    rot = vk.make_rotary((8,), head_dim=32, rot_dim=16, freq=[-1.0, 0.0, 2 * math.pi, 1e9, 1, 1, 1, 1])
    assert rot.turn[1] == 0 and min(rot.turn[2], 2 ** 64 - rot.turn[2]) < 2 ** 14        # 2 pi is a turn, to a double's bits
    assert abs(rot.turn[0] + rot.turn[4] - 2 ** 64) <= 1


def test_rotary_init_refuses():
    L, r = vk.lib(), vk.VidkvRotary()
    def init(d=128, rd=128, adj=0, sec=(16, 24, 24), theta=1e6, rot=C.byref(r), axes=None, freq=None):
        s = (C.c_int32 * 8)(*sec) if sec is not None else None
        return L.vidkv_rotary_init(rot, d, rd, adj, len(sec or ()) if axes is None else axes, s, theta, freq)
    assert init() == vk.OK
    assert init(rot=None) == vk.EINVAL and init(sec=None, axes=3) == vk.EINVAL
    for d, rd in ((0, 0), (8, 8), (136, 136), (272, 272), (128, 144), (128, 0), (128, 24)):
        assert init(d=d, rd=rd) == vk.ESHAPE
    assert init(axes=0) == vk.ESHAPE and init(axes=5) == vk.ESHAPE
    assert init(sec=(16, 24, 23)) == vk.EINVAL and init(sec=(16, 24, 25)) == vk.EINVAL and init(sec=(-1, 65)) == vk.EINVAL
    assert init(sec=(2 ** 31 - 1, 1)) == vk.EINVAL
    assert init(adj=2) == vk.EINVAL and init(theta=0.0) == vk.EINVAL and init(theta=math.inf) == vk.EINVAL
    assert init(theta=math.nan) == vk.EINVAL
    assert init(freq=(C.c_double * 64)(*([math.nan] * 64))) == vk.EINVAL
    with pytest.raises(ValueError):
        vk.make_rotary((64,), freq=[1.0] * 63)


def view(data=A, b=512, h=128, n=256, dtype=0):
    return C.byref(vk.VidkvView(data, b, h, n, dtype))


def test_rotary_apply_refuses():
    L = vk.lib()
    rot = vk.make_rotary((16, 24, 24))
    def call(rot=C.byref(rot), inv=0, B=1, n=2, pos=A, hq=2, q=view(), qo=view(), hk=0, k=None, ko=None):
        return L.vidkv_rotary_apply(rot, inv, B, n, pos, hq, q, qo, hk, k, ko, None)
    assert call(B=0) == vk.OK and call(n=0) == vk.OK and call(hq=0) == vk.OK              # nothing to do
    assert call(rot=None) == vk.EINVAL and call(pos=None) == vk.EINVAL and call(pos=A + 2) == vk.EINVAL
    assert call(q=None) == vk.EINVAL and call(qo=None) == vk.EINVAL and call(k=view()) == vk.EINVAL
    assert call(inv=2) == vk.EINVAL and call(B=-1) == vk.EINVAL and call(n=-1) == vk.EINVAL and call(hq=-1) == vk.EINVAL
    assert call(B=1 << 16, n=1 << 16) == vk.ESHAPE and call(B=1, n=(1 << 26) + 1) == vk.ESHAPE and call(hq=65536) == vk.ESHAPE
    assert call(hq=40000, hk=40000, k=view(), ko=view()) == vk.ESHAPE
    for bad in (view(data=A + 8), view(data=None), view(b=4), view(h=129), view(n=2), view(dtype=3), view(n=1 << 60)):
        assert call(q=bad) == vk.EINVAL and call(qo=bad) == vk.EINVAL
    assert call(qo=view(dtype=1)) == vk.EINVAL and call(hk=1, k=view(dtype=2), ko=view(dtype=2)) == vk.EINVAL
    for name, v in (("head_dim", 120), ("rot_dim", 160), ("adjacent", 2), ("n_axes", 2), ("n_axes", 0)):
        other = vk.make_rotary((16, 24, 24))
        setattr(other, name, v)                                  # (two axes: the pairs of the third have no row)
        assert call(rot=C.byref(other)) == vk.EINVAL, name


def test_cache8_sizes():
    def size(L=1, B=1, H=4, Hq=28, cap=64, code=0, **kw):
        p = vk.make_cache8(L, B, H, Hq, cap, code)
        for k, v in kw.items():
            setattr(p, k, v)
        return vk.cache8_bytes(p)
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    for L, B, H, cap in ((1, 1, 1, 32), (28, 8, 4, 12544), (1, 64, 4, 25088), (3, 5, 2, 96)):
        nb = L * B * H * cap // 32
        assert size(L, B, H, H * 2, cap) == 2 * nb * 4096 + 2 * up(nb * 4)
    for kw in (dict(cap=33), dict(cap=0), dict(Hq=27), dict(Hq=0), dict(B=0), dict(L=0), dict(H=0), dict(code=2),
               dict(code=-1), dict(head_dim=64), dict(B=65536), dict(H=65536, Hq=65536)):
        assert size(**kw) == 0, kw
    assert size(L=2 ** 31 - 1, B=65535, H=65535, Hq=65535, cap=2 ** 31 - 32) == 0          # more than there can be
    p = vk.make_cache8(1, 2, 4, 28, 6272)
    for n in (1, 2, 5, 196, 6272):
        assert vk.cache8_workspace_bytes(p, n) >= 256
    assert vk.cache8_workspace_bytes(p, 0) == 0 and vk.cache8_workspace_bytes(p, -1) == 0
    assert vk.cache8_workspace_bytes(p, 2 ** 31 - 1) == 0
    assert size(cap=2 ** 28) > 0 and size(cap=2 ** 28 + 32) == 0
    assert vk.lib().vidkv_cache8_bytes(None) == 0


@pytest.mark.parametrize("B,H,rep,cap", [(1, 4, 7, 98208), (1, 1, 1, 1568), (3, 2, 8, 6016), (64, 4, 7, 25088), (1, 1, 48, 640)])
def test_a_workspace_for_many_queries_holds_fewer(B, H, rep, cap):
    """(More rows can mean fewer splits, and smaller partials.)"""
    p = vk.make_cache8(1, B, H, H * rep, cap)
    sizes = [vk.cache8_workspace_bytes(p, n) for n in range(1, 400)]
    assert sizes == sorted(sizes)
    assert vk.cache8_workspace_bytes(p, 10 ** 6) >= sizes[-1]


def test_cache8_calls_refuse():
    L = vk.lib()
    p = vk.make_cache8(2, 1, 4, 28, 64)
    big, need = 1 << 40, vk.cache8_bytes(p)
    rot = vk.make_rotary((16, 24, 24))
    half = vk.make_rotary((16, 16), head_dim=64)

    def write(p=C.byref(p), layer=0, n=2, K=view(), V=view(), start=A, count=None, rot=None, pos=None, c=A, cb=big):
        return L.vidkv_cache8_write(p, layer, n, K, V, start, count, rot, pos, c, cb, None)
    def read(p=C.byref(p), layer=0, n=2, start=A, c=A, cb=big, K=view(), V=view()):
        return L.vidkv_cache8_read(p, layer, n, start, c, cb, K, V, None)
    def attend(p=C.byref(p), layer=0, n=2, causal=1, q=view(), c=A, cb=big, length=A, count=None, out=view(), ws=A, wb=big):
        return L.vidkv_cache8_attention(p, layer, n, causal, q, c, cb, length, count, out, ws, wb, None)

    assert write(n=0) == vk.OK and read(n=0) == vk.OK and attend(n=0) == vk.OK            # nothing to do
    for call in (write, read, attend):
        assert call(p=None) == vk.EINVAL and call(c=None) == vk.EINVAL and call(c=A + 16) == vk.EINVAL
        assert call(layer=2) == vk.EINVAL and call(layer=-1) == vk.EINVAL and call(n=-1) == vk.EINVAL
        assert call(cb=need - 1) == vk.ENOSPACE
        bad = vk.make_cache8(2, 1, 4, 28, 65)
        assert call(p=C.byref(bad)) == vk.ESHAPE
    for bad in (view(data=A + 8), view(data=None), view(b=4), view(h=129), view(n=2), view(dtype=5)):
        assert write(K=bad) == vk.EINVAL and write(V=bad) == vk.EINVAL and read(K=bad) == vk.EINVAL
        assert read(V=bad) == vk.EINVAL and attend(q=bad) == vk.EINVAL and attend(out=bad) == vk.EINVAL
    assert write(K=None) == vk.EINVAL and write(V=None) == vk.EINVAL and write(V=view(dtype=1)) == vk.EINVAL
    assert write(K=view(dtype=2), V=view(dtype=2)) == vk.EINVAL                              # keys of 32 bits
    assert write(start=None) == vk.EINVAL and write(start=A + 2) == vk.EINVAL and write(count=A + 1) == vk.EINVAL
    assert write(rot=C.byref(rot)) == vk.EINVAL and write(pos=A) == vk.EINVAL
    assert write(rot=C.byref(half), pos=A) == vk.EINVAL and write(rot=C.byref(rot), pos=A + 2) == vk.EINVAL
    assert read(start=None) == vk.EINVAL and read(K=None, V=None) == vk.EINVAL and read(K=view(dtype=2)) == vk.EINVAL
    assert attend(q=None) == vk.EINVAL and attend(out=None) == vk.EINVAL and attend(out=view(dtype=1)) == vk.EINVAL
    assert attend(q=view(dtype=2), out=view(dtype=2)) == vk.EINVAL
    assert attend(length=None) == vk.EINVAL and attend(length=A + 2) == vk.EINVAL and attend(count=A + 2) == vk.EINVAL
    assert attend(causal=2) == vk.EINVAL and attend(ws=None) == vk.EINVAL and attend(ws=A + 16) == vk.EINVAL
    assert attend(wb=vk.cache8_workspace_bytes(p, 2) - 1) == vk.ENOSPACE
    assert attend(n=2 ** 31 - 1) == vk.ESHAPE and write(n=2 ** 28 + 1) == vk.ESHAPE and read(n=2 ** 28 + 1) == vk.ESHAPE
    wide = vk.make_cache8(1, 65535, 65535, 65535, 32)                       # more workgroups than a grid holds
    assert attend(p=C.byref(wide), n=2 ** 20, cb=1 << 62) == vk.ESHAPE
    for scale in (0.0, -1.0, math.nan, math.inf):
        odd = vk.make_cache8(2, 1, 4, 28, 64, softmax_scale=scale)
        assert attend(p=C.byref(odd)) == vk.EINVAL


def test_binding_refuses_host_tensors():
    x = torch.zeros((1, 2, 3, 128), dtype=torch.float16)
    rot = vk.make_rotary((64,))
    p = vk.make_cache8(1, 1, 2, 2, 32)
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        vk.rotary(rot, torch.zeros((1, 1, 3), dtype=torch.int32), x, x)
    with pytest.raises(ValueError):
        vk.rotary(rot, i, None, None)
    with pytest.raises(TypeError):
        vk.cache8_write(p, 0, torch.zeros(8, dtype=torch.uint8), x, x, i)
    with pytest.raises(TypeError):
        vk.cache8_read(p, 0, torch.zeros(8, dtype=torch.uint8), i, x, x)
    with pytest.raises(TypeError):
        vk.cache8_attention(p, 0, torch.zeros(8, dtype=torch.uint8), x, x, i, torch.zeros(256, dtype=torch.uint8))


def test_odd_arguments_are_left_to_the_python_path():
    """The native call layer takes plain arguments that pass, and no others."""
    vk.lib()
    n = vk._native
    assert n.rotary(*[None] * 9) is None and n.rotary(1) is None
    assert n.cache8_write(*[None] * 11) is None and n.cache8_read(*[None] * 8) is None
    assert n.cache8_attention(*[None] * 11) is None
    with pytest.raises(TypeError):
        n.bind8(1, 2)
    x = torch.zeros((1, 2, 3, 128), dtype=torch.float16)
    i = torch.zeros(1, dtype=torch.int32)
    u = torch.zeros(4096, dtype=torch.uint8)
    rot, p = vk.make_rotary((64,)), vk.make_cache8(1, 1, 2, 2, 32)
    pos = torch.zeros((1, 1, 3), dtype=torch.int32)
    for r in (rot, bytes(C.sizeof(vk.VidkvRotary)), p):                      # host tensors; foreign structures
        assert n.rotary(r, pos, x, x, None, None, False, vk._stream, None) is None
    for c in (p, bytes(C.sizeof(vk.VidkvCache8)), rot):
        assert n.cache8_write(c, 0, u, x, x, i, None, rot, pos, vk._stream, None) is None
        assert n.cache8_write(c, 0, u, x, x, i, None, None, None, vk._stream, None) is None
        assert n.cache8_read(c, 0, u, i, x, None, vk._stream, None) is None
        assert n.cache8_attention(c, 0, u, x, x, i, u, None, True, vk._stream, None) is None
