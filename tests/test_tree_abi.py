"""The calls for trees of drafted tokens refuse what they cannot take before anything is launched (no GPU here: the
addresses are made up and never looked at)."""
import ctypes as C
import math
import os

import pytest
import torch

from paper_2503_16257_amd import binding as vk

A = 0x10000                                                # a 256-aligned address
BIG = 1 << 40


def view(data=A, b=1 << 16, h=1 << 10, n=128, dtype=0):
    return C.byref(vk.VidkvView(data, b, h, n, dtype))


def rows(data=A, b=3000, r=1000, dtype=2):
    return C.byref(vk.VidkvRows(data, b, r, dtype))


def masks(B=1, n=5, parent=A, count=None, mask=A, axes=3, base=A, pos=A):
    return vk.lib().vidkv_tree_masks(B, n, parent, count, mask, axes, base, pos, None)


def test_masks_refuse():
    assert masks(B=0) == vk.OK
    assert masks(mask=None) == vk.EINVAL and masks(mask=A + 4) == vk.EINVAL
    assert masks(base=None) == vk.EINVAL and masks(pos=None) == vk.EINVAL
    assert masks(axes=0) == vk.EINVAL and masks(axes=5) == vk.EINVAL
    assert masks(n=0) == vk.ESHAPE and masks(n=257) == vk.ESHAPE and masks(B=-1) == vk.ESHAPE and masks(B=65536) == vk.ESHAPE
    for k in ("parent", "count", "base", "pos"):
        assert masks(**{k: A + 2}) == vk.EINVAL


def attend(p=None, layer=0, n=5, q=view(), K=view(), V=view(), mask=A, c=A, cb=BIG, length=A, count=None, out=view(), ws=A, wb=BIG):
    p = vk.make_cache8(2, 1, 4, 28, 64) if p is None else p
    return vk.lib().vidkv_cache8_tree_attention(p if p == 0 else C.byref(p), layer, n, q, K, V, mask, c, cb, length, count, out, ws, wb, None)


def test_attention_refuses():
    p = vk.make_cache8(2, 1, 4, 28, 64)
    for k in ("q", "K", "V", "mask", "c", "length", "out", "ws"):
        assert attend(**{k: None}) == vk.EINVAL, k
    assert vk.lib().vidkv_cache8_tree_attention(None, 0, 5, view(), view(), view(), A, A, BIG, A, None, view(), A, BIG, None) == vk.EINVAL
    for bad in (view(data=A + 8), view(data=None), view(b=4), view(h=129), view(n=2), view(dtype=5), view(dtype=2), view(dtype=1)):
        for k in ("q", "K", "V", "out"):
            assert attend(**{k: bad}) == vk.EINVAL, k
    assert attend(layer=2) == vk.EINVAL and attend(layer=-1) == vk.EINVAL
    assert attend(n=0) == vk.ESHAPE and attend(n=257) == vk.ESHAPE and attend(n=-1) == vk.ESHAPE
    assert attend(mask=A + 4) == vk.EINVAL and attend(c=A + 16) == vk.EINVAL and attend(ws=A + 16) == vk.EINVAL
    assert attend(length=A + 2) == vk.EINVAL and attend(count=A + 2) == vk.EINVAL
    assert attend(cb=vk.cache8_bytes(p) - 1) == vk.ENOSPACE
    long = vk.make_cache8(1, 1, 4, 28, 196000)
    assert attend(p=long, n=64, wb=vk.cache8_workspace_bytes(long, 64) // 2) == vk.ENOSPACE
    assert attend(p=vk.make_cache8(2, 1, 4, 28, 65)) == vk.ESHAPE
    assert attend(p=vk.make_cache8(1, 65535, 65535, 65535, 32), n=256, cb=1 << 62) == vk.ESHAPE
    for scale in (0.0, -1.0, math.nan, math.inf):
        assert attend(p=vk.make_cache8(2, 1, 4, 28, 64, softmax_scale=scale)) == vk.EINVAL


def verify(B=2, n=3, V=1000, target=rows(), draft=rows(), distinct=0, token=A, parent=A, count=None, u=A, path=A, accepted=A, nxt=A,
           ws=A, wb=BIG):
    return vk.lib().vidkv_tree_verify(B, n, V, target, draft, distinct, token, parent, count, u, path, accepted, nxt, ws, wb, None)


def test_verify_refuses():
    assert verify(B=0) == vk.OK
    for k in ("target", "token", "u", "path", "accepted", "nxt", "ws"):
        assert verify(**{k: None}) == vk.EINVAL, k
    for k in ("token", "parent", "count", "u", "path", "accepted", "nxt", "ws"):
        assert verify(**{k: A + 2}) == vk.EINVAL, k
    assert verify(ws=A + 16) == vk.EINVAL
    for bad in (rows(data=None), rows(data=A + 2), rows(dtype=3), rows(dtype=-1), rows(b=1 << 50), rows(r=-(1 << 50))):
        assert verify(target=bad) == vk.EINVAL and verify(draft=bad) == vk.EINVAL
    assert verify(target=rows(dtype=0), draft=rows(dtype=1)) == vk.EINVAL
    assert verify(target=rows(dtype=0, data=A + 1), draft=None) == vk.EINVAL
    assert verify(distinct=2) == vk.EINVAL and verify(distinct=1, draft=None) == vk.EINVAL
    for bad in (dict(B=-1), dict(B=65536), dict(n=0), dict(n=257), dict(V=0), dict(V=(1 << 22) + 1)):
        assert verify(**bad) == vk.ESHAPE, bad
    assert verify(wb=vk.tree_verify_workspace_bytes(2, 3, 1000) - 1) == vk.ENOSPACE


def test_verify_sizes():
    size = vk.tree_verify_workspace_bytes
    assert size(1, 1, 1) >= 256 and size(1, 1, 1) % 256 == 0
    assert size(65535, 256, 1 << 22) >= size(1, 256, 1 << 22) >= size(1, 1, 1)
    for bad in ((0, 1, 1), (65536, 1, 1), (1, 0, 1), (1, 257, 1), (1, 1, 0), (1, 1, (1 << 22) + 1), (-1, 1, 1)):
        assert size(*bad) == 0, bad


def append(p=None, n=5, K=view(), ks=1 << 20, V=view(), vs=1 << 20, path=A, accepted=A, start=A, c=A, cb=BIG):
    p = vk.make_cache8(2, 1, 4, 28, 64) if p is None else p
    return vk.lib().vidkv_cache8_append_path(C.byref(p), n, K, ks, V, vs, path, accepted, start, c, cb, None)


def test_append_refuses():
    for k in ("K", "V", "path", "accepted", "start", "c"):
        assert append(**{k: None}) == vk.EINVAL, k
    for bad in (view(data=A + 8), view(b=4), view(h=129), view(n=2), view(dtype=5), view(dtype=2), view(dtype=1)):
        assert append(K=bad) == vk.EINVAL and append(V=bad) == vk.EINVAL
    assert append(ks=4) == vk.EINVAL and append(vs=1 << 50) == vk.EINVAL
    for k in ("path", "accepted", "start"):
        assert append(**{k: A + 2}) == vk.EINVAL, k
    assert append(c=A + 16) == vk.EINVAL and append(cb=vk.cache8_bytes(vk.make_cache8(2, 1, 4, 28, 64)) - 1) == vk.ENOSPACE
    assert append(n=0) == vk.ESHAPE and append(n=257) == vk.ESHAPE and append(p=vk.make_cache8(2, 1, 4, 28, 65)) == vk.ESHAPE
    assert append(p=vk.make_cache8(3000, 1000, 8, 8, 512), cb=1 << 62) == vk.ESHAPE          # more workgroups than a grid holds
    assert vk.lib().vidkv_cache8_append_path(None, 5, view(), 8, view(), 8, A, A, A, A, BIG, None) == vk.EINVAL


def test_the_header_and_the_binding_agree():
    src = open(os.path.join(os.path.dirname(vk.LIB_PATH), "..", "include", "vidkv.h")).read()
    assert f"#define VIDKV_TREE_NODES {vk.TREE_NODES}\n" in src and "#define VIDKV_TREE_VOCAB (1 << 22)\n" in src
    assert vk.TREE_VOCAB == 1 << 22 and C.sizeof(vk.VidkvRows) == 32


def test_binding_refuses_host_tensors_and_shapes():
    x, i = torch.zeros((1, 2, 3, 128), dtype=torch.float16), torch.zeros((1, 3), dtype=torch.int32)
    p, u8 = vk.make_cache8(1, 1, 2, 2, 32), torch.zeros(4096, dtype=torch.uint8)
    f, one = torch.zeros((1, 3, 9)), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(TypeError):
        vk.tree_masks(i, torch.zeros((1, 3, 1), dtype=torch.int64))
    with pytest.raises(ValueError):
        vk.tree_masks(i, None)
    with pytest.raises(ValueError):
        vk.tree_masks(i, torch.zeros((1, 3, 1), dtype=torch.int64), base=one)
    with pytest.raises(TypeError):
        vk.cache8_tree_attention(p, 0, u8, x, x, x, torch.zeros((1, 3, 1), dtype=torch.int64), x, one, u8)
    with pytest.raises(TypeError):
        vk.tree_verify(f, i, torch.zeros((1, 3)), i, one, one, u8)
    with pytest.raises(ValueError):
        vk.tree_verify(f, one, torch.zeros((1, 3)), i, one, one, u8)
    with pytest.raises(ValueError):
        vk.cache8_append_path(p, u8, x, x, i, one, one)
    with pytest.raises(TypeError):
        vk.cache8_append_path(p, u8, x[None], x[None], i, one, one)


def test_odd_arguments_are_left_to_the_python_path():
    """The native call layer takes plain arguments that pass, and no others."""
    vk.lib()
    m = vk._native
    assert m.tree_masks(*[None] * 7) is None and m.tree_masks(1) is None
    assert m.cache8_tree_attention(*[None] * 13) is None and m.tree_verify(*[None] * 13) is None and m.cache8_append_path(*[None] * 9) is None
    with pytest.raises(TypeError):
        m.bind_tree(1, 2)
    x, i = torch.zeros((1, 2, 3, 128), dtype=torch.float16), torch.zeros((1, 3), dtype=torch.int32)
    u, one, words = torch.zeros(4096, dtype=torch.uint8), torch.zeros(1, dtype=torch.int32), torch.zeros((1, 3, 1), dtype=torch.int64)
    p, rot, f = vk.make_cache8(1, 1, 2, 2, 32), vk.make_rotary((64,)), torch.zeros((1, 3, 9))
    assert m.tree_masks(i, words, None, None, None, vk._stream, None) is None                    # host tensors; foreign structures
    assert m.tree_verify(f, i, torch.zeros((1, 3)), i, one, one, u, None, None, None, False, vk._stream, None) is None
    for c in (p, bytes(C.sizeof(vk.VidkvCache8)), rot):
        assert m.cache8_tree_attention(c, 0, u, x, x, x, words, x, one, u, None, vk._stream, None) is None
        assert m.cache8_append_path(c, u, x[None], x[None], i, one, one, vk._stream, None) is None
