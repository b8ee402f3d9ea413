"""The attention's workspace: what the size query says for n queries is taken for every call of up to n."""
import ctypes as C
import random

import pytest
import torch

from paper_2503_16257_amd import binding as vk

A = 0x10000                                                # a 256-aligned address
DEV = "cuda:0"


def plan(B, H, rep, cap):
    return vk.make_cache8(1, B, H, H * rep, cap)


def refused_for_space(p, n, size):
    """Whether a call of n queries finds `size` bytes too few (else it goes on to a launch, which ends without a device)."""
    v = C.byref(vk.VidkvView(A, 1 << 20, 128, 1 << 16, 0))
    st = vk.lib().vidkv_cache8_attention(C.byref(p), 0, n, 1, v, A, 1 << 62, A, None, v, A, size, None)
    assert st in (vk.ENOSPACE, vk.EHIP), st
    return st == vk.ENOSPACE


# (batch, heads, ratio, capacity), numbers of queries: on both sides of where the tiles of rows come to one and to two a
# compute unit, and of where a workgroup has eight blocks
SHAPES = [((1, 8, 8, 2048), range(1, 1600, 7)), ((2, 4, 7, 2048), range(1, 1800, 9)), ((4, 4, 7, 2048), range(1, 900, 3)),
          ((8, 4, 7, 1280), range(1, 420)), ((9, 4, 7, 1024), range(1, 300)), ((32, 1, 7, 992), range(1, 700, 2)),
          ((64, 8, 8, 256), range(1, 100)), ((1, 1, 1, 196000), range(1, 120000, 601)), ((3, 5, 2, 288), range(1, 4000, 29))]


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls would launch")
@pytest.mark.parametrize("shape,ns", SHAPES)
def test_every_call_fits_what_was_asked_for(shape, ns):
    p = plan(*shape)
    sizes = [vk.cache8_workspace_bytes(p, n) for n in ns]
    assert sizes == sorted(sizes)                          # so the smallest that has to do for n is that of n itself
    assert [n for n, size in zip(ns, sizes) if refused_for_space(p, n, size)] == []


@pytest.mark.skipif(torch.cuda.is_available(), reason="the calls would launch")
def test_every_call_fits_what_was_asked_for_in_drawn_shapes():
    r = random.Random(8)
    for _ in range(4000):
        shape = (r.choice([1, 2, 3, 5, 8, 9, 16, 33, 64]), r.choice([1, 2, 4, 8]), r.choice([1, 2, 4, 7, 8, 13]),
                 32 * int(2 ** r.uniform(0, 12)))
        p, n = plan(*shape), int(2 ** r.uniform(0, 13))
        size = vk.cache8_workspace_bytes(p, n)
        for m in {n, r.randint(1, n), r.randint(max(1, n // 2), n)}:
            assert not refused_for_space(p, m, size), (shape, n, m)


@pytest.mark.gpu
@pytest.mark.parametrize("B,H,rep,cap,n", [(9, 4, 7, 1024, 196), (1, 8, 8, 2048, 1200)])
def test_a_frame_in_the_band_behind_the_first_unsplit_plan(B, H, rep, cap, n):
    """A workspace of just the size: taken, nothing behind it written, and the result that of any larger one.  Sampled rows
    against dense attention over what the cache reads back, with the bound of the attention's tests in short: weights to
    2^-10 of the largest value, the type's half step."""
    print(f"[case] B={B} H={H} rep={rep} cap={cap} n={n}", flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(B)
    p = plan(B, H, rep, cap)
    buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
    K, V = (torch.randn((B, H, cap, 128), generator=g, device=DEV).half() for _ in range(2))
    start = torch.zeros(B, dtype=torch.int32, device=DEV)
    vk.cache8_write(p, 0, buf, K, V, start)
    q = torch.randn((B, H * rep, n, 128), generator=g, device=DEV).half()
    out = torch.empty_like(q)
    size = vk.cache8_workspace_bytes(p, n)
    ws = vk.alloc_bytes(size + 4096, DEV)
    ws.fill_(0x5A)
    vk.cache8_attention(p, 0, buf, q, out, start + cap, ws[:size])
    assert (ws[size:] == 0x5A).all()
    Kb, Vb = (torch.empty((B, H, cap, 128), device=DEV) for _ in range(2))
    vk.cache8_read(p, 0, buf, start, Kb, Vb)
    for b, h, i in ((0, 0, 0), (B - 1, H * rep - 1, n - 1), (B // 2, 3, n // 2)):
        t = cap - n + i + 1
        k, v = Kb[b, h // rep, :t].double().cpu(), Vb[b, h // rep, :t].double().cpu()
        w = torch.softmax(k @ q[b, h, i].double().cpu() / 128 ** 0.5, dim=0)
        ref, got = w @ v, out[b, h, i].double().cpu()
        assert ((got - ref).abs() <= 2.0 ** -10 * (w @ v.abs()) + 2.0 ** -11 * ref.abs() + 2.0 ** -12 * v.abs().max()).all()
