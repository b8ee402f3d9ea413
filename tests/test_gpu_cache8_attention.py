"""Attention over the 8-bit cache against dense attention in float64 over the values that the cache holds.

Tolerance (u = 2^-24), for a row with weights w_t = softmax(x), x_t = scale q.K'_t:
  x in the exponent of 2 is off by e = u (128 + 8) S, S = max_t scale log2(e) sum_c |q_c K'_tc|: 128 additions of exact products
  and the factors' roundings, each relative to the terms; the offsets added to it (magnitude, maximum; both at most |x| + 48)
  add 4 u (S + 48).  exp2 itself: 2^-22.  So each weight is off by d = ln 2 (136 u S + 4 u (S + 48)) + 2^-22 relative, in the sum
  over the tokens and in the denominator;
  the product takes weights rounded to fp16: 2^-11 of each, or, below 2^-14 of 2^7 at least, 2^-32 of the largest magnitude;
  sums of n tokens in float32 over 32-token products, waves and splits: u (n + 600) as if every addition rounded;
  the result is rounded once.
With W = sum_t w_t |V'_t|:  |error| <= W (2^-11 + 2 d + u (n + 600)) + n 2^-32 max A_V + half a step of the type."""
import math

import numpy as np
import pytest
import torch

from oracle import cache8 as O
from paper_2503_16257_amd import binding as vk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16 = torch.float16, torch.bfloat16
SCALE = 1.0 / math.sqrt(128)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def filled(B, H, rep, cap, lens, code, seed, L=1, layer=0, wild=False, dtype=F16):
    """A cache of 0xFF bytes (NaN in e4m3) with `lens` tokens a sequence written."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    p = vk.make_cache8(L, B, H, H * rep, cap, code)
    buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
    buf.fill_(0xFF)
    n = max(max(lens), 1)
    K, V = (torch.randn((B, H, n, 128), generator=g, device=DEV) for _ in range(2))
    if wild:                                       # blocks of very different magnitudes, a heavy channel
        V *= torch.exp2(torch.randint(-12, 13, (B, H, n, 1), generator=g, device=DEV).float())
        K[..., 5] *= 30
    vk.cache8_write(p, layer, buf, K.to(dtype), V.to(dtype), i32([0] * B), i32(lens))
    return p, buf


def check(p, layer, buf, q, out, lens, causal=True, counts=None, rows=None):
    B, Hq, n, _ = q.shape
    H, cap = p.n_kv_heads, p.capacity
    rep = Hq // H
    kc, vc, km, vm = O.unpack(buf.cpu().numpy(), p.n_layers, B, H, cap)
    q64, o64 = q.double().cpu().numpy(), out.double().cpu().numpy()
    assert np.isfinite(o64).all()
    eps = torch.finfo(out.dtype).eps / 2
    worst = 0.0
    for b in range(B):
        T = min(max(lens[b], 0), cap)
        nq = n if counts is None else min(max(counts[b], 0), n)
        assert (o64[b, :, nq:] == 0).all()
        pick = range(nq) if rows is None else sorted({i for i in rows if 0 <= i < nq})
        for h in range(H):
            K = O.values(kc[layer, b, h], km[layer, b, h], p.code)[:T]
            V = O.values(vc[layer, b, h], vm[layer, b, h], p.code)[:T]
            big = vm[layer, b, h][:-(-T // 32)].max() if T else 0.0
            for r in range(h * rep, h * rep + rep):
                for i in pick:
                    t = min(max(T - nq + i + 1, 0), T) if causal else T
                    if t == 0:
                        assert (o64[b, r, i] == 0).all(), (b, r, i)
                        continue
                    x = SCALE * (K[:t] @ q64[b, r, i])
                    w = np.exp(x - x.max())
                    w /= w.sum()
                    ref, W = w @ V[:t], w @ np.abs(V[:t])
                    S = SCALE * math.log2(math.e) * (np.abs(K[:t]) @ np.abs(q64[b, r, i])).max()
                    u = 2.0 ** -24
                    d = math.log(2) * (136 * u * S + 4 * u * (S + 48)) + 2.0 ** -22
                    tol = W * (2.0 ** -11 + 2 * d + u * (t + 600)) + t * 2.0 ** -32 * big + eps * np.abs(ref) * 1.01
                    tol = tol + (2.0 ** -25 if out.dtype == F16 else 0.0)
                    err = np.abs(o64[b, r, i] - ref)
                    worst = max(worst, (err / tol).max())
                    assert (err <= tol).all(), (b, r, i, t, (err / tol).max())
    print(f"  worst {worst:.3f} of the bound", flush=True)


def attend(p, layer, buf, q, lens, causal=True, counts=None, strided=False):
    B, Hq, n, _ = q.shape
    out = torch.full((B, n, Hq, 128), float("nan"), dtype=q.dtype, device=DEV).transpose(1, 2) if strided else \
        torch.full_like(q, float("nan"))
    ws = vk.alloc_bytes(vk.cache8_workspace_bytes(p, n), DEV)
    ws.fill_(0xFF)
    vk.cache8_attention(p, layer, buf, q, out, i32(lens), ws, q_count=None if counts is None else i32(counts), causal=causal)
    torch.cuda.synchronize()
    return out


def queries(B, Hq, n, dtype, seed, strided=False, size=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed + 99)
    q = (size * torch.randn((B, n, Hq, 128), generator=g, device=DEV)).to(dtype).transpose(1, 2)
    return q if strided else q.contiguous()


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("B,H,rep,cap,lens", [
    (1, 1, 1, 32, [1]), (9, 1, 7, 1024, [0, 1, 2, 31, 32, 33, 64, 1000, 1024]), (3, 4, 7, 6272, [6272, 5, 4001]),
    (2, 3, 8, 96, [96, 95]), (1, 2, 16, 320, [300]), (2, 1, 13, 160, [-3, 999]), (70, 2, 2, 64, list(range(70))),
    (1, 1, 20, 640, [611]), (1, 1, 33, 640, [611]),
])
def test_single_tokens(B, H, rep, cap, lens, code, dtype):
    print(f"[case] single B={B} H={H} rep={rep} cap={cap} code={code} {dtype}", flush=True)
    p, buf = filled(B, H, rep, cap, lens, code, 1, dtype=dtype)
    q = queries(B, H * rep, 1, dtype, 2)
    check(p, 0, buf, q, attend(p, 0, buf, q, lens), lens)


@pytest.mark.parametrize("code,dtype", [(0, F16), (1, BF16)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("B,H,rep,n,cap,lens,counts", [
    (3, 2, 8, 2, 96, [0, 1, 70], None), (2, 1, 7, 3, 512, [2, 500], [3, 1]), (2, 2, 8, 5, 256, [3, 251], None),
    (4, 1, 1, 17, 64, [17, 5, 64, 33], [17, 17, 0, 40]), (2, 2, 7, 37, 320, [300, 37], None),
    (1, 1, 4, 130, 160, [130], None), (2, 1, 7, 100, 640, [640, 20], [99, 100]), (1, 2, 1, 300, 320, [310], None),
    (3, 2, 7, 8, 1024, [1000, 8, 3], [8, 5, 8]), (2, 1, 7, 16, 2048, [2048, 33], None), (2, 1, 8, 24, 512, [480, 25], None),
    (2, 1, 64, 1, 320, [320, 1], None), (1, 1, 65, 2, 96, [70], None),
])
def test_several_queries(B, H, rep, n, cap, lens, counts, causal, code, dtype):
    print(f"[case] several B={B} H={H} rep={rep} n={n} cap={cap} code={code}", flush=True)
    p, buf = filled(B, H, rep, cap, lens, code, 3, dtype=dtype)
    q = queries(B, H * rep, n, dtype, 4, strided=True)
    check(p, 0, buf, q, attend(p, 0, buf, q, lens, causal, counts, strided=True), lens, causal, counts)


@pytest.mark.parametrize("B,H,rep,n,T,code,dtype", [
    (1, 4, 7, 1, 98000, 0, F16), (1, 4, 7, 196, 30011, 1, BF16), (1, 2, 7, 1999, 1999, 0, BF16), (2, 4, 7, 700, 1500, 1, F16),
])
def test_long(B, H, rep, n, T, code, dtype):
    """Many splits, many row tiles; sampled queries."""
    print(f"[case] long n={n} T={T}", flush=True)
    lens = [T - 300 * b for b in range(B)]
    p, buf = filled(B, H, rep, -(-T // 32) * 32, lens, code, 5, dtype=dtype)
    q = queries(B, H * rep, n, dtype, 6)
    check(p, 0, buf, q, attend(p, 0, buf, q, lens), lens, rows=[0, 1, 63, 64, n // 2, n - 2, n - 1])


@pytest.mark.parametrize("code", [0, 1])
def test_many_heads(code):
    """As many heads as compute units, short and long (a workgroup a head, and several): sampled sequences against a cache of
    their own, which the other ways of sharing the work go through."""
    for B, H, rep, cap in ((128, 2, 7, 96), (96, 2, 4, 12320), (300, 4, 1, 64), (1100, 1, 2, 320)):
        print(f"[case] many heads B={B} H={H} cap={cap}", flush=True)
        g = torch.Generator(device=DEV)
        g.manual_seed(40 + B)
        lens = [(cap - 7 * b) % (cap + 1) for b in range(B)]
        K, V = (torch.randn((B, H, cap, 128), generator=g, device=DEV, dtype=torch.float16) for _ in range(2))
        p = vk.make_cache8(1, B, H, H * rep, cap, code)
        buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
        buf.fill_(0xFF)
        vk.cache8_write(p, 0, buf, K, V, i32([0] * B), i32(lens))
        q = queries(B, H * rep, 1, F16, 41)
        out = attend(p, 0, buf, q, lens)
        for b in (0, 1, B // 2, B - 1):
            one = vk.make_cache8(1, 1, H, H * rep, cap, code)
            small = vk.alloc_bytes(vk.cache8_bytes(one), DEV)
            small.fill_(0xFF)
            vk.cache8_write(one, 0, small, K[b:b + 1], V[b:b + 1], i32([0]), i32([lens[b]]))
            check(one, 0, small, q[b:b + 1], out[b:b + 1], [lens[b]])
        del K, V, buf


@pytest.mark.parametrize("code", [0, 1])
def test_wild_magnitudes_and_queries(code):
    """Blocks whose values differ by 2^24, scores that take the whole softmax, queries from 1e-6 to 1e4."""
    for dtype, size in ((F16, 1.0), (F16, 50.0), (BF16, 1e4), (BF16, 1e-6), (BF16, 3.0)):
        p, buf = filled(2, 1, 7, 640, [640, 333], code, 7, wild=True)
        for n in (1, 40):
            q = queries(2, 7, n, dtype, 8, size=size)
            if dtype == BF16:
                q[..., 3] *= 1e-5                  # and channels far apart
            check(p, 0, buf, q, attend(p, 0, buf, q, [640, 333]), [640, 333])


def test_scores_at_the_ends_of_float():
    """Scores that vanish (equal weights) beside masked tokens, keys of the least magnitude.  Weights are exact here but for
    fp16's half step and log2's and exp2's last bits.  (Scores of 2^24 and more are not the interface's: S in the bound above
    is then 2^24 u = 1 and more in a weight's exponent.)"""
    g = torch.Generator(device=DEV)
    g.manual_seed(50)
    for key, query, scale in ((2.0 ** -41, 1e-35, 1e-30), (1.0, 1e-36, SCALE), (2.0 ** -20, 1e-30, SCALE)):
        p = vk.make_cache8(1, 1, 1, 3, 96, 0, softmax_scale=scale)
        buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
        K = torch.zeros((1, 1, 96, 128), device=DEV)
        K[..., 0] = key * (1 + torch.arange(96, device=DEV) / 256)             # ascending: the last seen token has the largest score
        V = torch.randn((1, 1, 96, 128), generator=g, device=DEV)
        vk.cache8_write(p, 0, buf, K.bfloat16(), V.bfloat16(), i32([0]))
        kc, vc, km, vm = O.unpack(buf.cpu().numpy(), 1, 1, 1, 96)
        Kd, Vd = O.values(kc[0, 0, 0], km[0, 0, 0], 0), O.values(vc[0, 0, 0], vm[0, 0, 0], 0)
        for n, T in ((1, 70), (40, 70), (1, 96)):
            q = torch.full((1, 3, n, 128), query, dtype=torch.float32, device=DEV).bfloat16()
            out = attend(p, 0, buf, q, [T]).double().cpu().numpy()
            for i in range(n):
                t = T - n + i + 1
                x = (Kd[:t, 0] * float(query)).astype(np.float64) * scale
                w = np.exp(np.clip(x - x.max(), -1e4, 0))
                ref = (w / w.sum()) @ Vd[:t]
                tol = (np.abs(Vd[:t]).max() * 2.0 ** -10 + 2.0 ** -8 * np.abs(ref))
                assert (np.abs(out[0, :, i] - ref) <= tol).all(), (key, query, n, i)


def test_rising_scores():
    """Every block's scores above all before by more than the maximum's slack: the running sums are rescaled each time."""
    p = vk.make_cache8(1, 1, 1, 2, 1024, 0)
    buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
    K = torch.zeros((1, 1, 1024, 128), device=DEV)
    K[..., 0] = torch.arange(1024, device=DEV) * 4.0
    V = torch.randn((1, 1, 1024, 128), device=DEV)
    vk.cache8_write(p, 0, buf, K.half(), V.half(), i32([0]))
    for n in (1, 100):
        q = torch.zeros((1, 2, n, 128), dtype=F16, device=DEV)
        q[:, 0, :, 0], q[:, 1, :, 0] = 8.0, -8.0
        check(p, 0, buf, q, attend(p, 0, buf, q, [1024]), [1024])


def test_rows_of_unseen_queries_do_not_depend_on_them():
    """NaN in queries behind q_count, in dead codes and in other sequences stays there."""
    p, buf = filled(2, 1, 4, 128, [100, 128], 1, 9)
    for n in (3, 60):
        q = queries(2, 4, n, F16, 10)
        a = attend(p, 0, buf, q, [100, 128], counts=[n - 1, n])
        q2 = q.clone()
        q2[0, :, n - 1:] = float("nan")
        b = attend(p, 0, buf, q2, [100, 128], counts=[n - 1, n])
        assert torch.equal(a, b)
        q2 = q.clone()
        q2[1] = float("nan")
        b = attend(p, 0, buf, q2, [100, 128], counts=[n - 1, n])
        assert torch.equal(a[0], b[0]) and torch.isnan(b[1]).all()


def test_one_workspace_for_every_number_of_queries():
    """Sized once for the most queries: fewer ones fit, and nothing behind it is written."""
    p, buf = filled(1, 1, 7, 6272, [6272], 0, 25)
    size = vk.cache8_workspace_bytes(p, 29)
    ws = vk.alloc_bytes(size + 4096, DEV)
    for n in (29, 28, 27, 7, 6, 1):
        ws.fill_(0x5A)
        q = queries(1, 7, n, F16, 26 + n)
        out = torch.empty_like(q)
        vk.cache8_attention(p, 0, buf, q, out, i32([6272]), ws[:size])
        check(p, 0, buf, q, out, [6272], rows=[0, n - 1])
        assert (ws[size:] == 0x5A).all()


def test_a_layer_beyond_32_bit_offsets():
    L, B, H, cap = 5, 8, 8, 131200
    p = vk.make_cache8(L, B, H, H * 2, cap, 1)
    buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(21)
    K, V = (torch.randn((B, H, 70, 128), generator=g, device=DEV).half() for _ in range(2))
    small = vk.make_cache8(1, B, H, H * 2, 96, 1)
    sbuf = vk.alloc_bytes(vk.cache8_bytes(small), DEV)
    for pp, bb, layer in ((p, buf, L - 1), (small, sbuf, 0)):
        vk.cache8_write(pp, layer, bb, K, V, i32([0] * B))
    q = queries(B, H * 2, 1, F16, 22)
    out = attend(small, 0, sbuf, q, [70] * B)
    check(small, 0, sbuf, q, out, [70] * B)
    far = attend(p, L - 1, buf, q, [70] * B)
    assert (far.double() - out.double()).abs().max() <= 2.0 ** -9 * out.abs().max().item()   # two splits of the same sums


def test_refusals_of_the_binding():
    p, buf = filled(2, 2, 3, 64, [3, 4], 0, 23)
    q = queries(2, 6, 4, F16, 24)
    out = torch.full_like(q, 7.0)
    ws = vk.alloc_bytes(vk.cache8_workspace_bytes(p, 4), DEV)
    n = i32([3, 4])
    for kw in (dict(q=q[:1]), dict(q=q[:, :2]), dict(q=q.float(), out=out.float()), dict(out=out[:, :, :3]), dict(q=q.double()),
               dict(length=n.long()), dict(length=i32([1])), dict(q_count=i32([1])), dict(length=n.cpu()), dict(q=q[..., ::2]),
               dict(out=out[:, :1].expand(2, 6, 4, 128)), dict(out=out.to(BF16)), dict(cache=buf[:-256])):
        a = dict(cache=buf, q=q, out=out, length=n, workspace=ws) | kw
        with pytest.raises((TypeError, ValueError, vk.VidkvError)):
            vk.cache8_attention(p, 0, **a)
    assert (out == 7.0).all()
    vk.cache8_attention(p, 0, buf, q[:, :, :0], out[:, :, :0], n, ws)
