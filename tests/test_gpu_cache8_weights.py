"""Attention over the 8-bit cache where blocks differ: blocks of zero values and of very small ones beside ordinary ones,
blocks of a cleared buffer, equal values, queries that are not numbers behind q_count.

Tolerance (u = 2^-24) against dense attention in float64 over the values that the cache holds, for a row of weights w_t over n
tokens, W = sum_t w_t |V'_t|, S = max_t scale log2(e) sum_c |q_c K'_tc|:
  a weight's exponent: 136 u S + 4 u (S + 48), exp2 and log2 2^-22 each: d = ln 2 of the first + 2^-21, in the sum over the
  tokens and in the denominator;
  weights in fp16, in the products and in the denominator: 2^-11 of each, twice; below 2^-14 of 2^7 at least, half of fp16's
  smallest step, 2^-25: of 2^7 2^-32, in the sum of the largest magnitude, in the denominator - of blocks whose magnitude is an
  eighth of the largest at least; others' weights have float32's range there - of 2^-3 of the largest weight;
  sums in float32: u (n + 600); the result is rounded once.
|error| <= W (2^-10 + 2 d + u (n + 600)) + |result| n 2^-29 + n 2^-32 max A_V + half a step of the type."""
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


def empty(B, H, rep, cap, code, fill=0xFF):
    p = vk.make_cache8(1, B, H, H * rep, cap, code)
    buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
    buf.fill_(fill)
    return p, buf


def attend(p, buf, q, lens, causal=False, counts=None):
    out = torch.full_like(q, float("nan"))
    ws = vk.alloc_bytes(vk.cache8_workspace_bytes(p, q.shape[2]), DEV)
    vk.cache8_attention(p, 0, buf, q, out, i32(lens), ws, q_count=None if counts is None else i32(counts), causal=causal)
    torch.cuda.synchronize()
    return out


def check(p, buf, q, out, lens, causal=False):
    B, Hq, n, _ = q.shape
    rep, u = Hq // p.n_kv_heads, 2.0 ** -24
    kc, vc, km, vm = O.unpack(buf.cpu().numpy(), 1, B, p.n_kv_heads, p.capacity)
    q64, got = q.double().cpu().numpy(), out.double().cpu().numpy()
    assert np.isfinite(got).all()
    for b in range(B):
        for r in range(Hq):
            T, h = lens[b], r // rep
            K = O.values(kc[0, b, h], km[0, b, h], p.code)[:T]
            V = O.values(vc[0, b, h], vm[0, b, h], p.code)[:T]
            x = SCALE * (q64[b, r] @ K.T)
            S = SCALE * math.log2(math.e) * (np.abs(q64[b, r]) @ np.abs(K).T).max()
            limit = T - n + 1 + np.arange(n) if causal else np.full(n, T)
            x = np.where(np.arange(T)[None] < limit[:, None], x, -np.inf)
            w = np.exp(x - x.max(axis=1, keepdims=True))
            w /= w.sum(axis=1, keepdims=True)
            ref, W = w @ V, w @ np.abs(V)
            d = math.log(2) * (136 * u * S + 4 * u * (S + 48)) + 2.0 ** -21
            tol = W * (2.0 ** -10 + 2 * d + u * (T + 600)) + np.abs(ref) * (T * 2.0 ** -29 + 1.01 * torch.finfo(out.dtype).eps / 2)
            tol = tol + T * 2.0 ** -32 * vm[0, b, h, :-(-T // 32)].max() + (2.0 ** -25 if out.dtype == F16 else 0)
            err = np.abs(got[b, r] - ref)
            assert (err <= tol).all(), (b, r, (err / tol).max())


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("rep,n", [(1, 1), (7, 5), (1, 64), (2, 64), (7, 40)])
def test_half_of_the_tokens_have_no_value(rep, n, code):
    """Scores of zero, values 1 in the first block and 0 in the second: every result is 1/2, in either order."""
    for order in ((1.0, 0.0), (0.0, 1.0)):
        p, buf = empty(1, 1, rep, 64, code)
        V = torch.tensor(order, device=DEV).repeat_interleave(32)[None, None, :, None].expand(1, 1, 64, 128)
        vk.cache8_write(p, 0, buf, torch.zeros((1, 1, 64, 128), dtype=F16, device=DEV), V.half().contiguous(), i32([0]))
        q = torch.ones((1, rep, n, 128), dtype=F16, device=DEV)
        out = attend(p, buf, q, [64])
        print(f"[case] rep={rep} n={n} code={code} {order}: {out.float().min().item()} .. {out.float().max().item()}", flush=True)
        assert ((out.double() - 0.5).abs() <= 0.5 * 2.0 ** -10).all()


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,H,rep,n,cap,lens", [
    (2, 2, 3, 1, 256, [256, 131]), (1, 2, 5, 1, 8192, [8100]), (130, 2, 1, 1, 640, [640 - b for b in range(130)]),
    (2, 1, 7, 5, 256, [256, 99]), (2, 2, 1, 64, 256, [256, 160]), (1, 1, 2, 64, 2048, [2048]), (1, 1, 7, 30, 2048, [2013]),
    (2, 1, 7, 60, 256, [250, 256]),
])
def test_blocks_far_apart(B, H, rep, n, cap, lens, causal, code):
    """A magnitude drawn for each block: none, 2^-30, 2^-16, 1/16, 1/8, 1 or 2^9; the first block ordinary."""
    print(f"[case] apart B={B} H={H} rep={rep} n={n} cap={cap} causal={causal} code={code}", flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(71 + n)
    p, buf = empty(B, H, rep, cap, code)
    K, V = (torch.randn((B, H, cap, 128), generator=g, device=DEV) for _ in range(2))
    sizes = torch.tensor([0.0, 2.0 ** -30, 2.0 ** -16, 2.0 ** -4, 2.0 ** -3, 1.0, 512.0], device=DEV)
    pick = torch.randint(0, 7, (B, H, cap // 32), generator=g, device=DEV)
    pick[:, :, 0] = 5
    V = V * sizes[pick].repeat_interleave(32, dim=2)[..., None]
    vk.cache8_write(p, 0, buf, K.bfloat16(), V.bfloat16(), i32([0] * B), i32(lens))
    dtype = BF16 if code else F16
    q = torch.randn((B, H * rep, n, 128), generator=g, device=DEV).to(dtype)
    check(p, buf, q, attend(p, buf, q, lens, causal), lens, causal)


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("rep,n,B,cap", [(16, 1, 300, 2048), (32, 1, 300, 2048), (16, 3, 300, 2048), (16, 8, 20, 2048),
                                         (16, 12, 20, 256)])
def test_equal_values_come_out_as_they_are(rep, n, B, cap, code):
    """Values of 1 throughout: numerator and denominator are then the same sum of the same weights, whatever these are rounded
    to.  Scores are 0 and one number a row up to 5.5 (2^8 of weight, which the maximum is not raised for) in turn of blocks.
    Off by u (n + 600) <= 1.6e-4 before the rounding, less than the 2^-12 that fp16's 1 is rounded from."""
    print(f"[case] equal rep={rep} n={n} B={B} cap={cap} code={code}", flush=True)
    p, buf = empty(B, 1, rep, cap, code)
    K = torch.zeros((B, 1, cap, 128), dtype=F16, device=DEV)
    K[..., 0] = torch.arange(cap, device=DEV) // 32 % 2
    vk.cache8_write(p, 0, buf, K, torch.ones_like(K), i32([0] * B))
    q = torch.zeros((B, rep, n, 128), dtype=F16, device=DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(72)
    q[..., 0] = (5.5 / SCALE * torch.rand((B, rep, n), generator=g, device=DEV)).half()
    out = attend(p, buf, q, [cap] * B)
    print("  ", out.float().min().item(), out.float().max().item(), flush=True)
    assert (out == 1.0).all()


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("rep,n", [(4, 1), (4, 9), (2, 40), (7, 40)])
def test_cleared_blocks_are_tokens_of_zeros(rep, n, code):
    """A cleared buffer whose first 69 tokens were never written: a left-padded sequence.  They come back as zeros, and the
    attention takes them as such."""
    for cap in (128, 4096):
        print(f"[case] cleared rep={rep} n={n} cap={cap} code={code}", flush=True)
        p, buf = empty(1, 1, rep, cap, code, fill=0)
        g = torch.Generator(device=DEV)
        g.manual_seed(73)
        K, V = (torch.randn((1, 1, cap - 69, 128), generator=g, device=DEV).half() for _ in range(2))
        vk.cache8_write(p, 0, buf, K, V, i32([69]))
        q = torch.randn((1, rep, n, 128), generator=g, device=DEV).half()
        for lens, causal in (([cap], False), ([110], True), ([69], False), ([64], True)):
            check(p, buf, q, attend(p, buf, q, lens, causal), lens, causal)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("rep,n", [(4, 3), (16, 2), (2, 40), (7, 60)])
def test_infinite_queries_behind_the_count_give_zeros(rep, n, dtype):
    """Keys above zero in the channel where such a query is infinite: its scores are infinite, not NaN."""
    for cap, causal in ((320, True), (320, False), (6272, True)):
        print(f"[case] behind the count rep={rep} n={n} cap={cap} {dtype}", flush=True)
        p, buf = empty(1, 1, rep, cap, 0)
        g = torch.Generator(device=DEV)
        g.manual_seed(74)
        K, V = (torch.randn((1, 1, cap, 128), generator=g, device=DEV) for _ in range(2))
        K[..., 0] = K[..., 0].abs() + 2
        vk.cache8_write(p, 0, buf, K.to(dtype), V.to(dtype), i32([0]))
        q = torch.randn((1, rep, n, 128), generator=g, device=DEV).to(dtype)
        q[:, :, n - 1:] = 0
        want = attend(p, buf, q, [cap], causal, [n - 1])
        q[:, :, n - 1:, 0] = float("inf")
        got = attend(p, buf, q, [cap], causal, [n - 1])
        assert (got[:, :, n - 1:] == 0).all() and torch.equal(got, want)
