"""Trees of drafted tokens on the GPU against oracle/tree.py: masks and positions, attention over the 8-bit cache and the
tree's own keys and values, the accepted path appended.

Masks, positions and codes have to be equal.  Tolerance of the attention: that of the attention over the cache (derived in
test_gpu_cache8_attention.py), whose sums take the drafted tokens along: products of 16-bit keys and queries are exact in float32
as those of codes are; an fp16 value's weight is rounded as a code's, a bf16 value's to 16 bits.  What 2^-32 of the largest magnitude
bounds there (weights below fp16's range) is here relative to the cached magnitudes and to `level` for a drafted block:
  |error| <= W (2^-11 + 2 d + u (n + 600)) + n 2^-32 max(A_V, level) + half a step of the type."""
import math

import numpy as np
import pytest
import torch

from oracle import cache8 as C
from oracle import tree as O
from paper_2503_16257_amd import binding as vk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16 = torch.float16, torch.bfloat16
SCALE = 1.0 / math.sqrt(128)
TOP = {F16: 65504.0, BF16: 2.0 ** 40}


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def f64(t):
    return t.double().cpu().numpy()


def bits(words):
    """uint64 words on the host -> int64 tensor on the GPU."""
    return torch.from_numpy(np.ascontiguousarray(words).view(np.int64)).to(DEV)


def some_tree(r, n, width):
    return [-1] + [int(r.integers(max(0, i - width), i)) for i in range(1, n)]


# ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("n", [1, 2, 33, 64, 65, 128, 129, 200, 256])
@pytest.mark.parametrize("axes", [0, 1, 3, 4])
def test_masks(n, axes):
    r = np.random.default_rng(n)
    B = 5
    parents = np.array([some_tree(r, n, w) for w in (1, 2, 5, n, n)])
    parents[4] = r.integers(-3, n + 3, n)                       # (anything)
    for counts in (None, [n, 0, n + 9, n // 2, -1]):
        print(f"[case] masks n={n} axes={axes} counts={counts}", flush=True)
        base = r.integers(-1000, 2 ** 30, B)
        out = torch.full((B, n, -(-n // 64)), -1, dtype=torch.int64, device=DEV)
        pos = torch.full((axes, B, n), -9, dtype=torch.int32, device=DEV) if axes else None
        vk.tree_masks(i32(parents), out, i32(base) if axes else None, pos, count=None if counts is None else i32(counts))
        for b in range(B):
            sees, depth = O.masks(n, parents[b], n if counts is None else counts[b])
            assert (out[b].cpu().numpy().view(np.uint64) == O.words(sees)).all(), b
            if axes:
                assert (pos[:, b].cpu().numpy() == base[b] + depth).all(), b


@pytest.mark.parametrize("n", [1, 7, 64, 100, 256])
def test_masks_of_chains(n):
    out = torch.zeros((2, n, -(-n // 64)), dtype=torch.int64, device=DEV)
    pos = torch.zeros((1, 2, n), dtype=torch.int32, device=DEV)
    vk.tree_masks(None, out, i32([0, 50]), pos, count=i32([n, n - 1]))
    for b in range(2):
        sees, depth = O.masks(n, None, n - b)
        assert (out[b].cpu().numpy().view(np.uint64) == O.words(sees)).all()
        assert (pos[0, b].cpu().numpy() == 50 * b + depth).all()


# ---------------------------------------------------------------------------------------
class Case:
    """A cache of 0xFF bytes (NaN in e4m3) with lens[b] tokens written, a tree beside it, and a workspace of NaN."""

    def __init__(self, B, H, rep, n, cap, lens, code, dtype, seed, L=1, layer=0, strided=False, size=1.0, v_size=1.0):
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        mk = lambda h, t, s=1.0: (s * torch.randn((B, t, h, 128), generator=g, device=DEV)).to(dtype).transpose(1, 2)  # noqa: E731
        lay = (lambda x: x) if strided else (lambda x: x.contiguous())
        self.p = vk.make_cache8(L, B, H, H * rep, cap, code)
        self.layer, self.dtype, self.lens, self.n = layer, dtype, lens, n
        self.buf = vk.alloc_bytes(vk.cache8_bytes(self.p), DEV)
        self.buf.fill_(0xFF)
        t = max(max(lens), 1)
        vk.cache8_write(self.p, layer, self.buf, mk(H, t), mk(H, t), i32([0] * B), i32(lens))
        self.q, self.K, self.V = lay(mk(H * rep, n, size)), lay(mk(H, n)), lay(mk(H, n, v_size))
        self.ws = vk.alloc_bytes(vk.cache8_workspace_bytes(self.p, n), DEV)
        self.ws.fill_(0xFF)

    def run(self, masks, counts=None, stream=None):
        out = torch.full_like(self.q, float("nan"))
        vk.cache8_tree_attention(self.p, self.layer, self.buf, self.q, self.K, self.V, masks, out, i32(self.lens), self.ws,
                                 count=None if counts is None else i32(counts), stream=stream)
        return out

    def check(self, out, sees, counts=None, rows=None):
        p, n, lay = self.p, self.n, self.layer
        B, H, cap = p.batch, p.n_kv_heads, p.capacity
        rep = p.n_q_heads // H
        kc, vc, km, vm = C.unpack(self.buf.cpu().numpy(), p.n_layers, B, H, cap)
        q, o = f64(self.q), f64(out)
        top = TOP[self.dtype]
        Kt, Vt = O.taken(f64(self.K), top), O.taken(f64(self.V), top)
        assert np.isfinite(o).all()
        eps, u, worst = torch.finfo(self.dtype).eps / 2, 2.0 ** -24, 0.0
        for b in range(B):
            T = min(max(self.lens[b], 0), cap)
            m = n if counts is None else min(max(counts[b], 0), n)
            assert (o[b, :, m:] == 0).all(), b
            for h in range(H):
                K = np.concatenate([C.values(kc[lay, b, h], km[lay, b, h], p.code)[:T], Kt[b, h, :m]])
                V = np.concatenate([C.values(vc[lay, b, h], vm[lay, b, h], p.code)[:T], Vt[b, h, :m]])
                big = max(vm[lay, b, h][:-(-T // 32)].max() if T else 0.0, C.LEVEL[p.code])
                see = np.concatenate([np.ones((m, T), bool), sees[b][:m, :m]], axis=1)
                pick = range(m) if rows is None else sorted({i for i in rows if i < m})
                for r in range(h * rep, h * rep + rep):
                    ref, W = O.attention(q[b, r][list(pick)], K, V, SCALE, see[list(pick)])
                    for k, i in enumerate(pick):
                        t = np.flatnonzero(see[i])
                        if t.size == 0:
                            assert (o[b, r, i] == 0).all(), (b, r, i)
                            continue
                        S = SCALE * math.log2(math.e) * (np.abs(K[t]) @ np.abs(q[b, r, i])).max()
                        d = math.log(2) * (136 * u * S + 4 * u * (S + 48)) + 2.0 ** -22
                        tol = W[k] * (2.0 ** -11 + 2 * d + u * (t.size + 600)) + t.size * 2.0 ** -32 * big + eps * np.abs(ref[k]) * 1.01
                        tol = tol + (2.0 ** -25 if self.dtype == F16 else 0.0)
                        err = np.abs(o[b, r, i] - ref[k])
                        worst = max(worst, (err / tol).max())
                        assert (err <= tol).all(), (b, r, i, (err / tol).max())
        print(f"  worst {worst:.3f} of the bound", flush=True)


def trees(B, n, seed, width=4):
    r = np.random.default_rng(seed)
    return [O.masks(n, some_tree(r, n, width), n)[0] for _ in range(B)]


def words(sees):
    return bits(np.stack([O.words(s) for s in sees]))


SHAPES = [
    # few rows: a tile, two, three; twelve waves (a cache of a block a wave); several splits; every count of waves and blocks
    (1, 1, 1, 1, 32, [1], None), (1, 1, 1, 2, 32, [0], None), (2, 1, 1, 16, 64, [40, 0], [16, 3]),
    (3, 2, 7, 2, 96, [0, 33, 96], [2, 0, 1]), (2, 1, 8, 4, 2048, [2000, 31], None), (2, 2, 8, 6, 512, [511, 100], [5, 6]),
    (1, 4, 7, 6, 6272, [6000], None), (1, 1, 1, 48, 1024, [1000], None), (70, 4, 1, 5, 64, list(range(-5, 65)), None),
    (2, 1, 48, 1, 320, [300, 0], None), (300, 1, 2, 3, 64, [b % 65 for b in range(300)], None),
    # many rows: a wave's tile, two, three; several tiles, splits; trees of several blocks, the last one begun
    (1, 1, 1, 49, 64, [50], None), (2, 2, 7, 8, 320, [320, 17], [8, 1]), (2, 1, 7, 16, 1024, [1024, 1], [16, 0]),
    (2, 2, 7, 33, 512, [400, 511], [33, 32]), (3, 1, 7, 64, 640, [640, 0, 31], [64, 40, 1]), (1, 2, 8, 100, 96, [96], None),
    (2, 1, 2, 256, 320, [320, 5], [256, 193]), (1, 1, 7, 255, 32, [0], None), (40, 4, 7, 16, 64, list(range(0, 80, 2)), None),
]


@pytest.mark.parametrize("code,dtype", [(0, F16), (1, F16), (0, BF16), (1, BF16)])
@pytest.mark.parametrize("B,H,rep,n,cap,lens,counts", SHAPES)
def test_attention(B, H, rep, n, cap, lens, counts, code, dtype):
    print(f"[case] tree attention B={B} H={H} rep={rep} n={n} cap={cap} code={code} {dtype}", flush=True)
    c = Case(B, H, rep, n, cap, lens, code, dtype, n + cap, strided=bool(n % 2))
    sees = trees(B, n, n)
    c.check(c.run(words(sees), counts), sees, counts, rows=None if B * n < 300 else (0, 1, n // 2, n - 1))


@pytest.mark.parametrize("code,dtype", [(0, F16), (1, BF16)])
@pytest.mark.parametrize("B,H,rep,n,cap,lens", [(2, 1, 7, 5, 64, [0, 40]), (2, 2, 7, 40, 96, [0, 70]), (1, 1, 1, 150, 64, [0])])
def test_any_mask(B, H, rep, n, cap, lens, code, dtype):
    """Masks that are no tree's, rows of nothing among them; bits of nodes that are not there."""
    c = Case(B, H, rep, n, cap, lens, code, dtype, 5, L=2, layer=1)
    r = np.random.default_rng(6)
    sees = [r.random((n, n)) < 0.4 for _ in range(B)]
    for s in sees:
        s[::3] = False
        s[1] = True
    full = np.stack([O.words(s) for s in sees])
    if n % 64:
        full[:, :, -1] |= ~np.uint64(0) << np.uint64(n % 64)
    counts = [n - 2] * B
    c.check(c.run(bits(full), counts), sees, counts)


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("n,rep", [(6, 1), (40, 7)])
def test_what_is_not_seen_does_not_matter(n, rep, dtype, code):
    """NaN and infinities in keys and values that a node does not see, and in rows behind the count; nodes that see them take
    them as the cache does."""
    c = Case(2, 1, rep, n, 64, [50, 0], code, dtype, 8)
    sees = [np.tril(np.ones((n, n), bool)) for _ in range(2)]
    for s in sees:
        s[:, 2] = False                                          # nobody sees node 2
        s[4:, 3] = False                                         # node 3 itself alone sees node 3
    counts = [n, n - 1]
    clean = c.run(words(sees), counts)
    c.K[:, :, 2], c.V[:, :, 2] = float("nan"), float("inf")
    c.K[1, :, n - 1:], c.V[1, :, n - 1:] = float("inf"), float("nan")
    dirty = c.run(words(sees), counts)
    assert torch.equal(clean, dirty)
    c.V[:, :, 3, ::2], c.V[:, :, 3, 1::4] = float("nan"), float("-inf")
    c.K[:, :, 3, 7] = float("nan")
    out = c.run(words(sees), counts)
    rest = [i for i in range(n) if i != 3]
    assert torch.equal(out[:, :, rest], clean[:, :, rest])
    c.check(out, sees, counts)


@pytest.mark.parametrize("v_size", [2.0 ** -14, 2.0 ** 12])
@pytest.mark.parametrize("n,rep", [(6, 7), (40, 7)])
@pytest.mark.parametrize("code,dtype", [(0, F16), (1, BF16)])
def test_values_of_other_sizes_than_the_caches(code, dtype, n, rep, v_size):
    c = Case(2, 2, rep, n, 256, [200, 7], code, dtype, 11, v_size=v_size)
    sees = trees(2, n, 3)
    c.check(c.run(words(sees)), sees, rows=(0, 3, n - 1))


@pytest.mark.parametrize("n,rep", [(6, 7), (40, 7)])
@pytest.mark.parametrize("size", [8.0, 0.01])
def test_queries_of_other_sizes(n, rep, size):
    """Sharp and flat weights: the largest scores among the drafted tokens or among the cached ones."""
    c = Case(2, 1, rep, n, 512, [500, 64], 0, F16, 12, size=size)
    sees = trees(2, n, 4)
    c.check(c.run(words(sees)), sees, rows=(0, 3, n - 1))


def test_a_cleared_cache_and_a_far_block():
    """Cached values a billion times the drafted ones, and the reverse: weights that fp16 would lose."""
    for big_cache in (False, True):
        c = Case(1, 1, 7, 8, 64, [0], 0, F16, 13)
        g = torch.Generator(device=DEV)
        g.manual_seed(1)
        V = torch.randn((1, 1, 64, 128), generator=g, device=DEV) * (60000.0 if big_cache else 2.0 ** -20)
        K = torch.randn((1, 1, 64, 128), generator=g, device=DEV)
        vk.cache8_write(c.p, 0, c.buf, K.half(), V.clamp(-65000, 65000).half(), i32([0]))
        c.lens = [64]
        sees = trees(1, 8, 2)
        c.check(c.run(words(sees)), sees)


def test_long_cache():
    """Many splits; sampled nodes."""
    print("[case] long", flush=True)
    for n, T, code, dtype in ((64, 50000, 0, F16), (3, 98000, 1, BF16)):
        c = Case(1, 4, 7, n, 98016, [T], code, dtype, 14, size=0.5)
        sees = trees(1, n, 5)
        c.check(c.run(words(sees)), sees, rows=(0, n - 1))


@pytest.mark.parametrize("n", [5, 20])
def test_a_chain_is_the_causal_attention_of_16_bit_tokens(n):
    """A chain's nodes over an empty cache: the same numbers as dense causal attention; and an empty tree changes nothing
    that is cached."""
    c = Case(2, 2, 3, n, 64, [0, 0], 0, F16, 15)
    sees = [np.tril(np.ones((n, n), bool))] * 2
    before = c.buf.clone()
    c.check(c.run(words(sees)), sees)
    assert torch.equal(before, c.buf)
    assert (c.run(words(sees), [0, 0]) == 0).all()


# ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("code,dtype", [(0, F16), (1, BF16)])
@pytest.mark.parametrize("L,B,H,n,cap,start,accepted", [
    (1, 1, 1, 1, 32, [0], [1]), (3, 2, 2, 9, 96, [31, 64], [9, 3]), (2, 4, 1, 40, 64, [0, 30, 63, -1], [40, 2, 5, 7]),
    (2, 3, 2, 256, 320, [5, 32, 300], [256, 255, 200]), (28, 2, 4, 16, 64, [17, 40], [0, 99]), (5, 1, 3, 33, 64, [7], [-2]),
])
def test_append(L, B, H, n, cap, start, accepted, code, dtype):
    """The cache's bytes are those that writing the path's rows in every layer leaves."""
    print(f"[case] append L={L} B={B} H={H} n={n}", flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    r = np.random.default_rng(n)
    mk = lambda t, s: (s * torch.randn((L, B, t, H, 128), generator=g, device=DEV)).to(dtype).transpose(2, 3)  # noqa: E731
    p = vk.make_cache8(L, B, H, H, cap, code)
    buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
    buf.fill_(0xFF)
    oldK, oldV = mk(cap, 1.0), mk(cap, 1.0)
    for layer in range(L):
        vk.cache8_write(p, layer, buf, oldK[layer], oldV[layer], i32([0] * B), i32([max(s, 0) for s in start]))
    want = buf.clone()
    K, V = mk(n, 2.0), mk(n, 2.0).contiguous()
    path = np.full((B, n), -1)
    for b in range(B):
        m = min(max(accepted[b], 0), n)
        path[b, :m] = np.sort(r.permutation(n)[:m]) if b % 2 == 0 else r.integers(0, n, m)          # (a node twice too)
    vk.cache8_append_path(p, buf, K, V, i32(path), i32(accepted), i32(start))
    rows = torch.from_numpy(np.maximum(path, 0)).to(DEV)[:, None, :, None].expand(B, H, n, 128)
    for layer in range(L):
        vk.cache8_write(p, layer, want, K[layer].gather(2, rows), V[layer].gather(2, rows), i32(start), i32(accepted))
    assert torch.equal(buf, want)


def test_append_ends_before_an_entry_that_is_no_node():
    p = vk.make_cache8(2, 3, 1, 1, 96, 0)
    K = torch.randn((2, 3, 1, 70, 128), device=DEV).half()
    path = torch.arange(70, dtype=torch.int32, device=DEV).repeat(3, 1)
    path[0, 0], path[1, 40], path[2, 5] = -1, 70, 1 << 30
    got, want = (torch.full((vk.cache8_bytes(p),), 7, dtype=torch.uint8, device=DEV) for _ in range(2))
    vk.cache8_append_path(p, got, K, K, path, i32([70, 70, 70]), i32([3, 3, 3]))
    for layer in range(2):
        vk.cache8_write(p, layer, want, K[layer], K[layer], i32([3, 3, 3]), i32([0, 40, 5]))
    assert torch.equal(got, want)


def test_a_cache_beyond_32_bits():
    """Two layers of 8 heads x 2^20 tokens, 8.6 GB: cleared, so tokens of zeros, but for the last ones of the second layer; nodes over all of
    it, and a path appended at its end.  K: 1 for zeros; V: the last tokens' alone."""
    L, H, cap, n = 4, 8, 1 << 20, 5
    p = vk.make_cache8(L, 1, H, H, cap, 0)
    buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
    buf.zero_()
    assert buf.numel() > 1 << 33
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    K, V, q = (torch.randn((1, H, t, 128), generator=g, device=DEV).half() for t in (64, 64, n))
    q *= 4.0
    vk.cache8_write(p, L - 1, buf, K, V, i32([cap - 64]))
    Kt, Vt = (torch.randn((L, 1, H, n, 128), generator=g, device=DEV).half() for _ in range(2))
    masks = torch.zeros((1, n, 1), dtype=torch.int64, device=DEV)
    vk.tree_masks(i32([[-1, 0, 0, 1, 2]]), masks)
    out = torch.empty_like(q)
    ws = vk.alloc_bytes(vk.cache8_workspace_bytes(p, n), DEV)
    vk.cache8_tree_attention(p, L - 1, buf, q, Kt[L - 1], Vt[L - 1], masks, out, i32([cap]), ws)
    Kr, Vr = (torch.empty((1, H, 64, 128), device=DEV) for _ in range(2))
    vk.cache8_read(p, L - 1, buf, i32([cap - 64]), Kr, Vr)
    sees = O.masks(n, [-1, 0, 0, 1, 2], n)[0]
    for h in range(H):
        k = np.concatenate([f64(Kr)[0, h], f64(Kt)[L - 1, 0, h]])
        v = np.concatenate([f64(Vr)[0, h], f64(Vt)[L - 1, 0, h]])
        for i in range(n):
            w = np.exp(SCALE * (k @ f64(q)[0, h, i])) * np.concatenate([np.ones(64), sees[i]])
            ref, W = (w @ v) / (w.sum() + cap - 64), (w @ np.abs(v)) / (w.sum() + cap - 64)
            # the module's bound: 2^20 weights of zeros' blocks are summed in float32, in 256 splits and waves
            tol = W * (2.0 ** -11 + 2.0 ** -10 + 2.0 ** -24 * 40000) + 2.0 ** -11 * np.abs(ref) + 2.0 ** -25
            assert (np.abs(f64(out)[0, h, i] - ref) <= tol).all(), (h, i)
    before = [buf[:1 << 20].clone(), buf[-(1 << 20):].clone()]
    vk.cache8_append_path(p, buf, Kt, Vt, i32([[0, 2, 4, -1, -1]]), i32([3]), i32([cap - 3]))
    for layer in range(L):
        back = torch.empty((1, H, 3, 128), device=DEV)
        vk.cache8_read(p, layer, buf, i32([cap - 3]), back)
        x = Kt[layer][:, :, [0, 2, 4]].float()
        a = torch.maximum(x.abs().amax(dim=(2, 3), keepdim=True), K.float()[:, :, 32:].abs().amax(dim=(2, 3), keepdim=True) if layer == L - 1 else x.new_zeros(()))
        assert ((back - x).abs() <= a * (0.5 / 127 * 1.0001)).all(), layer          # (half a step of the code)
    assert torch.equal(before[0], buf[:1 << 20])
