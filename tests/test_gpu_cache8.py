"""Writing the 8-bit cache and reading it back, against the float64 oracle.

The codes and magnitudes have to be the oracle's byte for byte: x * level and code * A_old are exact in float32, the
quotient is correct to the last bit, a quotient on the border of two codes is itself a float32 number and any other is
2^-20 of it or more away from one.  Values read back: code * (A * (1 / level)), three roundings of float32 and one to the
output's type."""
import numpy as np
import pytest
import torch

from oracle import cache8 as O
from paper_2503_16257_amd import binding as vk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def tokens(r, shape, dtype, strided=False, spread=1.0):
    x = r.standard_normal(shape) * np.exp(spread * r.standard_normal(shape[:3] + (1,)))
    x = torch.from_numpy(x).to(dtype).to(DEV)
    return x.transpose(1, 2).contiguous().transpose(1, 2) if strided else x


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def f64(t):
    return t.double().cpu().numpy()


class Cache:
    """A cache buffer full of a byte, and the same as the oracle sees it."""

    def __init__(self, L, B, H, cap, code, rep=1, fill=0xFF):
        self.p = vk.make_cache8(L, B, H, H * rep, cap, code)
        self.buf = vk.alloc_bytes(vk.cache8_bytes(self.p), DEV)
        self.buf.fill_(fill)
        self.geom = (L, B, H, cap)
        self.code = code
        self.want = [a.copy() for a in self.state()]

    def state(self):
        return O.unpack(self.buf.cpu().numpy(), *self.geom)

    def write(self, layer, K, V, start, count=None, **kw):
        vk.cache8_write(self.p, layer, self.buf, K, V, i32(start), None if count is None else i32(count), **kw)
        n = K.shape[2]
        for x, c, m in ((f64(K), self.want[0], self.want[2]), (f64(V), self.want[1], self.want[3])):
            for b, s in enumerate(start):
                k = n if count is None else min(max(count[b], 0), n)
                if k:
                    O.write(x[b], s, k, c[layer, b], m[layer, b], self.code)

    def check(self):
        for name, g, w in zip(("K codes", "V codes", "K magnitudes", "V magnitudes"), self.state(), self.want):
            np.testing.assert_array_equal(g.view(np.uint8), w.view(np.uint8), err_msg=name)


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_appends_match_oracle_byte_for_byte(code, dtype):
    """Single tokens, pieces, whole blocks, ends inside a block; magnitudes that grow and do not."""
    r = np.random.default_rng(11)
    c = Cache(2, 3, 2, 160, code)
    start = [0, 0, 0]
    for n in (1, 1, 3, 1, 26, 33, 1, 64, 30):
        print(f"[case] append {n} at {start}", flush=True)
        c.write(1, tokens(r, (3, 2, n, 128), dtype, n % 2 == 1), tokens(r, (3, 2, n, 128), dtype), start)
        start = [s + n for s in start]
    c.check()                                     # and layer 0 as it was


@pytest.mark.parametrize("code", [0, 1])
def test_ragged_overwriting_and_dropped(code):
    r = np.random.default_rng(12)
    c = Cache(1, 6, 1, 96, code, fill=0x80)
    for start, count, n in (([0, 5, 31, 32, 64, 95], [40, 0, 40, 7, 40, 3], 40),      # behind the capacity: dropped
                            ([10, 0, -1, 2 ** 31 - 1, 96, 94], [3, 1, 5, 5, 5, -7], 5),
                            ([3, 90, 17, 33, 40, 50], [99, 99, 1, 2, 99, 4], 4)):
        K, V = tokens(r, (6, 1, n, 128), F16, spread=2.0), tokens(r, (6, 1, n, 128), F16, spread=2.0)
        for b, k in enumerate(count):                                                # what is not counted is not read
            K[b, :, max(k, 0):] = float("nan")
            V[b, :, max(k, 0):] = float("inf")
        Kc, Vc = torch.nan_to_num(K, 0.0), torch.nan_to_num(V, 0.0, 0.0)
        vk.cache8_write(c.p, 0, c.buf, K, V, i32(start), i32(count))
        for x, cc, m in ((f64(Kc), c.want[0], c.want[2]), (f64(Vc), c.want[1], c.want[3])):
            for b, s in enumerate(start):
                k = min(max(count[b], 0), n)
                if k:
                    O.write(x[b], s, k, cc[0, b], m[0, b], code)
    c.check()


def test_magnitudes_at_their_bounds():
    """Zeros, values below 2^-40 and above 2^40, the smallest and largest of fp16, exact borders of codes."""
    r = np.random.default_rng(13)
    for code in (0, 1):
        c = Cache(1, 1, 5, 64, code)
        x = r.standard_normal((1, 5, 64, 128))
        x[:, 0] = 0.0
        x[:, 1] *= 2.0 ** -60
        x[:, 2] *= 2.0 ** 60
        x[:, 3, :, ::2] = 127.0
        x[:, 3, :, 1::2] = np.arange(64) + 0.5
        x[:, 4] = 448.0 * r.choice([1.0, -1.0, 2.0 ** -10, 3 * 2.0 ** -10, 17 / 448, 1.0625 * 2 ** -6], (64, 128))
        t = torch.from_numpy(x).to(BF16).to(DEV)
        c.write(0, t, -t, [0])
        c.check()
    c = Cache(1, 1, 1, 64, 0)
    t = torch.tensor([6e-8, 65504.0, -65504.0, 6.1e-5], dtype=F16, device=DEV).repeat(32 * 32).view(1, 1, 32, 128)
    c.write(0, t[:, :, :1], t[:, :, :1] * 0 + 6e-8, [0])
    c.write(0, t * 0 + 6e-8, t, [1])
    c.check()


@pytest.mark.parametrize("adjacent,rot", [(False, 128), (True, 128), (False, 64), (True, 96)])
def test_keys_turned_on_the_way(adjacent, rot):
    """The same bytes as the rotation by itself, then a write."""
    r = np.random.default_rng(14)
    pairs = rot // 2
    plan = vk.make_rotary((pairs // 4, pairs - pairs // 4), theta=1e6, rot_dim=rot, adjacent=adjacent)
    for dtype, code, n in ((F16, 0, 70), (BF16, 1, 1), (BF16, 0, 33)):
        K, V = tokens(r, (2, 4, n, 128), dtype, True), tokens(r, (2, 4, n, 128), dtype)
        pos = i32(r.integers(0, 200000, (2, 2, n)).tolist())
        Kt = torch.empty_like(K)
        vk.rotary(plan, pos, K, Kt)
        # (tokens 0..8 were never written: zeros in a cleared buffer, unspecified in another)
        a, b = Cache(1, 2, 4, 128, code, fill=0), Cache(1, 2, 4, 128, code, fill=0)
        a.write(0, Kt, V, [9, 32], [n, n - n // 2])
        a.check()
        vk.cache8_write(b.p, 0, b.buf, K, V, i32([9, 32]), i32([n, n - n // 2]), rotary=plan, positions=pos)
        assert torch.equal(a.buf, b.buf)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("code", [0, 1])
def test_read_back(code, dtype):
    r = np.random.default_rng(15)
    c = Cache(2, 4, 2, 128, code, fill=0)
    c.write(1, tokens(r, (4, 2, 128, 128), F16), tokens(r, (4, 2, 128, 128), F16), [0] * 4)
    for start, n in (([0] * 4, 128), ([5, 31, 64, 127], 1), ([-3, 100, 120, 33], 40), ([128, -40, 2 ** 31 - 1, -2 ** 31], 40)):
        K = torch.full((4, n, 2, 128), float("nan"), dtype=dtype, device=DEV).transpose(1, 2)
        V = torch.full((4, 2, n, 128), float("nan"), dtype=dtype, device=DEV)
        vk.cache8_read(c.p, 1, c.buf, i32(start), K, V)
        for got, cc, m in ((K, c.want[0], c.want[2]), (V, c.want[1], c.want[3])):
            v = O.values(cc[1], m[1], code)
            for b, s in enumerate(start):
                want = np.zeros((2, n, 128))
                lo, hi = max(s, 0), min(s + n, 128)
                if lo < hi:
                    want[:, lo - s:hi - s] = v[b, :, lo:hi]
                tol = (3 * 2.0 ** -24 + (0 if dtype == F32 else torch.finfo(dtype).eps / 2)) * np.abs(want) * 1.0001
                assert (np.abs(f64(got[b]) - want) <= tol + (2.0 ** -25 if dtype == F16 else 0)).all()
        only = torch.empty_like(V)
        vk.cache8_read(c.p, 1, c.buf, i32(start), None, only)
        assert torch.equal(only, V)


@pytest.mark.parametrize("code", [0, 1])
def test_every_code_reads_as_its_number(code):
    """All 256 bytes, at K's and at V's places, under a magnitude of the level itself (value = code) and an odd one."""
    c = Cache(1, 1, 1, 64, code)
    nb = 2 * 32 * 128
    c.buf[:2 * nb] = torch.arange(2 * nb, dtype=torch.int32, device=DEV).mul(37).to(torch.uint8)
    c.buf[2 * nb:].view(torch.float32)[:2] = torch.tensor([127.0 if code == 0 else 448.0, 3.3], device=DEV)
    c.buf[2 * nb + 256:].view(torch.float32)[:2] = torch.tensor([127.0 if code == 0 else 448.0, 2.0 ** -40], device=DEV)
    K, V = torch.empty((1, 1, 64, 128), device=DEV), torch.empty((1, 1, 64, 128), device=DEV)
    vk.cache8_read(c.p, 0, c.buf, i32([0]), K, V)
    kc, vc, km, vm = c.state()
    assert len(np.unique(kc)) == 256 and len(np.unique(vc)) == 256
    for got, cc, m in ((K, kc, km), (V, vc, vm)):
        want = O.values(cc[0, 0, 0], m[0, 0, 0], code)
        got = f64(got)[0, 0]
        np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
        ok = ~np.isnan(want)
        assert (np.abs(got - want)[ok] <= 3 * 2.0 ** -24 * np.abs(want[ok])).all()


def test_a_buffer_beyond_32_bit_offsets():
    """8.6 GB: the last layer's last sequence, codes and magnitudes."""
    L, B, H, cap = 4, 8, 8, 131200
    p = vk.make_cache8(L, B, H, H, cap, 0)
    assert vk.cache8_bytes(p) > 2 ** 33
    buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
    r = np.random.default_rng(16)
    K, V = tokens(r, (B, H, 3, 128), F16), tokens(r, (B, H, 3, 128), F16)
    start = i32([cap - 3] * B)
    buf[-(1 << 20):].zero_()
    vk.cache8_write(p, L - 1, buf, K, V, start)
    Kb, Vb = torch.empty_like(K), torch.empty_like(V)
    vk.cache8_read(p, L - 1, buf, start, Kb, Vb)
    # cap is a multiple of 32: these tokens are a block's last, whose magnitude an uncleared buffer may hold
    lo = i32([cap - 32] * B)
    vk.cache8_write(p, L - 1, buf, torch.zeros((B, H, 32, 128), dtype=F16, device=DEV),
                    torch.zeros((B, H, 32, 128), dtype=F16, device=DEV), lo)
    vk.cache8_write(p, L - 1, buf, K, V, start)
    vk.cache8_read(p, L - 1, buf, start, Kb, Vb)
    for x, y in ((K, Kb), (V, Vb)):
        a = x.abs().amax(dim=(2, 3), keepdim=True).double()
        # half a step of the code, and half a step of fp16 of a value of at most the magnitude
        assert ((x.double() - y.double()).abs() <= a * (0.5 / 127 + 2.0 ** -11)).all()


def test_refusals_of_the_binding():
    r = np.random.default_rng(17)
    c = Cache(1, 2, 3, 64, 0)
    K = tokens(r, (2, 3, 4, 128), F16)
    s = i32([0, 0])
    plan = vk.make_rotary((16, 24, 24))
    for kw in (dict(K=K[:1]), dict(K=K[:, :2]), dict(V=K[:, :, :3]), dict(K=K.double()), dict(V=K[..., ::2]),
               dict(start=s.long()), dict(start=i32([0])), dict(count=i32([0, 0, 0])), dict(start=s.cpu()),
               dict(rotary=plan), dict(positions=s), dict(rotary=plan, positions=torch.zeros((2, 2, 4), dtype=torch.int32, device=DEV)),
               dict(cache=c.buf.float())):
        a = dict(cache=c.buf, K=K, V=K, start=s) | kw
        with pytest.raises((TypeError, ValueError)):
            vk.cache8_write(c.p, 0, **a)
    with pytest.raises(vk.VidkvError):
        vk.cache8_write(c.p, 0, c.buf[:-256], K, K, s)
    with pytest.raises(vk.VidkvError):
        vk.cache8_write(c.p, 0, c.buf, K, K.to(BF16), s)
    with pytest.raises(vk.VidkvError):
        vk.cache8_write(c.p, 1, c.buf, K, K, s)
    with pytest.raises(ValueError):
        vk.cache8_read(c.p, 0, c.buf, s, K[:, :1].expand(2, 3, 4, 128), None)
    c.check()                                     # nothing was written
