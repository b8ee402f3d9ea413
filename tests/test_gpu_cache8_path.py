"""The operators together as a server runs them: a prompt in pieces (turn, write, attend), then single tokens, eager, on
another stream and as a captured graph; and the 8-bit cache beside the packed one."""
import math

import numpy as np
import pytest
import torch

from oracle import cache8 as O
from paper_2503_16257_amd import binding as vk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
B, H, REP, CAP = 3, 2, 7, 320
SECTIONS = (16, 24, 24)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


class Server:
    """One layer's tensors as the projections leave them, [B, n, heads, 128]."""

    def __init__(self, code, dtype, seed=31):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        self.dtype = dtype
        self.plan = vk.make_rotary(SECTIONS, theta=1e6)
        self.p = vk.make_cache8(1, B, H, H * REP, CAP, code)
        self.buf = vk.alloc_bytes(vk.cache8_bytes(self.p), DEV)
        self.buf.fill_(0xFF)
        self.ws = vk.alloc_bytes(max(vk.cache8_workspace_bytes(self.p, n) for n in (1, 50, 100)), DEV)
        self.length = torch.zeros(B, dtype=torch.int32, device=DEV)

    def inputs(self, n):
        mk = lambda h: torch.randn((B, n, h, 128), generator=self.g, device=DEV).to(self.dtype).transpose(1, 2)  # noqa: E731
        return mk(H * REP), mk(H), mk(H)

    def positions(self, n, length=None):
        t = (self.length if length is None else length)[:, None] + torch.arange(n, device=DEV)
        return torch.stack([t // 14, t % 14 // 7, t % 7]).to(torch.int32)

    def step(self, q, k, v, pos, out, q_turned, count, after):
        vk.rotary(self.plan, pos, q, q_turned)
        vk.cache8_write(self.p, 0, self.buf, k, v, self.length, count, rotary=self.plan, positions=pos)
        vk.cache8_attention(self.p, 0, self.buf, q_turned, out, after, self.ws, q_count=count)


def expected(s, q, pos, out, count, lens):
    """Dense attention of the turned queries over what the cache reads back."""
    K, V = (torch.empty((B, H, CAP, 128), device=DEV) for _ in range(2))
    vk.cache8_read(s.p, 0, s.buf, i32([0] * B), K, V)
    K, V = K.double().cpu().numpy(), V.double().cpu().numpy()
    qt = O.rotary(q.double().cpu().numpy(), pos.cpu().numpy(), SECTIONS, 1e6)
    eps = torch.finfo(s.dtype).eps / 2
    got = out.double().cpu().numpy()
    for b in range(B):
        n = count[b]
        for h in range(H * REP):
            k, v = K[b, h // REP, :lens[b]], V[b, h // REP, :lens[b]]
            limit = lens[b] - n + 1 + np.arange(n)
            ref = O.attention(qt[b, h, :n], k, v, 1 / math.sqrt(128), limit)
            # weights: fp16's half step, and the queries' own rounding (half a step of every product) in the scores
            S = (np.abs(qt[b, h, :n]) @ np.abs(k).T).max(initial=0.0) / math.sqrt(128)
            tol = np.abs(v).max() * (2.0 ** -11 + 2 * eps * S + 2.0 ** -12) + eps * np.abs(ref)
            assert (np.abs(got[b, h, :n] - ref) <= tol).all(), (b, h)
        assert (got[b, :, n:] == 0).all()


@pytest.mark.parametrize("code,dtype", [(0, torch.float16), (1, torch.bfloat16)])
def test_prompt_then_tokens(code, dtype):
    s = Server(code, dtype)
    lens = [0] * B
    for n, count in ((100, [100, 61, 1]), (50, [50, 0, 49]), (1, [1, 1, 1]), (1, [1, 1, 0]), (1, [1, 1, 1])):
        print(f"[case] piece of {n}, {count}, after {lens}", flush=True)
        q, k, v = s.inputs(n)
        pos = s.positions(n)
        out, qt = torch.empty_like(q), torch.empty_like(q)
        lens = [a + c for a, c in zip(lens, count)]
        s.step(q, k, v, pos, out, qt, i32(count), i32(lens))
        s.length = i32(lens)
        expected(s, q, pos, out, count, lens)


def test_another_stream_gives_the_same_bits():
    outs = []
    for stream in (None, torch.cuda.Stream()):
        s = Server(0, torch.float16, seed=32)
        q, k, v = s.inputs(50)
        pos, out, qt = s.positions(50), torch.empty_like(q), torch.empty_like(q)
        n, after = i32([50] * B), i32([50] * B)
        torch.cuda.synchronize()
        kw = {} if stream is None else {"stream": stream}
        vk.rotary(s.plan, pos, q, qt, **kw)
        vk.cache8_write(s.p, 0, s.buf, k, v, s.length, n, rotary=s.plan, positions=pos, **kw)
        vk.cache8_attention(s.p, 0, s.buf, qt, out, after, s.ws, **kw)
        back = torch.empty_like(k)
        vk.cache8_read(s.p, 0, s.buf, s.length, back, **kw)
        torch.cuda.synchronize()
        outs.append((out, back, s.buf.clone()))
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_captured_steps_follow_the_lengths():
    """A graph of one decode step, replayed as the sequences grow, with eager work in between: every replay equals the
    eager call on a copy of the cache."""
    s = Server(0, torch.float16, seed=33)
    q, k, v = s.inputs(100)
    out = torch.empty_like(q)
    s.step(q, k, v, s.positions(100), out, torch.empty_like(q), i32([100, 64, 31]), i32([100, 64, 31]))
    s.length = i32([100, 64, 31])
    q, k, v = s.inputs(1)
    out, qt = torch.empty_like(q), torch.empty_like(q)
    pos, count, after = s.positions(1), i32([1] * B), s.length + 1
    s.step(q, k, v, pos, out, qt, count, after)                     # (first calls are made outside a capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step(q, k, v, pos, out, qt, count, after)
    for step in range(6):
        nq, nk, nv = s.inputs(1)
        q.copy_(nq); k.copy_(nk); v.copy_(nv)
        pos.copy_(s.positions(1))
        after.copy_(s.length + 1)
        e = Server(0, torch.float16)
        e.buf.copy_(s.buf)
        e.length = s.length.clone()
        eo, eq = torch.empty_like(q), torch.empty_like(q)
        e.step(q, k, v, pos, eo, eq, count, after)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eo) and torch.equal(s.buf, e.buf), step
        s.length.add_(1)                                            # (the graph reads this very tensor)
        (out.float() @ out.float().transpose(2, 3)).sum().item()    # the program's own work between replays


def test_keys_turned_for_the_packed_cache():
    """The rotation in front of the packed cache's quantizer: its view of a projection's output and the dense copy give the
    same packed bytes."""
    g = torch.Generator(device=DEV)
    g.manual_seed(34)
    T = 196 * 8
    k = torch.randn((1, T, 2, 128), generator=g, device=DEV).half()
    plan = vk.make_rotary(SECTIONS, theta=1e6)
    t = torch.arange(T, device=DEV)[None]
    pos = torch.stack([t // 196, t % 196 // 14, t % 14]).to(torch.int32)
    p = vk.make_params(1, 1, 2, 14, T, 16, 0)
    packed = []
    for x in (k.transpose(1, 2), k.transpose(1, 2).contiguous()):
        y = torch.empty((1, 2, T, 128), dtype=torch.float16, device=DEV)
        vk.rotary(plan, pos, x, y)
        b, ws = vk.alloc_bytes(vk.packed_keys_bytes(p)), vk.alloc_bytes(vk.workspace_bytes(p, 0))
        b.zero_()
        vk.quantize_keys(p, y[None], b, ws)
        packed.append(b)
    assert torch.equal(*packed)


def test_tensors_of_another_device_are_refused():
    """(One device here: the check is asked with a current device that the tensors are not on; the native call layer has the
    same check, and leaves what fails it to this path.)"""
    s = Server(0, torch.float16)
    q, k, v = s.inputs(1)
    real, vk._cur_device = vk._cur_device, lambda: 1
    native, vk._native = vk._native, None
    try:
        with pytest.raises(ValueError):
            vk.rotary(s.plan, s.positions(1), q, torch.empty_like(q))
        with pytest.raises(ValueError):
            vk.cache8_write(s.p, 0, s.buf, k, v, s.length)
        with pytest.raises(ValueError):
            vk.cache8_read(s.p, 0, s.buf, s.length, k, v)
        with pytest.raises(ValueError):
            vk.cache8_attention(s.p, 0, s.buf, q, torch.empty_like(q), s.length, s.ws)
    finally:
        vk._cur_device, vk._native = real, native


def test_the_same_with_and_without_the_native_call_layer():
    assert vk._native is not None
    outs = []
    native = vk._native
    for layer in (native, None):
        vk._native = layer
        try:
            s = Server(1, torch.bfloat16, seed=35)
            q, k, v = s.inputs(50)
            pos, out, qt = s.positions(50), torch.empty_like(q), torch.empty_like(q)
            kt = torch.empty((B, H, 50, 128), dtype=s.dtype, device=DEV)
            vk.rotary(s.plan, pos, q, qt, k, kt, inverse=True)
            vk.rotary(s.plan, pos, None, None, kt, kt)
            s.step(q, k, v, pos, out, qt, i32([50, 0, 49]), i32([50, 0, 49]))
            vk.cache8_attention(s.p, 0, s.buf, qt, out, i32([50, 0, 49]), s.ws, causal=False)
            back = torch.empty((B, H, 50, 128), device=DEV)
            vk.cache8_read(s.p, 0, s.buf, i32([0, 1, 2]), None, back)
            torch.cuda.synchronize()
            outs.append((qt, kt, out, back[:, :, :40], s.buf.clone()))
        finally:
            vk._native = native
    for a, b in zip(*outs):
        assert torch.equal(a.nan_to_num(7.0) if a.is_floating_point() else a, b.nan_to_num(7.0) if b.is_floating_point() else b)


def test_two_streams_at_once():
    """Calls on two streams, each with its own cache and workspace, in turn and many deep: the results of calls by themselves."""
    servers = [Server(i, torch.float16, seed=60 + i) for i in (0, 1)]
    alone, jobs = [], []
    for s in servers:
        q, k, v = s.inputs(50)
        q1, k1, v1 = s.inputs(1)
        s.length = i32([CAP - 51] * B)
        fill = torch.zeros((B, H, CAP - 51, 128), dtype=s.dtype, device=DEV)
        vk.cache8_write(s.p, 0, s.buf, fill + 0.25, fill - 0.5, i32([0] * B))
        jobs.append((q, k, v, s.positions(50), i32([50, 3, 0]), i32([CAP - 1, CAP - 48, CAP - 51])))
        out, qt = torch.empty_like(q), torch.empty_like(q)
        s.step(*jobs[-1][:4], out, qt, *jobs[-1][4:])
        alone.append((out, s.buf.clone()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in servers]
    outs = [[] for _ in servers]
    keep = []                                  # (what a side stream uses stays until both are done)
    for turn in range(8):
        for s, st, (q, k, v, pos, count, after), got in zip(servers, streams, jobs, outs):
            out, qt = torch.empty_like(q), torch.empty_like(q)
            keep.append((out, qt))
            st.wait_stream(torch.cuda.current_stream())
            vk.rotary(s.plan, pos, q, qt, stream=st)
            vk.cache8_write(s.p, 0, s.buf, k, v, s.length, count, rotary=s.plan, positions=pos, stream=st)
            vk.cache8_attention(s.p, 0, s.buf, qt, out, after, s.ws, q_count=count, stream=st)
            got.append(out)
    torch.cuda.synchronize()
    for s, (out, buf), got in zip(servers, alone, outs):
        assert all(torch.equal(out, o) for o in got) and torch.equal(s.buf, buf)


@pytest.mark.parametrize("batch,heads", [(65535, 1), (1, 65535)])
def test_the_most_sequences_and_heads(batch, heads):
    p = vk.make_cache8(1, batch, heads, heads, 32)
    buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(70)
    k, v, q = (torch.randn((batch, heads, 1, 128), generator=g, device=DEV).half() for _ in range(3))
    start = torch.zeros(batch, dtype=torch.int32, device=DEV)
    vk.cache8_write(p, 0, buf, k, v, start)
    back, out = torch.empty_like(v), torch.empty_like(q)
    vk.cache8_read(p, 0, buf, start, None, back)
    ws = vk.alloc_bytes(vk.cache8_workspace_bytes(p, 1))
    vk.cache8_attention(p, 0, buf, q, out, start + 1, ws)
    # one token: the weights are 1, and the result its value, rounded once more (2^-11 of it, and fp16's smallest)
    assert ((out.double() - back.double()).abs() <= 2.0 ** -10 * back.double().abs() + 2.0 ** -24).all()
    # half a step of the code, and of fp16
    assert ((back.double() - v.double()).abs() <= v.double().abs().amax(dim=3, keepdim=True) * (0.5 / 127 + 2.0 ** -11)).all()
    turned = torch.empty_like(q)
    plan = vk.make_rotary(SECTIONS, theta=1e6)
    if heads == 1:
        vk.rotary(plan, torch.ones((3, batch, 1), dtype=torch.int32, device=DEV), q, turned)
        vk.rotary(plan, torch.ones((3, batch, 1), dtype=torch.int32, device=DEV), turned, turned, inverse=True)
        # there and back: two roundings of each of a pair's elements
        assert ((turned.double() - q.double()).abs() <= 3 * 2.0 ** -11 * q.double().abs().amax(dim=3, keepdim=True)).all()
