"""The operators for drafted trees together, as a server runs them: masks, then in every layer rotation and attention, then
verification and the append; eager, captured, on other streams."""
import math

import numpy as np
import pytest
import torch

from oracle import cache8 as C
from oracle import tree as O
from paper_2503_16257_amd import binding as vk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
L, B, H, REP, CAP, N, V = 3, 4, 2, 7, 256, 20, 999
SECTIONS = (16, 24, 24)


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


class Server:
    """Caches of `lens` tokens, and the buffers of a step."""

    def __init__(self, code, dtype, rule, seed, lens=(0, 31, 100, 200)):
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        self.dtype, self.rule = dtype, rule
        self.plan = vk.make_rotary(SECTIONS, theta=1e6)
        self.p = vk.make_cache8(L, B, H, H * REP, CAP, code)
        self.buf = vk.alloc_bytes(vk.cache8_bytes(self.p), DEV)
        self.buf.fill_(0xFF)
        self.length = i32(lens)
        for layer in range(L):
            vk.cache8_write(self.p, layer, self.buf, self.heads(H, CAP), self.heads(H, CAP), i32([0] * B), self.length)
        self.ws = vk.alloc_bytes(vk.cache8_workspace_bytes(self.p, N), DEV)
        self.vws = vk.alloc_bytes(vk.tree_verify_workspace_bytes(B, N, V), DEV)
        self.K, self.V = (torch.zeros((L, B, H, N, 128), dtype=dtype, device=DEV) for _ in range(2))
        self.masks = torch.zeros((B, N, 1), dtype=torch.int64, device=DEV)
        self.pos = torch.zeros((3, B, N), dtype=torch.int32, device=DEV)
        self.out = torch.zeros((L, B, H * REP, N, 128), dtype=dtype, device=DEV)
        self.turned = torch.zeros((B, H * REP, N, 128), dtype=dtype, device=DEV)
        self.path, self.accepted, self.token = torch.zeros((B, N), dtype=torch.int32, device=DEV), i32([0] * B), i32([0] * B)
        self.new_inputs()

    def heads(self, h, n):
        return torch.randn((B, n, h, 128), generator=self.g, device=DEV).to(self.dtype).transpose(1, 2)

    def new_inputs(self):
        seed = int(torch.randint(0, 1 << 30, (1,), generator=self.g, device=DEV))
        r = np.random.default_rng(seed)
        new = dict(q=[self.heads(H * REP, N) for _ in range(L)], k=[self.heads(H, N) for _ in range(L)], v=[self.heads(H, N) for _ in range(L)])
        logits = 4.0 * torch.randn((B, N, V), generator=self.g, device=DEV)
        target = torch.softmax(logits, 2)
        draft = torch.softmax(logits + 0.3 * torch.randn((B, N, V), generator=self.g, device=DEV), 2)
        parents = np.array([[-1] + [max(0, (i - 1) // 2 - int(r.integers(0, 2))) for i in range(1, N)] for _ in range(B)])
        tokens = torch.zeros((B, N), dtype=torch.int32)
        q = draft.double().cpu().numpy()
        for b in range(B):
            for i in range(1, N):
                row = q[b, parents[b, i]].copy()
                for j in range(1, i):
                    if parents[b, j] == parents[b, i] and self.rule != "drawn":
                        row[int(tokens[b, j])] = 0.0
                tokens[b, i] = int(row.argmax()) if self.rule == "certain" else int(r.choice(V, p=row / row.sum()))
        new.update(target=target, draft=draft, parents=i32(parents), tokens=tokens.to(DEV), count=i32([N, N - 3, N, 7]),
                   uniform=torch.rand((B, N), generator=self.g, device=DEV))
        if not hasattr(self, "inputs"):
            self.inputs = new
        else:
            for k, x in new.items():
                for a, b in zip(self.inputs[k], x) if isinstance(x, list) else [(self.inputs[k], x)]:
                    a.copy_(b)

    def step(self, stream=None):
        x = self.inputs
        kw = {} if stream is None else {"stream": stream}
        vk.tree_masks(x["parents"], self.masks, self.length, self.pos, count=x["count"], **kw)
        for layer in range(L):
            vk.rotary(self.plan, self.pos, x["q"][layer], self.turned, x["k"][layer], self.K[layer], **kw)
            (self.V[layer].copy_(x["v"][layer]) if stream is None else self.copy(stream, self.V[layer], x["v"][layer]))
            vk.cache8_tree_attention(self.p, layer, self.buf, self.turned, self.K[layer], self.V[layer], self.masks, self.out[layer],
                                     self.length, self.ws, count=x["count"], **kw)
        vk.tree_verify(x["target"], x["tokens"], x["uniform"], self.path, self.accepted, self.token, self.vws,
                       draft=None if self.rule == "certain" else x["draft"], parents=x["parents"], count=x["count"],
                       distinct=self.rule == "distinct", **kw)
        vk.cache8_append_path(self.p, self.buf, self.K, self.V, self.path, self.accepted, self.length, **kw)

    @staticmethod
    def copy(stream, dst, src):
        with torch.cuda.stream(stream):
            dst.copy_(src)

    def results(self):
        return [x.clone() for x in (self.masks, self.pos, self.out, self.path, self.accepted, self.token, self.buf)]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("code,dtype,rule", [(0, torch.float16, "certain"), (1, torch.bfloat16, "drawn"), (1, torch.float16, "distinct")])
def test_steps_against_the_definitions(code, dtype, rule):
    s = Server(code, dtype, rule, 41)
    for turn in range(3):
        before, lens = s.buf.clone(), s.length.tolist()
        s.step()
        x = s.inputs
        parents, counts = x["parents"].cpu().numpy(), x["count"].tolist()
        kc, vc, km, vm = C.unpack(before.cpu().numpy(), L, B, H, CAP)
        out, paths = s.out.double().cpu().numpy(), []
        eps = torch.finfo(dtype).eps / 2
        for b in range(B):
            sees, depth = O.masks(N, parents[b], counts[b])
            pos = np.tile(lens[b] + depth, (3, 1, 1))
            path, token = O.verify(x["target"][b].double().cpu().numpy(), None if rule == "certain" else x["draft"][b].double().cpu().numpy(),
                                   x["tokens"][b].tolist(), parents[b], counts[b], x["uniform"][b].double().cpu().numpy(), rule == "distinct")
            paths.append(path)
            assert s.path[b].tolist() == path + [-1] * (N - len(path)) and int(s.accepted[b]) == len(path) and int(s.token[b]) == token
            for layer in range(L):
                qt = C.rotary(x["q"][layer][b:b + 1].double().cpu().numpy(), pos, SECTIONS, 1e6)[0]
                kt = C.rotary(x["k"][layer][b:b + 1].double().cpu().numpy(), pos, SECTIONS, 1e6)[0]
                vt = x["v"][layer][b].double().cpu().numpy()
                T, m = lens[b], counts[b]
                for h in range(H * REP):
                    g = h // REP
                    K = np.concatenate([C.values(kc[layer, b, g], km[layer, b, g], code)[:T], kt[g, :m]])
                    W = np.concatenate([C.values(vc[layer, b, g], vm[layer, b, g], code)[:T], vt[g, :m]])
                    ref, _ = O.attention(qt[h, :m], K, W, 1 / math.sqrt(128), np.concatenate([np.ones((m, T), bool), sees[:m, :m]], 1))
                    # weights: fp16's half step; keys and queries rounded behind their rotation, half a step each of every product
                    S = (np.abs(qt[h, :m]) @ np.abs(K).T).max() / math.sqrt(128)
                    tol = np.abs(W).max() * (2.0 ** -11 + 4 * eps * S + 2.0 ** -12) + eps * np.abs(ref)
                    assert (np.abs(out[layer, b, h, :m] - ref) <= tol).all(), (turn, b, layer, h)
                assert (out[layer, b, :, m:] == 0).all()
        # the cache is what writing the accepted rows in every layer leaves
        rows = s.path.long().clamp(min=0)[:, None, :, None].expand(B, H, N, 128)
        for layer in range(L):
            vk.cache8_write(s.p, layer, before, s.K[layer].gather(2, rows), s.V[layer].gather(2, rows), s.length, s.accepted)
        assert torch.equal(before, s.buf)
        s.length += s.accepted
        s.new_inputs()
    assert any(len(p) > 1 for p in paths)


@pytest.mark.parametrize("rule", ["certain", "drawn", "distinct"])
def test_captured_steps(rule):
    """A graph of a whole step, replayed as the sequences grow, with the program's own work in between: every replay is the
    eager step on a copy."""
    s, e = Server(0, torch.float16, rule, 42), Server(0, torch.float16, rule, 42)
    s.step()                                                     # (first calls are made outside a capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.step()
    for turn in range(5):
        s.new_inputs()
        e.new_inputs()
        e.buf.copy_(s.buf)
        e.length.copy_(s.length)
        for k in ("parents", "tokens", "uniform", "target", "draft"):
            e.inputs[k].copy_(s.inputs[k])
        for k in ("q", "k", "v"):
            for a, b in zip(e.inputs[k], s.inputs[k]):
                a.copy_(b)
        s.ws.fill_(0xFF), s.vws.fill_(0xFF), e.ws.fill_(0x11), e.vws.fill_(0x11)
        e.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert same(s.results(), e.results()), turn
        s.length.add_(s.accepted)                                # (the graph reads this very tensor)
        (s.out.float() * s.out.float()).sum().item()


def test_two_graphs_share_the_workspaces():
    """Captured with the same workspaces and replayed in turn."""
    s, t = Server(0, torch.float16, "drawn", 43), Server(0, torch.float16, "drawn", 44)
    t.ws, t.vws = s.ws, s.vws
    alone = []
    for x in (s, t):
        x.start = x.buf.clone()
        x.step()
        alone.append(x.results())
    torch.cuda.synchronize()
    graphs = []
    for x in (s, t):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            x.step()
    for turn in range(3):
        for x, graph, want in zip((s, t), graphs, alone):
            x.buf.copy_(x.start)                                 # (what was appended has re-coded the blocks that it went into)
            graph.replay()
            (x.out.float() ** 2).sum().item()
            assert same(x.results(), want), turn


def test_two_streams_at_once():
    """Each with its own buffers, in turn and many deep: the results of steps by themselves."""
    servers = [Server(i, torch.float16, "drawn", 45 + i) for i in (0, 1)]
    alone = []
    for s in servers:
        s.start = s.buf.clone()
        s.step()
        alone.append(s.results())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in servers]
    for turn in range(6):
        for s, st in zip(servers, streams):
            Server.copy(st, s.buf, s.start)
            s.step(stream=st)
    torch.cuda.synchronize()
    for s, want in zip(servers, alone):
        assert same(s.results(), want)


def test_tensors_of_another_device_are_refused():
    """(One device here: the check is asked with a current device that the tensors are not on.)"""
    s = Server(0, torch.float16, "certain", 47)
    x = s.inputs
    real, vk._cur_device = vk._cur_device, lambda: 1
    native, vk._native = vk._native, None
    try:
        for call in (lambda: vk.tree_masks(x["parents"], s.masks),
                     lambda: vk.cache8_tree_attention(s.p, 0, s.buf, s.turned, s.K[0], s.V[0], s.masks, s.out[0], s.length, s.ws),
                     lambda: vk.tree_verify(x["target"], x["tokens"], x["uniform"], s.path, s.accepted, s.token, s.vws),
                     lambda: vk.cache8_append_path(s.p, s.buf, s.K, s.V, s.path, s.accepted, s.length)):
            with pytest.raises(ValueError):
                call()
    finally:
        vk._cur_device, vk._native = real, native


def test_shapes_that_do_not_fit_are_refused():
    s = Server(0, torch.float16, "certain", 48)
    x = s.inputs
    for masks in (s.masks[:, :-1], s.masks.repeat(1, 1, 2), s.masks[:2]):
        with pytest.raises(ValueError):
            vk.cache8_tree_attention(s.p, 0, s.buf, s.turned, s.K[0], s.V[0], masks, s.out[0], s.length, s.ws)
    with pytest.raises(ValueError):
        vk.cache8_tree_attention(s.p, 0, s.buf, s.turned, s.K[0][:, :, :5], s.V[0], s.masks, s.out[0], s.length, s.ws)
    with pytest.raises(vk.VidkvError):
        vk.cache8_tree_attention(s.p, 0, s.buf, s.turned, s.K[0].bfloat16(), s.V[0], s.masks, s.out[0], s.length, s.ws)
    with pytest.raises(ValueError):
        vk.cache8_tree_attention(s.p, 0, s.buf, s.turned, s.K[0], s.V[0], s.masks, s.out[0][:1].expand(B, -1, -1, -1), s.length, s.ws)
    with pytest.raises(ValueError):
        vk.tree_verify(x["target"][:, :, ::2], x["tokens"], x["uniform"], s.path, s.accepted, s.token, s.vws)
    with pytest.raises(ValueError):
        vk.tree_verify(x["target"], x["tokens"], x["uniform"][:, :4], s.path, s.accepted, s.token, s.vws)
    with pytest.raises(vk.VidkvError):
        vk.tree_verify(x["target"], x["tokens"], x["uniform"], s.path, s.accepted, s.token, s.vws, distinct=True)
    with pytest.raises(TypeError):
        vk.tree_verify(x["target"].double(), x["tokens"], x["uniform"], s.path, s.accepted, s.token, s.vws)
    with pytest.raises(ValueError):
        vk.cache8_append_path(s.p, s.buf, s.K[:2], s.V, s.path, s.accepted, s.length)
    with pytest.raises(ValueError):
        vk.tree_masks(x["parents"], s.masks, s.length, s.pos[:, :2])


@pytest.mark.parametrize("rule", ["certain", "distinct"])
def test_the_same_with_and_without_the_native_call_layer(rule):
    assert vk._native is not None
    outs, native = [], vk._native
    for layer in (native, None):
        vk._native = layer
        try:
            s = Server(1, torch.bfloat16, rule, 49)
            s.step()
            vk.tree_masks(None, s.masks)
            outs.append(s.results())
        finally:
            vk._native = native
    assert same(*outs)


def test_workspaces_of_several_sizes():
    """What the size query says is enough, and more of it does no harm; one behind a call of more nodes neither."""
    p = vk.make_cache8(1, 1, 2, 14, 4096, 0)
    g = torch.Generator(device=DEV)
    g.manual_seed(50)
    buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
    mk = lambda h, n: torch.randn((1, h, n, 128), generator=g, device=DEV).half()  # noqa: E731
    vk.cache8_write(p, 0, buf, mk(2, 4000), mk(2, 4000), i32([0]))
    for n in (1, 7, 8, 33, 64, 100):
        q, K, V = mk(14, n), mk(2, n), mk(2, n)
        masks = torch.zeros((1, n, (n + 63) // 64), dtype=torch.int64, device=DEV)
        vk.tree_masks(None, masks)
        outs = []
        for size in (vk.cache8_workspace_bytes(p, n), vk.cache8_workspace_bytes(p, 256), 1 << 27):
            ws = torch.full((size,), 255, dtype=torch.uint8, device=DEV)
            out = torch.empty_like(q)
            vk.cache8_tree_attention(p, 0, buf, q, K, V, masks, out, i32([4000]), ws)
            outs.append(out.float())
        # the same sums in other orders: 2^-11 of weights' roundings either way, of values of some units
        assert max(float((o - outs[0]).abs().max()) for o in outs) <= 2.0 ** -9, n
