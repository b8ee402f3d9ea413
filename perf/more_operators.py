"""Measured cases of the operators that check a tree of drafted tokens against the 8-bit cache.

  masks      the plan of a tree: which nodes each node sees, and their positions
  attention  the tree's queries over the cache and over the tree's own keys and values, which stay in 16 bits
  verify     which drafted tokens stand, from the target's probabilities and given random numbers, and the next token
  append     the accepted path's keys and values coded into the cache of every layer; the blocks read back

Node 0 of a tree is the last token that was sampled; the others are drafted behind it, each behind its parent.
Shapes are those of the repository's workloads (28 layers, 4 KV / 28 query heads, head_dim 128, 64 sequences of 25088
tokens, one of 196000) or generic.  With `own` false the operators are elementary torch operations; with `own`
true they are the library's calls.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
D, G = 128, 32
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
LEVEL = {"int8": 127.0, "e4m3": 448.0}
LEAST, MOST = 2.0 ** -40, 2.0 ** 40          # bounds of a block's stored magnitude
MOST_NODES = 256

_BASE = dict(kind="", B=1, n=1, ragged=False, type="f16", L=1, H=4, rep=7, T=0, code="int8", strided=False,
             width=8, axes=3, vocab=0, rule="certain", branch=2, longest=8)


def _case(**kw):
    c = dict(_BASE)
    c.update(kw)
    return c


def listed():
    return [
        # one user's tree, drafted anew for every step
        _case(name="masks_user", kind="masks", n=33),
        # a batch of trees of the most nodes, of different sizes, deep ones among them
        _case(name="masks_batch", kind="masks", B=64, n=256, ragged=True, width=3),
        # the smallest call: one head over 8 frames, eight drafted tokens
        _case(name="tree_toy", kind="attention", H=1, rep=1, T=1568, n=8),
        # one layer for one user over the 1000-frame video, 64 nodes
        _case(name="tree_long", kind="attention", T=196000, n=64),
        # one layer for 64 users with caches of their own length, small trees, e4m3 codes
        _case(name="tree_serving", kind="attention", B=64, T=25088, n=16, ragged=True, type="bf16", code="e4m3", strided=True),
        # 16 users, 8 query heads to a KV head, six nodes
        _case(name="tree_few", kind="attention", B=16, rep=8, T=6001, n=6, ragged=True, code="e4m3"),
        # two sequences with trees of the most nodes
        _case(name="tree_wide", kind="attention", B=2, T=25088, n=256, type="bf16", ragged=True),
        # five drafted tokens in a row of one user, drawn from the draft model's probabilities
        _case(name="verify_chain", kind="verify", n=6, vocab=32000, type="f32", rule="drawn", branch=1),
        # trees of the draft model's most probable tokens, 16 users, an odd vocabulary
        _case(name="verify_tree", kind="verify", B=16, n=64, vocab=150001, type="f32", rule="certain", branch=4, ragged=True),
        # trees whose siblings were drawn without putting back, 16-bit probabilities
        _case(name="verify_drawn", kind="verify", B=8, n=24, vocab=150000, type="bf16", rule="distinct", branch=3),
        # one user's accepted tokens into the caches of 28 layers
        _case(name="append_user", kind="append", L=28, T=1000, n=32, longest=6),
        # the same for 64 users at places of their own
        _case(name="append_batch", kind="append", L=28, B=64, T=500, n=64, type="bf16", code="e4m3", ragged=True, strided=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges, none dearer than the dearest listed one of its kind."""
    kind = rng.choice(["masks", "attention", "attention", "verify", "verify", "append"])
    B, n, ragged = _log_int(rng, 1, 64), _log_int(rng, 1, MOST_NODES), rng.random() < 0.6
    width = rng.choice([1, 2, 3, 8, 20])
    if kind == "masks":
        return _case(kind=kind, B=B, n=n, ragged=ragged, width=width, axes=rng.choice([1, 2, 3, 4]))
    H, rep = rng.choice([1, 2, 4, 4, 8]), rng.choice([1, 2, 4, 7, 7, 8])
    code, kind_type, strided = rng.choice(["int8", "e4m3"]), rng.choice(["f16", "bf16"]), rng.random() < 0.5
    if kind == "attention":
        T = rng.choice([0, 1, _log_int(rng, 20, 196000), _log_int(rng, 20, 196000), _log_int(rng, 20, 196000)])
        T = min(T, 64 * 4 * 25088 // (B * H), 28 * 64 * 196000 // (B * H * rep * n))
        return _case(kind=kind, B=B, H=H, rep=rep, n=n, T=T, type=kind_type, code=code, ragged=ragged, strided=strided,
                     width=width)
    if kind == "verify":
        rule = rng.choice(["certain", "drawn", "distinct"])
        vocab = _log_int(rng, 100, 150000)
        rows = 16 * 64 * 150001 if rule == "certain" else 8 * 24 * 150000
        return _case(kind=kind, B=B, n=max(1, min(n, rows // (B * vocab))), vocab=vocab, type=rng.choice(["f32", "f32", "f16", "bf16"]),
                     rule=rule, branch=rng.choice([1, 1, 2, 3, 4]), ragged=ragged)
    return _case(kind=kind, L=_log_int(rng, 1, 28), B=B, H=rng.choice([1, 2, 4, 4]), T=rng.randint(0, 500), n=min(n, 64),
                 type=kind_type, code=code, ragged=ragged, strided=strided, longest=rng.randint(1, 8))


# ---------------------------------------------------------------------------------------
# inputs: keys, values and queries as in the cases of the 8-bit cache (per channel a mean of N(0, 0.5^2) and N(0, 1) around
# it, 6 channels of a key's head with an additional 10 x Student-t); probabilities from logits of N(0, 6^2), where one token
# or a few hold most of it, the draft model's logits N(0, 1) beside them
# ---------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFF)
    return g


def _randint(g, lo, hi, shape):
    """int32 of lo .. hi."""
    return torch.randint(lo, hi + 1, shape, generator=g, device=DEV).to(torch.int32)


def _tokens(g, B, H, n, keys):
    y = torch.randn((B, H, n, D), generator=g, device=DEV)
    y += 0.5 * torch.randn((B, H, 1, D), generator=g, device=DEV)
    if keys:
        ch = torch.rand((B, H, D), generator=g, device=DEV).argsort(dim=2)[:, :, :6]
        z = torch.randn((B, H, n, 6), generator=g, device=DEV)
        e = -torch.log(torch.rand((B, H, n, 6), generator=g, device=DEV).clamp_min(1e-30))
        y.scatter_add_(3, ch[:, :, None, :].expand(B, H, n, 6), 10.0 * z / torch.sqrt(e))
    return y.clamp_(-60000.0, 60000.0)


def _laid(x, strided):
    """[..., H, n, d], in memory as it is or with the tokens outside the heads, as a projection leaves them."""
    return x.transpose(-3, -2).contiguous().transpose(-3, -2) if strided else x


def _tree(g, c):
    """Parents [B, n]: each node behind one of the `width` nodes before it."""
    B, n = c["B"], c["n"]
    i = torch.arange(n, device=DEV)
    back = (torch.rand((B, n), generator=g, device=DEV) * i.clamp(max=c["width"])).floor().long()
    return (i - 1 - back).clamp(min=-1).to(torch.int32)


def _counts(g, c):
    return _randint(g, (c["n"] + 1) // 2, c["n"], (c["B"],)) if c["ragged"] else None


def _to_bytes(r, code):
    """The 8-bit codes of values already in units of the code, to the nearest, ties to even."""
    if code == "int8":
        return torch.round(r).clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return r.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _of_bytes(b, code):
    return b.view(torch.int8).float() if code == "int8" else b.view(torch.float8_e4m3fn).float()


def _coded(g, B, H, T, cap, code, keys):
    """A cache's codes as stored bytes [B, H, cap, 128] and magnitudes [B, H, cap / 32]."""
    codes = torch.zeros((B, H, cap, D), dtype=torch.uint8, device=DEV)
    mags = torch.zeros((B, H, cap // G), dtype=torch.float32, device=DEV)
    used = -(-T // G) * G
    per = max(1, (1 << 26) // max(1, H * used * D))
    for b in range(0, B if T else 0, per):
        nb = min(per, B - b)
        x = _tokens(g, nb, H, used, keys).half().float().view(nb, H, used // G, G * D)
        a = x.abs().amax(dim=3).clamp(LEAST, MOST)
        codes[b:b + nb, :, :used] = _to_bytes(x * LEVEL[code] / a[..., None], code).view(nb, H, used, D)
        mags[b:b + nb, :, :used // G] = a
    return codes, mags


def _packed(kc, ka, vc, va):
    """The library's buffer (LAYOUT.md, 8-bit cache) with these contents."""
    B, H, cap, _ = kc.shape
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    codes, mags = up(B * H * cap * D), up(B * H * cap // G * 4)
    buf = torch.zeros(2 * codes + 2 * mags, dtype=torch.uint8, device=DEV)
    buf[:kc.numel()] = kc.reshape(-1)
    # values: [mp 4][kb 4][x 16][mh 2][half 2][i 4] is channel 32 mp + 16 mh + x of token 16 half + 4 kb + i
    v = vc.view(B * H * cap // G, 2, 4, 4, 4, 2, 16).permute(0, 4, 2, 6, 5, 1, 3)
    buf[codes:codes + vc.numel()] = v.reshape(-1)
    buf[2 * codes:2 * codes + 4 * ka.numel()] = ka.reshape(-1).view(torch.uint8)
    buf[2 * codes + mags:2 * codes + mags + 4 * va.numel()] = va.reshape(-1).view(torch.uint8)
    return buf


def _capacity(c):
    return max(G, -(-(c["T"] + (c["longest"] if c["kind"] == "append" else 0)) // G) * G)


def _words(n):
    return -(-n // 64)


def _prepare_verify(g, c, s):
    B, n, V, t = c["B"], c["n"], c["vocab"], TYPES[c["type"]]
    k, i = c["branch"], torch.arange(n, device=DEV)
    # every node has `branch` children, breadth first; with one it is a chain, and the call needs no parents
    s["parents"] = ((i - 1).div(k, rounding_mode="floor") if k > 1 else i - 1).to(torch.int32).repeat(B, 1)
    logits = 6.0 * torch.randn((B, n, V), generator=g, device=DEV)
    target = torch.softmax(logits, dim=2).to(t)
    draft = torch.softmax(logits.add_(torch.randn((B, n, V), generator=g, device=DEV)), dim=2).to(t)
    del logits
    if c["rule"] == "certain":
        chosen = draft.float().topk(min(k, V), dim=2).indices
    else:
        chosen = torch.multinomial(draft.view(B * n, V).float(), k, replacement=c["rule"] == "drawn", generator=g).view(B, n, k)
    up, rank = s["parents"].long().clamp(min=0), (i - 1).clamp(min=0) % k
    s["tokens"] = chosen[torch.arange(B, device=DEV)[:, None], up, rank].to(torch.int32)
    s["target"] = target
    s["draft"] = None if c["rule"] == "certain" else draft
    s["uniform"] = torch.rand((B, n), generator=g, device=DEV)
    s["count"] = _counts(g, c)
    s["path"] = torch.empty((B, n), dtype=torch.int32, device=DEV)
    s["accepted"] = torch.empty((B,), dtype=torch.int32, device=DEV)
    s["next"] = torch.empty((B,), dtype=torch.int32, device=DEV)


def prepare(case, seed):
    c = case
    g = _gen(seed)
    B, H, n, L = c["B"], c["H"], c["n"], c["L"]
    s = {"c": c}
    if c["kind"] == "masks":
        s["parents"], s["count"] = _tree(g, c), _counts(g, c)
        s["base"] = _randint(g, 0, 200000, (B,))
        s["masks"] = torch.empty((B, n, _words(n)), dtype=torch.int64, device=DEV)
        s["positions"] = torch.empty((c["axes"], B, n), dtype=torch.int32, device=DEV)
    elif c["kind"] == "verify":
        _prepare_verify(g, c, s)
    else:
        T, cap, t = c["T"], _capacity(c), TYPES[c["type"]]
        if c["kind"] == "attention":
            # queries small enough that a token of one of the heavy channels does not take the whole softmax
            s["q"] = _laid((0.3 * torch.randn((B, H * c["rep"], n, D), generator=g, device=DEV)).to(t), c["strided"])
            s["K"] = _laid(_tokens(g, B, H, n, True).to(t), c["strided"])
            s["V"] = _laid(_tokens(g, B, H, n, False).to(t), c["strided"])
            s["out"] = torch.empty_like(s["q"])
            s["count"] = _counts(g, c)
            s["masks"] = _masks(_tree(g, c), s["count"])[0]
            s["length"] = torch.full((B,), T, dtype=torch.int32, device=DEV)
            if c["ragged"]:
                s["length"] = _randint(g, T // 2, T, (B,))
        else:
            s["K"] = _laid(_tokens(g, L * B, H, n, True).to(t).view(L, B, H, n, D), c["strided"])
            s["V"] = _laid(_tokens(g, L * B, H, n, False).to(t).view(L, B, H, n, D), c["strided"])
            longest = min(c["longest"], n)
            s["accepted"] = _randint(g, 1, longest, (B,))
            # the nodes of a path: node 0, and others in order
            rest = torch.rand((B, n), generator=g, device=DEV).index_fill_(1, torch.zeros(1, dtype=torch.long, device=DEV), -1.0)
            keep = rest.argsort(dim=1).argsort(dim=1) < s["accepted"][:, None]
            i = torch.arange(n, device=DEV)
            order = torch.where(keep, i, n).sort(dim=1).values
            s["path"] = torch.where(order < n, order, -1).to(torch.int32)
            s["start"] = _randint(g, T // 2, T, (B,)) if c["ragged"] else torch.full((B,), T, dtype=torch.int32, device=DEV)
            s["first"] = (s["start"] // G * G).repeat(L)
            rows = longest + G - 1
            s["K_out"] = torch.empty((L * B, H, rows, D), dtype=t, device=DEV)
            s["V_out"] = torch.empty_like(s["K_out"])
        s["kc"], s["ka"] = _coded(g, L * B, H, T, cap, c["code"], True)
        s["vc"], s["va"] = _coded(g, L * B, H, T, cap, c["code"], False)
        s["cache"] = _packed(s["kc"], s["ka"], s["vc"], s["va"])
    if own:
        from paper_2503_16257_amd import binding as vk
        if c["kind"] == "verify":
            s["ws"] = vk.alloc_bytes(vk.tree_verify_workspace_bytes(B, n, c["vocab"]), DEV)
        if c["kind"] in ("attention", "append"):
            code = vk.CODE_INT8 if c["code"] == "int8" else vk.CODE_E4M3
            s["p"] = vk.make_cache8(L, B, H, H * c["rep"], _capacity(c), code=code)
        if c["kind"] == "attention":
            s["ws"] = vk.alloc_bytes(vk.cache8_workspace_bytes(s["p"], n), DEV)
        if c["kind"] == "append":
            # all layers' sequences as those of one layer, to read them back in one call
            s["all"] = vk.make_cache8(1, L * B, H, H * c["rep"], _capacity(c), code=code)
    return s


# ---------------------------------------------------------------------------------------
# the operators
# ---------------------------------------------------------------------------------------
def _masks(parents, count):
    """Bits of the nodes that each node sees [B, n, words], and its depth: the reach of a step, squared until it is
    everybody's."""
    B, n = parents.shape
    i = torch.arange(n, device=DEV)
    there = (i < (n if count is None else count[:, None])).expand(B, n)
    up = torch.where((parents >= 0) & (parents < i), parents, -1)
    reach = ((i[None, :, None] == i) | (up[:, :, None] == i)).float()
    for _ in range(max(1, (n - 1).bit_length())):
        reach = (torch.bmm(reach, reach) > 0).float()
    seen = (reach > 0) & there[:, :, None]
    seen = torch.nn.functional.pad(seen, (0, 64 * _words(n) - n)).view(B, n, _words(n), 64)
    words = (seen.long() << torch.arange(64, device=DEV)).sum(dim=3)
    return words, torch.where(there, reach.sum(dim=2).to(torch.int32) - 1, 0)


def _run_masks(s):
    if own:
        from paper_2503_16257_amd import binding as vk
        vk.tree_masks(s["parents"], s["masks"], s["base"], s["positions"], count=s["count"])
        return [s["masks"], s["positions"]]
    words, depth = _masks(s["parents"], s["count"])
    return [words, (s["base"][:, None] + depth).expand(s["c"]["axes"], -1, -1).contiguous()]


def _attention(s):
    c = s["c"]
    if own:
        from paper_2503_16257_amd import binding as vk
        vk.cache8_tree_attention(s["p"], 0, s["cache"], s["q"], s["K"], s["V"], s["masks"], s["out"], s["length"], s["ws"],
                                 count=s["count"])
        return s["out"]
    B, H, rep, n, T = c["B"], c["H"], c["rep"], c["n"], s["kc"].shape[2]
    level = LEVEL[c["code"]]
    K = (_of_bytes(s["kc"], c["code"]).view(B, H, T // G, G * D) * (s["ka"] / level)[..., None]).view(B * H, T, D)
    V = (_of_bytes(s["vc"], c["code"]).view(B, H, T // G, G * D) * (s["va"] / level)[..., None]).view(B * H, T, D)
    K = torch.cat((K, s["K"].float().reshape(B * H, n, D)), dim=1)
    V = torch.cat((V, s["V"].float().reshape(B * H, n, D)), dim=1)
    q = s["q"].float().reshape(B * H, rep * n, D)
    x = torch.bmm(q, K.transpose(1, 2).contiguous()).view(B, H * rep, n, T + n) / math.sqrt(D)
    i = torch.arange(n, device=DEV)
    there = (i < (n if s["count"] is None else s["count"][:, None])).expand(B, n)
    cached = (torch.arange(T, device=DEV) < s["length"][:, None])[:, None, :] & there[:, :, None]
    tree = ((s["masks"][:, :, i // 64] >> (i % 64)) & 1).bool() & there[:, :, None] & there[:, None, :]
    x.masked_fill_(~torch.cat((cached, tree), dim=2)[:, None], -math.inf)
    m = x.amax(dim=3, keepdim=True)
    p = x.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    z = p.sum(dim=3, keepdim=True)
    o = torch.bmm(p.view(B * H, rep * n, T + n), V).view(B, H * rep, n, D)
    return torch.where(z > 0, o / torch.where(z > 0, z, 1.0), 0.0).to(s["q"].dtype)


def _verify(s):
    c = s["c"]
    if own:
        from paper_2503_16257_amd import binding as vk
        vk.tree_verify(s["target"], s["tokens"], s["uniform"], s["path"], s["accepted"], s["next"], s["ws"], draft=s["draft"],
                       parents=s["parents"] if c["branch"] > 1 else None, count=s["count"], distinct=c["rule"] == "distinct")
        return [s["path"], s["accepted"], s["next"]]
    P, Q, tokens, r = s["target"], s["draft"], s["tokens"].long(), s["uniform"].double()
    B, n, V = P.shape
    at, i = torch.arange(B, device=DEV), torch.arange(n, device=DEV)
    up = s["parents"].long()
    count = torch.full((B,), n, device=DEV) if s["count"] is None else s["count"].long()
    same = (up[:, :, None] == up[:, None, :]) & (tokens[:, :, None] == tokens[:, None, :]) & (i[:, None] > i)
    live = (i < count[:, None]) & (tokens >= 0) & (tokens < V)
    if c["rule"] != "drawn":
        live = live & ~same.any(dim=2)          # a token that an earlier sibling had is passed over
    tokens = tokens.clamp(0, V - 1)
    u = torch.zeros(B, dtype=torch.long, device=DEV)
    a, b = torch.zeros(B, dtype=torch.float64, device=DEV), torch.ones(B, dtype=torch.float64, device=DEV)
    used = torch.zeros_like(a)                  # the draft's probability of the tokens tried
    on = count > 0
    accepted = on.to(torch.int32)
    path = torch.full((B, n), -1, dtype=torch.int32, device=DEV)
    path[:, 0] = torch.where(on, 0, -1)
    for j in range(1, n):
        x = tokens[:, j]
        tried = live[:, j] & (up[:, j] == u)
        p = P[at, u, x].double()
        if Q is None:
            good = tried & (r[:, j] * b < p)
            b = torch.where(tried & ~good, (b - p).clamp(min=0.0), b)
        else:
            q = Q[at, u, x].double()
            scale = torch.where(used < 1.0, 1.0 / (1.0 - used), 0.0) if c["rule"] == "distinct" else torch.ones_like(used)
            good = tried & (r[:, j] * (b * scale * q) < (p - a * q).clamp(min=0.0))
            bad = tried & ~good
            further = a + b * scale
            left = (P[at, u].double() - further[:, None] * Q[at, u].double()).clamp(min=0.0).sum(dim=1)
            some = bad & (left > 0.0)
            a, b = torch.where(some, further, a), torch.where(some, left, b)
            used = torch.where(bad, used + q, used)
        u = torch.where(good, j, u)
        a, b, used = torch.where(good, 0.0, a), torch.where(good, 1.0, b), torch.where(good, 0.0, used)
        path[at, torch.where(good, accepted, 0).long()] = torch.where(good, j, path[at, torch.where(good, accepted, 0).long()])
        accepted = accepted + good.to(torch.int32)
    row = P[at, u].double()
    if Q is None:
        tried = live & (up == u[:, None]) & (i > 0)
        w = torch.where(torch.zeros_like(row).scatter_add_(1, tokens, tried.double()) > 0.0, 0.0, row)
    else:
        w = (row - a[:, None] * Q[at, u].double()).clamp(min=0.0)
    w = torch.where(w.sum(dim=1, keepdim=True) > 0.0, w, row)
    total = w.cumsum(dim=1)
    over = (total > (r[:, 0] * total[:, -1])[:, None]) & (w > 0.0)
    last = (V - 1 - (w > 0.0).flip(1).to(torch.int32).argmax(dim=1))
    token = torch.where(over.any(dim=1), over.to(torch.int32).argmax(dim=1), last)
    return [path, accepted, torch.where(on, token, -1).to(torch.int32)]


def _append_plain(c, x, codes, mags, start, count):
    """Code the tokens x [N, H, n, 128] (32 bits) into a cache's arrays, in place."""
    n = x.shape[2]
    nb, cap = codes.shape[2] // G, codes.shape[2]
    level = LEVEL[c["code"]]
    blocks = start.long()[:, None] // G + torch.arange((n + 2 * G - 2) // G, device=DEV)[None, :]      # [N, w]
    t = blocks[:, :, None] * G + torch.arange(G, device=DEV)                                            # [N, w, 32]
    src = t - start.long()[:, None, None]
    new = (src >= 0) & (src < count.long()[:, None, None]) & (t < cap)
    old = (src < 0)[:, None, :, :, None]
    at = torch.arange(x.shape[0], device=DEV)[:, None]
    inside = blocks.clamp(max=nb - 1)
    y = x[at[:, :, None], :, src.clamp(0, n - 1)].permute(0, 3, 1, 2, 4)                                # [N, H, w, 32, 128]
    y = torch.where(new[:, None, :, :, None], y, 0.0)
    was = codes.view(-1, c["H"], nb, G, D)[at, :, inside].permute(0, 2, 1, 3, 4)
    a_old = torch.where(src[:, None, :, 0] < 0, mags[at, :, inside].permute(0, 2, 1), 0.0)
    a = torch.maximum(y.abs().amax(dim=(3, 4)), a_old).clamp(LEAST, MOST)
    again = _to_bytes(_of_bytes(was.contiguous(), c["code"]) * a_old[..., None, None] / a[..., None, None], c["code"])
    fresh = _to_bytes(y * level / a[..., None, None], c["code"])
    got = torch.where(new[:, None, :, :, None], fresh, torch.where(old, again, was))
    b, w = torch.nonzero(new.any(dim=2), as_tuple=True)
    codes.view(-1, c["H"], nb, G, D)[b, :, blocks[b, w]] = got[b, :, w]
    mags[b, :, blocks[b, w]] = a[b, :, w]


def _back(c, codes, mags, first, rows):
    cap = codes.shape[2]
    t = first.long()[:, None] + torch.arange(rows, device=DEV)
    at = torch.arange(codes.shape[0], device=DEV)[:, None]
    inside = t.clamp(max=cap - 1)
    v = _of_bytes(codes[at, :, inside], c["code"]) * (mags[at, :, inside // G] / LEVEL[c["code"]])[..., None]
    return torch.where((t < cap)[..., None, None], v, 0.0).transpose(1, 2)


def _append(s):
    c = s["c"]
    if own:
        from paper_2503_16257_amd import binding as vk
        vk.cache8_append_path(s["p"], s["cache"], s["K"], s["V"], s["path"], s["accepted"], s["start"])
        vk.cache8_read(s["all"], 0, s["cache"], s["first"], s["K_out"], s["V_out"])
        return [s["K_out"], s["V_out"]]
    L, B, H = c["L"], c["B"], c["H"]
    longest = min(c["longest"], c["n"])
    nodes = s["path"][:, :longest].long().clamp(min=0)[None, :, None, :, None].expand(L, B, H, longest, D)
    start, count = s["start"].repeat(L), s["accepted"].repeat(L)
    got = []
    for x, codes, mags in ((s["K"], s["kc"], s["ka"]), (s["V"], s["vc"], s["va"])):
        y = x.gather(3, nodes).float().view(L * B, H, longest, D)
        _append_plain(c, y, codes, mags, start, count)
        got.append(_back(c, codes, mags, s["first"], s["K_out"].shape[2]).to(x.dtype))
    return got


def run(state):
    return {"masks": _run_masks, "attention": _attention, "verify": _verify, "append": _append}[state["c"]["kind"]](state)


def work(case):
    """Each input read once, each output written once."""
    c = case
    B, H, n, T = c["B"], c["H"], c["n"], c["T"]
    e = 4 if c["type"] == "f32" else 2
    if c["kind"] == "masks":
        return {"bytes": B * n * (4 + 8 * _words(n) + 4 * c["axes"]) + 4 * B, "flops": B * n * _words(n)}
    if c["kind"] == "verify":
        # the last row of each sequence; two probabilities and three numbers of a node
        rows = 1 if c["rule"] == "certain" else 2
        return {"bytes": B * (c["vocab"] * e * rows + n * (8 + 2 * e + 8) + 8), "flops": 2 * rows * B * c["vocab"]}
    if c["kind"] == "append":
        longest = min(c["longest"], n)
        x = 2 * c["L"] * B * H * D * (longest + 1) / 2
        # accepted tokens in, codes out; codes in, tokens back out
        return {"bytes": e * x + x + (1 + e) * 2 * c["L"] * B * H * D * (longest + G - 1), "flops": 4 * x}
    length, nodes = (0.75 * T, 0.75 * n) if c["ragged"] else (T, n)
    rows = B * H * c["rep"] * n
    return {"bytes": 2 * B * H * (length * (D + 4 / G) + e * nodes * D) + 2 * e * rows * D + 8 * B * n * _words(n),
            "flops": 4 * D * B * H * c["rep"] * nodes * (length + min(nodes, 2 * nodes / (c["width"] + 1) + 1) / 2)}


# ---------------------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------------------
def _exact_value(b, code):
    b = b.long()
    if code == "int8":
        return torch.where(b > 127, b - 256, b).double()
    e, m = (b >> 3) & 15, (b & 7).double()
    v = torch.where(e > 0, (8 + m) * torch.exp2(e.double() - 10), m * 2.0 ** -9)
    return torch.where(b > 127, -v, v)


def _exact_code(r, code):
    """The nearest value of the code, ties to the even one."""
    if code == "int8":
        return torch.round(r).clamp(-127, 127)
    r = r.clamp(-448, 448)
    _, e = torch.frexp(r)
    step = torch.exp2((e.double() - 4).clamp(min=-9))
    return torch.round(r / step) * step


def _exact_masks(c, s):
    n = c["n"]
    words = np.zeros((c["B"], n, _words(n)), dtype=np.uint64)
    depth = np.zeros((c["B"], n), dtype=np.int64)
    parents = s["parents"].tolist()
    for b, count in enumerate([n] * c["B"] if s["count"] is None else s["count"].tolist()):
        for i in range(count):
            j, steps = i, 0
            while j >= 0:
                words[b, i, j // 64] |= np.uint64(1 << (j % 64))
                j, steps = parents[b][j], steps + 1
            depth[b, i] = steps - 1
    pos = torch.from_numpy(depth).to(DEV) + s["base"].long()[:, None]
    return [torch.from_numpy(words.view(np.int64)).to(DEV), pos.to(torch.int32).repeat(c["axes"], 1, 1)]


def _exact_attention(c, s):
    B, H, rep, n = c["B"], c["H"], c["rep"], c["n"]
    out = torch.zeros((B, H * rep, n, D), dtype=torch.float64, device=DEV)
    level = LEVEL[c["code"]]
    lengths = s["length"].tolist()
    counts = [n] * B if s["count"] is None else s["count"].tolist()
    words = s["masks"].cpu().numpy().view(np.uint64)
    for b in range(B):
        T, m = lengths[b], counts[b]
        sees = np.array([[(int(words[b, i, j // 64]) >> (j % 64)) & 1 for j in range(m)] for i in range(m)], dtype=bool).reshape(m, m)
        blind = torch.cat((torch.zeros((m, T), dtype=torch.bool, device=DEV), torch.from_numpy(~sees).to(DEV)), dim=1)
        for h in range(H if m else 0):
            unit = [s[a][b, h].double().repeat_interleave(G)[:T, None] / level for a in ("ka", "va")]
            K = torch.cat((_exact_value(s["kc"][b, h, :T], c["code"]) * unit[0], s["K"][b, h, :m].double()))
            V = torch.cat((_exact_value(s["vc"][b, h, :T], c["code"]) * unit[1], s["V"][b, h, :m].double()))
            Kt = K.t().contiguous()
            for r in range(h * rep, h * rep + rep):
                x = (s["q"][b, r, :m].double() @ Kt / math.sqrt(D)).masked_fill_(blind, -math.inf)
                e = torch.exp(x - x.amax(dim=1, keepdim=True))
                out[b, r, :m] = (e @ V) / e.sum(dim=1, keepdim=True)
    return out


def _exact_verify(c, s):
    B, n, V = c["B"], c["n"], c["vocab"]
    tokens, up = s["tokens"].tolist(), s["parents"].tolist()
    r = s["uniform"].double().tolist()
    counts = [n] * B if s["count"] is None else s["count"].tolist()
    paths, number, following = [], [], []

    def row(x, b, u):
        return x[b, u].double().cpu().numpy()

    for b in range(B):
        u, path = 0, [0]
        R, Q = row(s["target"], b, 0), None if s["draft"] is None else row(s["draft"], b, 0)
        for j in range(1, counts[b]):
            if up[b][j] != u:
                continue
            x = tokens[b][j]
            q = 1.0 if Q is None else Q[x]
            if r[b][j] * q < R[x]:
                u = j
                path.append(j)
                R, Q = row(s["target"], b, u), None if s["draft"] is None else row(s["draft"], b, u)
                continue
            if Q is None:
                left = R.copy()
                left[x] = 0.0
                R = left / (1.0 - R[x])
            else:
                left = np.maximum(R - Q, 0.0)
                R = left / left.sum()
                if c["rule"] == "distinct":
                    Q = Q.copy()
                    Q[x] = 0.0
                    Q /= 1.0 - q
        total = np.cumsum(R)
        paths.append(path + [-1] * (n - len(path)))
        number.append(len(path))
        following.append(int(np.argmax(total > r[b][0] * total[-1])))
    return [torch.tensor(x, dtype=torch.int32, device=DEV) for x in (paths, number, following)]


def _exact_append(c, s):
    L, B, H = c["L"], c["B"], c["H"]
    level, rows, cap = LEVEL[c["code"]], s["K_out"].shape[2], s["kc"].shape[2]
    got = []
    starts, counts, paths = s["start"].tolist(), s["accepted"].tolist(), s["path"].tolist()
    for x, codes, mags in ((s["K"], s["kc"], s["ka"]), (s["V"], s["vc"], s["va"])):
        out = torch.zeros((L, B, H, rows, D), dtype=torch.float64, device=DEV)
        codes, mags = codes.view(L, B, H, cap, D), mags.view(L, B, H, cap // G).double()
        for b in range(B):
            t0, m = starts[b], counts[b]
            lo, hi = t0 // G * G, min(cap, -(-(t0 + m) // G) * G)
            head, end = t0 - lo, min(cap, lo + rows)
            val = _exact_value(codes[:, b, :, lo:end], c["code"])                   # [L, H, t, 128]
            old = mags[:, b, :, lo // G:-(-end // G)]
            a = old.clone()
            live = torch.zeros((L, H, hi - lo, D), dtype=torch.float64, device=DEV)
            live[:, :, head:head + m] = x[:, b, :, paths[b][:m]].double()
            most = live.abs().view(L, H, -1, G * D).amax(dim=3)
            if head:
                most[:, :, 0] = torch.maximum(most[:, :, 0], old[:, :, 0])
            k = most.shape[2]
            a[:, :, :k] = most.clamp(LEAST, MOST)
            per = a.repeat_interleave(G, dim=2)[:, :, :end - lo, None]
            fresh = _exact_code(live * level / a[:, :, :k].repeat_interleave(G, dim=2)[..., None], c["code"])
            stop = min(head + m, end - lo)
            val[:, :, head:stop] = fresh[:, :, head:stop]
            if head:
                val[:, :, :head] = _exact_code(val[:, :, :head] * (old[:, :, 0] / a[:, :, 0])[..., None, None], c["code"])
            out[:, b, :, :end - lo] = val * per / level
        got.append(out.view(L * B, H, rows, D))
    return got


def exact(case, seed):
    s = prepare(case, seed)
    return {"masks": _exact_masks, "attention": _exact_attention, "verify": _exact_verify, "append": _exact_append}[case["kind"]](case, s)
