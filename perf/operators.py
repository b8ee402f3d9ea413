"""Measured cases of the operators around the 8-bit cache: rotary positions on several axes, the cache
written and read back, and the attention that reads it.

  rotary     rotate the queries and keys of a batch (or, inverse, their gradients)
  write      code new keys and values into the 8-bit cache, read the blocks that it touched back
  attention  queries over the 8-bit cache: single tokens, a few, a frame's or a whole prompt's

Shapes are those of the repository's workloads (4 KV / 28 query heads, head_dim 128, 196 tokens a frame, 64
sequences of 25088 tokens, one of 196000) or generic.  With `own` false the operators are elementary torch
operations in 32 bits; with `own` true they are the library's calls.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
D, G = 128, 32
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
LEVEL = {"int8": 127.0, "e4m3": 448.0}
LEAST, MOST = 2.0 ** -40, 2.0 ** 40          # bounds of a block's stored magnitude

_BASE = dict(kind="", B=1, H=4, rep=7, n=1, T=0, type="f16", code="int8", ragged=False, causal=True,
             rot=False, d=D, rot_dim=D, axes=3, adjacent=False, inverse=False, strided=False)


def _case(**kw):
    c = dict(_BASE)
    c.update(kw)
    return c


def listed():
    return [
        # one new token of one user: queries and keys of one layer; a launch is all it costs
        _case(name="rotary_token", kind="rotary", n=1),
        # the 32 frames of a clip, as the projections leave them (token-major), bfloat16
        _case(name="rotary_clip", kind="rotary", n=6272, type="bf16", strided=True),
        # gradients of an image encoder's heads: two axes, 80 channels, an odd number of patches, float32
        _case(name="rotary_patches_back", kind="rotary", B=3, H=16, rep=1, n=4097, type="f32", d=80, rot_dim=80,
              axes=2, inverse=True),
        # 64 users at places of their own append one token each, keys rotated on the way
        _case(name="write_token", kind="write", B=64, T=6272, n=1, ragged=True, rot=True),
        # a padded batch of short prompts that begin inside a block
        _case(name="write_ragged", kind="write", B=5, T=4000, n=1999, type="bf16", code="e4m3", ragged=True),
        # the clips of 8 users: 64 frames each
        _case(name="write_clips", kind="write", B=8, T=0, n=12544, type="f16", code="int8"),
        # the smallest decode call: one head over 8 frames
        _case(name="decode_toy", kind="attention", H=1, rep=1, T=1568),
        # one layer of a decode step over the 1000-frame video
        _case(name="decode_long", kind="attention", T=196000),
        # one layer for 64 users, lengths of their own, e4m3 codes
        _case(name="decode_serving", kind="attention", B=64, T=25088, ragged=True, type="bf16", code="e4m3"),
        # five drafted tokens of 16 users checked at once, 8 query heads to a KV head
        _case(name="draft_check", kind="attention", B=16, rep=8, n=5, T=6001, ragged=True, code="e4m3"),
        # the 196 tokens of a new frame over the video before it
        _case(name="frame_long", kind="attention", n=196, T=98196, type="bf16"),
        # a whole prompt: the clip's tokens over themselves
        _case(name="prompt_clip", kind="attention", n=6272, T=6272, type="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges, none dearer than the dearest listed one of its kind."""
    kind = rng.choice(["rotary", "write", "attention", "attention"])
    H, rep = rng.choice([1, 2, 4, 4, 8]), rng.choice([1, 2, 4, 7, 7, 8])
    B = _log_int(rng, 1, 64)
    code, ragged = rng.choice(["int8", "e4m3"]), rng.random() < 0.6
    if kind == "rotary":
        d = rng.choice([64, 80, 96, 128, 128, 128, 256])
        n = max(1, min(_log_int(rng, 1, 12544), 6272 * 32 * D // (B * H * (rep + 1) * d)))
        return _case(kind=kind, B=B, H=H, rep=rep, n=n, type=rng.choice(["f16", "bf16", "f32"]), d=d,
                     rot_dim=rng.choice([d, d, 32, d - 16]), axes=rng.choice([1, 2, 3, 3]),
                     adjacent=rng.random() < 0.3, inverse=rng.random() < 0.4, strided=rng.random() < 0.5)
    kind_type = rng.choice(["f16", "bf16"])
    if kind == "write":
        n = max(1, min(_log_int(rng, 1, 12544), 8 * 4 * 12544 // (B * H)))
        return _case(kind=kind, B=B, H=H, rep=rep, n=n, T=rng.choice([0, rng.randint(0, 4000)]), type=kind_type,
                     code=code, ragged=ragged, rot=rng.random() < 0.4, strided=rng.random() < 0.5)
    if rng.random() < 0.5:              # single tokens, or a few
        n = rng.choice([1, 1, 1, 2, 5, 8])
        T = max(n, min(_log_int(rng, 20, 196000), 64 * 4 * 25088 // (B * H)))
    else:
        n = _log_int(rng, 16, 6272)
        T = n + rng.choice([0, _log_int(rng, 1, 100000)])
        B = max(1, min(B, 8, (196 * 28 * 98196) // (n * H * rep * T)))
        T = max(n, min(T, (196 * 28 * 98196) // (n * H * rep * B)))
    return _case(kind=kind, B=B, H=H, rep=rep, n=n, T=T, type=kind_type, code=code, ragged=ragged,
                 causal=rng.random() < 0.8, strided=rng.random() < 0.5)


# ---------------------------------------------------------------------------------------
# inputs: per channel a mean of N(0, 0.5^2) and N(0, 1) around it, for keys 6 of the 128 channels of a head
# with an additional 10 x Student-t (2 degrees of freedom); queries N(0, 1), a tenth of the size for keys with such channels
# ---------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) & 0x7FFFFFFFFFFF)
    return g


def _tokens(g, B, H, n, keys):
    y = torch.randn((B, H, n, D), generator=g, device=DEV)
    y += 0.5 * torch.randn((B, H, 1, D), generator=g, device=DEV)
    if keys:
        ch = torch.rand((B, H, D), generator=g, device=DEV).argsort(dim=2)[:, :, :6]
        z = torch.randn((B, H, n, 6), generator=g, device=DEV)
        e = -torch.log(torch.rand((B, H, n, 6), generator=g, device=DEV).clamp_min(1e-30))
        y.scatter_add_(3, ch[:, :, None, :].expand(B, H, n, 6), 10.0 * z / torch.sqrt(e))
    return y.clamp_(-60000.0, 60000.0)


def _sections(c):
    """Pairs of each axis: the first has a quarter, the others share the rest (16, 24, 24 of 64 with three)."""
    pairs = c["rot_dim"] // 2
    if c["axes"] == 1:
        return [pairs]
    if c["axes"] == 2:
        return [pairs // 2, pairs - pairs // 2]
    first = pairs // 4
    second = (pairs - first) // 2
    return [first, second, pairs - first - second]


THETA = 1.0e6


def _positions(g, c, first, n):
    """[axes, B, n]: frames of 196 patches (14 x 14) that follow `first` tokens of each sequence."""
    t = first[:, None].long() + torch.arange(n, device=DEV)[None, :]
    axes = [t // 196, t % 196 // 14, t % 14] if c["axes"] == 3 else [t // 14, t % 14] if c["axes"] == 2 else [t]
    offset = torch.randint(0, 3000, (c["B"], 1), generator=g, device=DEV)
    return torch.stack([a + offset for a in axes]).to(torch.int32)


def _laid(x, strided):
    """[B, H, n, d], in memory as it is or with the tokens outside the heads, as a projection leaves them."""
    return x.transpose(1, 2).contiguous().transpose(1, 2) if strided else x


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


def _to_bytes(r, code):
    """The 8-bit codes of values already in units of the code, to the nearest, ties to even."""
    if code == "int8":
        return torch.round(r).clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return r.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _of_bytes(b, code):
    return b.view(torch.int8).float() if code == "int8" else b.view(torch.float8_e4m3fn).float()


def _packed(kc, ka, vc, va):
    """The library's buffer of one layer (LAYOUT.md, 8-bit cache) with these contents."""
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
    return -(-(c["T"] + (c["n"] if c["kind"] == "write" else 0)) // G) * G


def prepare(case, seed):
    c = case
    g = _gen(seed)
    B, H, n, t = c["B"], c["H"], c["n"], TYPES[c["type"]]
    s = {"c": c}
    if c["kind"] == "rotary":
        s["q"] = _laid(torch.randn((B, H * c["rep"], n, c["d"]), generator=g, device=DEV).to(t), c["strided"])
        s["k"] = _laid(torch.randn((B, H, n, c["d"]), generator=g, device=DEV).to(t), c["strided"])
        s["q_out"], s["k_out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        s["pos"] = _positions(g, c, torch.zeros(B, dtype=torch.int32, device=DEV), n)
    else:
        T, cap = c["T"], _capacity(c)
        if c["kind"] == "write":
            start = torch.full((B,), T, dtype=torch.int32, device=DEV)
            count = torch.full((B,), n, dtype=torch.int32, device=DEV)
            if c["ragged"]:
                start = torch.randint(T // 2, T + 1, (B,), generator=g, device=DEV).to(torch.int32)
                count = torch.randint(n - n // 2, n + 1, (B,), generator=g, device=DEV).to(torch.int32)
            s["start"], s["count"] = start, count
            s["first"] = start // G * G
            s["K"] = _laid(_tokens(g, B, H, n, True).to(t), c["strided"])
            s["V"] = _laid(_tokens(g, B, H, n, False).to(t), c["strided"])
            s["pos"] = _positions(g, c, start, n)
            rows = n + (G - 1 if T else 0)
            s["K_out"] = torch.empty((B, H, rows, D), dtype=t, device=DEV)
            s["V_out"] = torch.empty_like(s["K_out"])
        else:
            # queries small enough that a token of one of the heavy channels does not take the whole softmax
            s["q"] = _laid((0.3 * torch.randn((B, H * c["rep"], n, D), generator=g, device=DEV)).to(t), c["strided"])
            s["out"] = torch.empty_like(s["q"])
            s["length"] = torch.full((B,), T, dtype=torch.int32, device=DEV)
            if c["ragged"]:
                s["length"] = torch.randint(min(n, T // 2), T + 1, (B,), generator=g, device=DEV).to(torch.int32)
        s["kc"], s["ka"] = _coded(g, B, H, T, cap, c["code"], True)
        s["vc"], s["va"] = _coded(g, B, H, T, cap, c["code"], False)
        s["cache"] = _packed(s["kc"], s["ka"], s["vc"], s["va"])
    if own:
        from paper_2503_16257_amd import binding as vk
        if c["kind"] == "rotary" or c["rot"]:
            s["rotary"] = vk.make_rotary(_sections(c), theta=THETA, head_dim=c["d"], rot_dim=c["rot_dim"],
                                         adjacent=c["adjacent"])
        if c["kind"] != "rotary":
            code = vk.CODE_INT8 if c["code"] == "int8" else vk.CODE_E4M3
            s["p"] = vk.make_cache8(1, B, H, H * c["rep"], _capacity(c), code=code)
        if c["kind"] == "attention":
            s["ws"] = vk.alloc_bytes(vk.cache8_workspace_bytes(s["p"], n), DEV)
    return s


# ---------------------------------------------------------------------------------------
# the operators
# ---------------------------------------------------------------------------------------
def _pairs(x, rot_dim, adjacent):
    r = x[..., :rot_dim]
    return (r[..., 0::2], r[..., 1::2]) if adjacent else (r[..., :rot_dim // 2], r[..., rot_dim // 2:])


def _rotated(c, x, pos):
    """x [B, H, n, d] in 32 bits, rotated; angles in 64."""
    pairs = c["rot_dim"] // 2
    f = THETA ** (-torch.arange(pairs, dtype=torch.float64, device=DEV) / pairs)
    axis = torch.repeat_interleave(torch.arange(c["axes"], device=DEV), torch.tensor(_sections(c), device=DEV))
    a = (pos.double()[axis] * f[:, None, None]).permute(1, 2, 0)[:, None]
    co, si = torch.cos(a).float(), torch.sin(a).float()
    si = -si if c["inverse"] else si
    x1, x2 = _pairs(x, c["rot_dim"], c["adjacent"])
    y1, y2 = x1 * co - x2 * si, x2 * co + x1 * si
    y = torch.stack((y1, y2), dim=-1).flatten(-2) if c["adjacent"] else torch.cat((y1, y2), dim=-1)
    return torch.cat((y, x[..., c["rot_dim"]:]), dim=-1)


def _rotary(s):
    c = s["c"]
    if own:
        from paper_2503_16257_amd import binding as vk
        vk.rotary(s["rotary"], s["pos"], s["q"], s["q_out"], s["k"], s["k_out"], inverse=c["inverse"])
        return [s["q_out"], s["k_out"]]
    return [_rotated(c, s[x].float(), s["pos"]).to(s[x].dtype) for x in ("q", "k")]


def _append(c, x, codes, mags, start, count):
    """Code the tokens x [B, H, n, 128] (32 bits) into a cache's arrays, in place."""
    B, H, n, _ = x.shape
    nb, cap = codes.shape[2] // G, codes.shape[2]
    level = LEVEL[c["code"]]
    blocks = start.long()[:, None] // G + torch.arange((n + 2 * G - 2) // G, device=DEV)[None, :]      # [B, w]
    t = blocks[:, :, None] * G + torch.arange(G, device=DEV)                                            # [B, w, 32]
    src = t - start.long()[:, None, None]
    new = (src >= 0) & (src < count.long()[:, None, None]) & (t < cap)
    old = (src < 0)[:, None, :, :, None]
    at = torch.arange(B, device=DEV)[:, None]
    inside = blocks.clamp(max=nb - 1)
    y = x[at[:, :, None], :, src.clamp(0, n - 1)].permute(0, 3, 1, 2, 4)                                # [B, H, w, 32, 128]
    y = torch.where(new[:, None, :, :, None], y, 0.0)
    was = codes.view(B, H, nb, G, D)[at, :, inside].permute(0, 2, 1, 3, 4)
    a_old = torch.where(src[:, None, :, 0] < 0, mags[at, :, inside].permute(0, 2, 1), 0.0)
    a = torch.maximum(y.abs().amax(dim=(3, 4)), a_old).clamp(LEAST, MOST)
    again = _to_bytes(_of_bytes(was.contiguous(), c["code"]) * a_old[..., None, None] / a[..., None, None], c["code"])
    fresh = _to_bytes(y * level / a[..., None, None], c["code"])
    got = torch.where(new[:, None, :, :, None], fresh, torch.where(old, again, was))
    b, w = torch.nonzero(new.any(dim=2), as_tuple=True)
    codes.view(B, H, nb, G, D)[b, :, blocks[b, w]] = got[b, :, w]
    mags[b, :, blocks[b, w]] = a[b, :, w]


def _back(c, codes, mags, first, rows):
    cap = codes.shape[2]
    t = first.long()[:, None] + torch.arange(rows, device=DEV)
    at = torch.arange(codes.shape[0], device=DEV)[:, None]
    inside = t.clamp(max=cap - 1)
    v = _of_bytes(codes[at, :, inside], c["code"]) * (mags[at, :, inside // G] / LEVEL[c["code"]])[..., None]
    return torch.where((t < cap)[..., None, None], v, 0.0).transpose(1, 2)


def _write(s):
    c = s["c"]
    if own:
        from paper_2503_16257_amd import binding as vk
        vk.cache8_write(s["p"], 0, s["cache"], s["K"], s["V"], s["start"], count=s["count"],
                        rotary=s.get("rotary"), positions=s["pos"] if c["rot"] else None)
        vk.cache8_read(s["p"], 0, s["cache"], s["first"], s["K_out"], s["V_out"])
        return [s["K_out"], s["V_out"]]
    K, V = s["K"].float(), s["V"].float()
    if c["rot"]:
        K = _rotated(c, K, s["pos"]).to(s["K"].dtype).float()
    _append(c, K, s["kc"], s["ka"], s["start"], s["count"])
    _append(c, V, s["vc"], s["va"], s["start"], s["count"])
    rows = s["K_out"].shape[2]
    return [_back(c, s["kc"], s["ka"], s["first"], rows).to(s["K"].dtype),
            _back(c, s["vc"], s["va"], s["first"], rows).to(s["V"].dtype)]


def _attention(s):
    c = s["c"]
    if own:
        from paper_2503_16257_amd import binding as vk
        vk.cache8_attention(s["p"], 0, s["cache"], s["q"], s["out"], s["length"], s["ws"], causal=c["causal"])
        return s["out"]
    B, H, rep, n, T = c["B"], c["H"], c["rep"], c["n"], s["kc"].shape[2]
    level = LEVEL[c["code"]]
    K = (_of_bytes(s["kc"], c["code"]).view(B, H, T // G, G * D) * (s["ka"] / level)[..., None]).view(B * H, T, D)
    V = (_of_bytes(s["vc"], c["code"]).view(B, H, T // G, G * D) * (s["va"] / level)[..., None]).view(B * H, T, D)
    q = s["q"].float().reshape(B * H, rep * n, D)
    x = torch.bmm(q, K.transpose(1, 2).contiguous()).view(B, H * rep, n, T) / math.sqrt(D)
    i, t = torch.arange(n, device=DEV), torch.arange(T, device=DEV)
    limit = s["length"][:, None] - (n - 1 - i if c["causal"] else torch.zeros_like(i))[None, :]           # [B, n]
    seen = t[None, None, :] < limit[..., None]
    x.masked_fill_(~seen[:, None], -math.inf)
    m = x.amax(dim=3, keepdim=True)
    p = x.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
    z = p.sum(dim=3, keepdim=True)
    o = torch.bmm(p.view(B * H, rep * n, T), V).view(B, H * rep, n, D)
    return torch.where(z > 0, o / torch.where(z > 0, z, 1.0), 0.0).to(s["q"].dtype)


def run(state):
    kind = state["c"]["kind"]
    return _rotary(state) if kind == "rotary" else _write(state) if kind == "write" else _attention(state)


def work(case):
    """Each input read once, each output written once."""
    c = case
    B, H, n, T = c["B"], c["H"], c["n"], c["T"]
    e = 4 if c["type"] == "f32" else 2
    if c["kind"] == "rotary":
        x = B * n * H * (c["rep"] + 1)
        return {"bytes": 2 * e * x * c["d"] + 4 * c["axes"] * B * n, "flops": 3 * x * c["rot_dim"]}
    if c["kind"] == "write":
        x = 2 * B * H * D * n * (0.75 if c["ragged"] else 1.0)
        # new tokens in, codes out; codes in, tokens back out
        back = 2 * B * H * D * (n + (G - 1 if T else 0))
        return {"bytes": e * x + x + (1 + e) * back, "flops": 4 * x}
    rows = B * H * c["rep"] * n
    length = T * (0.75 if c["ragged"] else 1.0)
    seen = length - (n - 1) / 2 if c["causal"] else length
    return {"bytes": 2 * B * H * length * (D + 4 / G) + 2 * e * rows * D, "flops": 4 * D * rows * max(seen, 1)}


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


def _exact_rotated(c, x, pos):
    out = x.clone()
    half, col = c["rot_dim"] // 2, 0
    for axis, size in enumerate(_sections(c)):
        for i in range(col, col + size):
            a = pos[axis].double() * math.exp(-math.log(THETA) * i / half)
            co, si = torch.cos(a)[:, None], torch.sin(a)[:, None]
            if c["inverse"]:
                si = -si
            u, v = (2 * i, 2 * i + 1) if c["adjacent"] else (i, half + i)
            out[..., u] = x[..., u] * co - x[..., v] * si
            out[..., v] = x[..., v] * co + x[..., u] * si
        col += size
    return out


def _exact_write(c, x, codes, mags, start, count, rows):
    B, H, cap, _ = codes.shape
    level = LEVEL[c["code"]]
    out = torch.zeros((B, H, rows, D), dtype=torch.float64, device=DEV)
    for b in range(B):
        t0, m = int(start[b]), int(count[b])
        lo = t0 // G * G
        hi = min(cap, -(-(t0 + m) // G) * G)
        head = t0 - lo
        val = _exact_value(codes[b, :, lo:hi], c["code"])                       # [H, t, 128]
        live = torch.zeros((H, hi - lo, D), dtype=torch.float64, device=DEV)
        live[:, head:head + m] = x[b, :, :hi - t0][:, :m]
        a = live.abs().view(H, -1, G * D).amax(dim=2)
        before = mags[b, :, lo // G].double()
        if head:
            a[:, 0] = torch.maximum(a[:, 0], before)
        a = a.clamp(LEAST, MOST)
        per = a.repeat_interleave(G, dim=1)[..., None]
        val[:, head:head + m] = _exact_code(live * level / per, c["code"])[:, head:head + m]
        if head:
            val[:, :head] = _exact_code(val[:, :head] * before[:, None, None] / a[:, 0, None, None], c["code"])
        k = min(rows, hi - lo)
        out[b, :, :k] = (val * per / level)[:, :k]
        if rows > k:
            end = min(cap, lo + rows)
            rest = _exact_value(codes[b, :, hi:end], c["code"]) / level
            out[b, :, k:k + end - hi] = rest * mags[b, :, hi // G:-(-end // G)].double().repeat_interleave(G, dim=1)[:, :end - hi, None]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["kind"] == "rotary":
        return [_exact_rotated(c, s[x].double(), s["pos"]) for x in ("q", "k")]
    if c["kind"] == "write":
        K = s["K"].double()
        if c["rot"]:
            K = _exact_rotated(c, K, s["pos"]).to(s["K"].dtype).double()
        rows = s["K_out"].shape[2]
        return [_exact_write(c, K, s["kc"], s["ka"], s["start"], s["count"], rows),
                _exact_write(c, s["V"].double(), s["vc"], s["va"], s["start"], s["count"], rows)]
    B, H, rep, n = c["B"], c["H"], c["rep"], c["n"]
    out = torch.zeros((B, H * rep, n, D), dtype=torch.float64, device=DEV)
    level = LEVEL[c["code"]]
    lengths = s["length"].tolist()
    for b in range(B):
        T = lengths[b]
        for h in range(H if T else 0):
            unit = [s[a][b, h].double().repeat_interleave(G)[:T, None] / level for a in ("ka", "va")]
            K = _exact_value(s["kc"][b, h, :T], c["code"]) * unit[0]
            V = _exact_value(s["vc"][b, h, :T], c["code"]) * unit[1]
            Kt = K.t().contiguous()
            for r in range(h * rep, h * rep + rep):
                x = s["q"][b, r].double() @ Kt / math.sqrt(D)
                if c["causal"]:
                    last = T - n + torch.arange(n, device=DEV)
                    x.masked_fill_(torch.arange(T, device=DEV)[None, :] > last[:, None], -math.inf)
                e = torch.exp(x - x.amax(dim=1, keepdim=True))
                y = (e @ V) / e.sum(dim=1, keepdim=True)
                out[b, r] = torch.where(torch.isnan(y), 0.0, y)
    return out
