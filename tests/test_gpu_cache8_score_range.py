"""Scores whose factors lie far apart: queries, keys and scales of any size, scores below 2^24.

Each row's scores are two numbers, x for tokens with a key of K0 in channel 1 and 0 for the others, so that the weights are
2^(x log2 e) : 1.  Tolerance against those, with values of 1 and -1 (u = 2^-24): a weight is off by ln 2 of its exponent's error, 8 u
|x| log2 e + 4 u 48, and exp2's and log2's 2^-22 each, rounded to fp16 above and below: the result, at most 1, by 2^-10 + 2^-20 + that, and by its own
rounding.  (The key's code is 127 of 127 or 448 of 448, and exact.)"""
import math

import pytest
import torch

from paper_2503_16257_amd import binding as vk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16 = torch.float16, torch.bfloat16


@pytest.mark.parametrize("code", [0, 1])
@pytest.mark.parametrize("dtype,scale,key,query,heavy", [
    (BF16, 2.0 ** -4, 2.0 ** -40, 2.0 ** 43, 2.0 ** 70),          # beside an element 2^27 times as large, where keys are zero
    (BF16, 2.0 ** -4, 2.0 ** -40, 2.0 ** 44, 0.0),
    (BF16, 2.0 ** -90, 2.0 ** -20, 2.0 ** 110, 2.0 ** 120),
    (F16, 2.0 ** 60, 2.0 ** -38, 2.0 ** -22, 0.0),                # a large scale, small queries and keys
    (F16, 2.0 ** 60, 2.0 ** -40, 2.0 ** -20, 1.0),
    (F16, 2.0 ** -20, 2.0 ** 6, 2.0 ** 14, 0.0),
])
@pytest.mark.parametrize("rep,n,cap", [(2, 1, 64), (7, 5, 64), (2, 40, 64), (7, 40, 2048)])
def test_factors_far_apart(rep, n, cap, dtype, scale, key, query, heavy, code):
    print(f"[case] rep={rep} n={n} cap={cap} {dtype} scale={scale} key={key} query={query} heavy={heavy} code={code}", flush=True)
    p = vk.make_cache8(1, 1, 1, rep, cap, code, softmax_scale=scale)
    buf = vk.alloc_bytes(vk.cache8_bytes(p), DEV)
    K = torch.zeros((1, 1, cap, 128), device=DEV)
    K[:, :, ::2, 1] = key
    V = torch.ones((1, 1, cap, 128), device=DEV)
    V[:, :, 1::2] = -1.0
    vk.cache8_write(p, 0, buf, K.bfloat16(), V.bfloat16(), torch.zeros(1, dtype=torch.int32, device=DEV))
    q = torch.zeros((1, rep, n, 128), dtype=dtype, device=DEV)
    q[..., 0] = heavy
    q[..., 1] = query
    q[:, 1:, :, 1] *= -0.5
    out = torch.empty_like(q)
    ws = vk.alloc_bytes(vk.cache8_workspace_bytes(p, n), DEV)
    vk.cache8_attention(p, 0, buf, q, out, torch.full((1,), cap, dtype=torch.int32, device=DEV), ws, causal=False)
    for h in range(rep):
        x = scale * key * query * (1.0 if h == 0 else -0.5)
        want = math.tanh(x / 2)
        tol = 2.0 ** -10 + 2.0 ** -20 + math.log(2) * 2.0 ** -24 * (8 * abs(x) * math.log2(math.e) + 200) + torch.finfo(dtype).eps / 2
        err = (out[:, h].double() - want).abs().max().item()
        assert err <= tol, (h, x, want, err, tol)
