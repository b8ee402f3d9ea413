"""Verification on the GPU where the tried tokens have all of a draft row as it is stored: rows in 16 bits whose first entry is
rounded to 1, several entries that sum to 1 or more.  Paths and tokens have to be those of oracle/tree.py (pinned for such rows in
test_tree_draft_rows.py)."""
import numpy as np
import pytest
import torch

from oracle import tree as O
from paper_2503_16257_amd import binding as vk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def verify(target, draft, tokens, parents, uniform):
    """Children drawn without putting back; target, draft [B, n, V] on the CPU."""
    B, n, V = target.shape
    out = [torch.full((B, n), -7, dtype=torch.int32, device=DEV)] + [torch.full((B,), -7, dtype=torch.int32, device=DEV) for _ in range(2)]
    ws = vk.alloc_bytes(vk.tree_verify_workspace_bytes(B, n, V), DEV)
    ws.fill_(0xFF)
    vk.tree_verify(target.to(DEV), i32(tokens), torch.from_numpy(uniform).to(DEV), *out, ws, draft=draft.to(DEV), parents=i32(parents),
                   distinct=True)
    return [x.cpu().numpy() for x in out]


# a vocabulary that one launch takes, and one whose passes are launches of their own
@pytest.mark.parametrize("V", [50, 33001])
@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("first", [[1.0], [0.75, 0.25], [0.5, 0.5], [0.5, 0.25, 0.375]])
def test_nothing_left_of_the_draft(first, dtype, V):
    """Five children of node 0, the first of them with all of its draft row; target rows that give them little or nothing."""
    print(f"[case] verify, nothing left: {first} {dtype} V={V}", flush=True)
    r = np.random.default_rng(len(first))
    B, n = 24, 6
    target = torch.from_numpy(r.dirichlet(np.full(V, 0.5), (B, n))).to(dtype)
    draft = torch.zeros((B, n, V), dtype=dtype)
    tokens = np.stack([r.permutation(V)[:n] for _ in range(B)])
    for b in range(B):
        for i, x in enumerate(first):
            draft[b, :, tokens[b, 1 + i]] = x
        if b % 2:
            target[b, 0, tokens[b, 1:1 + len(first)]] = 0.0      # (all of them are turned down)
        if b % 3 == 0:
            draft[b, :, tokens[b, 4:]] = 2.0 ** -10                # (a rest that the row's first entries hide)
    parents = np.tile([-1, 0, 0, 0, 0, 0], (B, 1))
    uniform = r.random((B, n)).astype(np.float32)
    uniform[::4, 1:] = 0.0
    path, accepted, token = verify(target, draft, tokens, parents, uniform)
    ended = 0
    for b in range(B):
        want, x = O.verify(target[b].double().numpy(), draft[b].double().numpy(), tokens[b], parents[b], n, uniform[b].astype(np.float64), True)
        assert path[b].tolist() == want + [-1] * (n - len(want)) and accepted[b] == len(want) and token[b] == x, (b, want, path[b], x, token[b])
        ended += len(want) == 1
    assert ended >= B // 3


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_frequencies_behind_a_nearly_certain_draft(dtype):
    """200000 sequences, the draft's first token rounded to 1 in its type: how often each token comes (5 standard deviations, and what
    the stored row's sum is off by)."""
    r = np.random.default_rng(21)
    B, V = 200000 // 4, 3
    P = np.array([0.5, 0.125, 0.375])
    Q = torch.tensor([0.9985, 0.00125, 0.00025] if dtype == BF16 else [0.99985, 0.0001, 0.00005], dtype=torch.float64).to(dtype).double().numpy()
    assert Q[0] == 1.0
    got = np.zeros(V)
    for _ in range(4):
        tokens = np.zeros((B, 3), int)
        tokens[:, 1] = r.choice(V, B, p=Q / Q.sum())
        left = np.where(np.arange(V) == tokens[:, 1:2], 0.0, Q)
        tokens[:, 2] = ((left.cumsum(1) / left.sum(1, keepdims=True)) <= r.random((B, 1))).sum(1).clip(max=V - 1)
        rows = [torch.from_numpy(np.broadcast_to(x, (B, 3, V)).copy()).to(dtype) for x in (P, Q)]
        path, accepted, token = verify(*rows, tokens, np.tile([-1, 0, 0], (B, 1)), r.random((B, 3)).astype(np.float32))
        got += np.bincount(np.where(accepted > 1, tokens[np.arange(B), np.maximum(path[:, 1], 0)], token), minlength=V)
    assert (np.abs(got / (4 * B) - P) < 5 * np.sqrt(P * (1 - P) / (4 * B)) + abs(1 - 1 / Q.sum())).all(), got / (4 * B)


@pytest.mark.parametrize("top", [0.985, 0.9985])
def test_frequencies_of_rows_divided_by_their_sums(top):
    """A draft whose rows are bfloat16, as float32 rows that sum to one: 200000 sequences, 5 standard deviations."""
    r = np.random.default_rng(22)
    B, V = 50000, 3
    P = np.array([0.5, 0.1, 0.4])
    Q = torch.tensor([top, 0.8 * (1 - top), 0.2 * (1 - top)], dtype=torch.float64).bfloat16().float()
    Q = (Q / Q.sum()).double().numpy()
    got = np.zeros(V)
    for _ in range(4):
        tokens = np.zeros((B, 3), int)
        tokens[:, 1] = r.choice(V, B, p=Q / Q.sum())
        left = np.where(np.arange(V) == tokens[:, 1:2], 0.0, Q)
        tokens[:, 2] = ((left.cumsum(1) / left.sum(1, keepdims=True)) <= r.random((B, 1))).sum(1).clip(max=V - 1)
        rows = [torch.from_numpy(np.broadcast_to(x, (B, 3, V)).copy()).float() for x in (P, Q)]
        path, accepted, token = verify(*rows, tokens, np.tile([-1, 0, 0], (B, 1)), r.random((B, 3)).astype(np.float32))
        got += np.bincount(np.where(accepted > 1, tokens[np.arange(B), np.maximum(path[:, 1], 0)], token), minlength=V)
    assert (np.abs(got / (4 * B) - P) < 5 * np.sqrt(P * (1 - P) / (4 * B)) + 1e-6).all(), got / (4 * B)
