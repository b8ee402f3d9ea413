"""Verification of drafted tokens on the GPU: paths and tokens have to be those of oracle/tree.py, whose literal residuals
in float64 decide as the kernels' closed form does wherever a uniform number is not within some 1e-13 of a border."""
import numpy as np
import pytest
import torch

from oracle import tree as O
from paper_2503_16257_amd import binding as vk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
RULES = ("certain", "drawn", "distinct")


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def probabilities(r, shape, spread, dtype):
    x = spread * r.standard_normal(shape)
    x = np.exp(x - x.max(axis=-1, keepdims=True))
    return torch.from_numpy(x / x.sum(axis=-1, keepdims=True)).to(dtype)


class Tree:
    """Probabilities that agree more or less, children drawn from the draft's rows."""

    def __init__(self, B, n, V, rule, dtype, seed, branch=3, agree=0.5, spread=3.0):
        r = np.random.default_rng(seed)
        self.rule = rule
        logits = spread * r.standard_normal((B, n, V))
        soft = lambda x: np.exp(x - x.max(-1, keepdims=True)) / np.exp(x - x.max(-1, keepdims=True)).sum(-1, keepdims=True)  # noqa: E731
        self.target = torch.from_numpy(soft(logits)).to(dtype)
        draft = torch.from_numpy(soft(logits + agree * r.standard_normal((B, n, V)))).to(dtype)
        self.draft = None if rule == "certain" else draft
        self.parents = np.array([[-1] + [int(r.integers(max(0, (i - 1) // branch - 1), min(i, (i - 1) // branch + 2))) for i in range(1, n)]
                                 for _ in range(B)])
        self.tokens = np.zeros((B, n), int)
        q = draft.double().numpy()
        for b in range(B):
            left = {}
            for i in range(1, n):
                u = int(self.parents[b, i])
                row = left.setdefault(u, q[b, u].copy())
                if rule == "certain":
                    x = int(row.argmax())
                else:
                    x = int(r.choice(V, p=row / row.sum())) if row.sum() > 0 else int(r.integers(0, V))
                if rule != "drawn":
                    row[x] = 0.0
                self.tokens[b, i] = x
        self.uniform = r.random((B, n)).astype(np.float32)

    def run(self, counts=None, parents=True, target=None, draft=None, stream=None):
        target = self.target.to(DEV) if target is None else target
        if self.draft is not None and draft is None:
            draft = self.draft.to(DEV)
        B, n, V = target.shape
        out = [torch.full((B, n), -7, dtype=torch.int32, device=DEV)] + [torch.full((B,), -7, dtype=torch.int32, device=DEV) for _ in range(2)]
        ws = vk.alloc_bytes(vk.tree_verify_workspace_bytes(B, n, V), DEV)
        ws.fill_(0xFF)
        vk.tree_verify(target, i32(self.tokens), torch.from_numpy(self.uniform).to(DEV), *out, ws, draft=draft,
                       parents=i32(self.parents) if parents else None, count=None if counts is None else i32(counts),
                       distinct=self.rule == "distinct", stream=stream)
        return [x.cpu().numpy() for x in out]

    def check(self, got, counts=None, parents=True):
        path, accepted, token = got
        B, n, _ = self.target.shape
        lengths = []
        for b in range(B):
            want, x = O.verify(self.target[b].double().numpy(), None if self.draft is None else self.draft[b].double().numpy(),
                               self.tokens[b], self.parents[b] if parents else None, n if counts is None else counts[b],
                               self.uniform[b].astype(np.float64), self.rule == "distinct")
            assert accepted[b] == len(want) and path[b].tolist() == want + [-1] * (n - len(want)), (b, want, path[b])
            assert token[b] == x, (b, x, token[b])
            lengths.append(len(want))
        return lengths


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("B,n,V,branch", [
    (1, 1, 1, 1), (3, 2, 2, 1), (40, 6, 7, 1), (40, 9, 64, 3), (20, 33, 1000, 3), (10, 64, 1025, 4), (6, 65, 4097, 2), (4, 130, 3001, 5),
    (3, 256, 2048, 6), (2, 256, 333, 200), (2, 12, 32000, 3),
])
def test_against_the_oracle(B, n, V, branch, rule, dtype):
    print(f"[case] verify B={B} n={n} V={V} {rule} {dtype}", flush=True)
    t = Tree(B, n, V, rule, dtype, 10 * n + V, branch)
    t.check(t.run())
    counts = [(7 * b + n) % (n + 2) for b in range(B)]
    t.check(t.run(counts), counts)


@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("agree", [0.0, 0.2, 2.0])
def test_long_paths_and_short_ones(rule, agree):
    t = Tree(60, 12, 50, rule, F32, 5, branch=1, agree=agree)
    t.parents[:] = np.arange(12) - 1
    lengths = t.check(t.run(parents=False), parents=False)
    t.check(t.run())
    if agree == 0.0 and rule != "certain":
        assert min(lengths) == 12                            # (equal rows: every token stands)


@pytest.mark.parametrize("rule", RULES)
def test_many_children_turned_down(rule):
    """All behind node 0, and the draft far from the target."""
    t = Tree(8, 100, 300, rule, F32, 6, branch=100, agree=6.0, spread=2.0)
    t.parents[:, 1:] = 0
    lengths = t.check(t.run())
    t.uniform[:, 1:] = 0.999999
    assert max(t.check(t.run())) <= max(max(lengths), 2)


@pytest.mark.parametrize("rule", RULES)
def test_tokens_and_parents_that_are_none(rule):
    t = Tree(30, 20, 40, rule, F32, 8)
    r = np.random.default_rng(1)
    t.tokens[:, 3::4] = r.choice([-1, 40, 2 ** 31 - 1, -2 ** 31], t.tokens[:, 3::4].shape)
    t.parents[:, 5::6] = r.choice([-2, 25, 19, 2 ** 31 - 1], t.parents[:, 5::6].shape)
    t.tokens[:, 2] = t.tokens[:, 1]                          # siblings with the same token
    t.parents[:, 2] = t.parents[:, 1]
    t.check(t.run())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rule", RULES)
def test_rows_where_they_lie(rule, dtype):
    """Odd vocabularies and strides: rows that begin anywhere, nodes outside the batch, one row for all."""
    t = Tree(4, 10, 2501, rule, dtype, 9)
    wide = torch.full((10, 4, 2600), float("nan"), dtype=dtype, device=DEV)
    odd = torch.full((4 * 10 * 2501 + 3,), float("nan"), dtype=dtype, device=DEV)[3:].view(4, 10, 2501)
    for a, b in ((wide.transpose(0, 1)[..., 37:2538], odd), (odd, wide.transpose(0, 1)[..., 1:2502])):
        a.copy_(t.target)
        if t.draft is not None:
            b.copy_(t.draft)
        t.check(t.run(target=a, draft=None if t.draft is None else b))
    t.target = t.target[:, :1].expand(4, 10, 2501).contiguous()
    t.check(t.run(target=t.target[:, :1].to(DEV).expand(4, 10, 2501)))


@pytest.mark.parametrize("rule", RULES)
def test_border_numbers(rule):
    """Uniform numbers at both ends: the first token that has any weight, and the last one where sums fall short."""
    for value in (0.0, float(np.nextafter(np.float32(1), np.float32(0)))):
        t = Tree(12, 8, 5000, rule, F32, 10, agree=1.0)
        t.uniform[:, 0] = value
        t.check(t.run())
        t.uniform[:] = value
        t.check(t.run())


def test_rows_without_weight():
    """Zero rows, entries below zero, a row of one token."""
    t = Tree(4, 3, 2000, "certain", F32, 11)
    t.target[0] = 0.0
    t.target[1] = -1.0
    t.target[2] = 0.0
    t.target[2, :, 1999] = 1.0
    t.target[3, :, 5::7] = -0.5
    path, accepted, token = t.run()
    t.check((path, accepted, token))
    assert token[0] == token[1] == -1 and token[2] == 1999
    t.tokens[2] = 1999                                       # it has everything, and is turned down by a number that is none
    t.uniform[2, 1:] = 1.0
    t.check(t.run())


@pytest.mark.parametrize("rule", ["drawn", "distinct"])
def test_entries_below_zero_and_nan_count_as_zero(rule):
    t = Tree(20, 8, 1500, rule, F32, 16, agree=2.0)
    want = Tree(20, 8, 1500, rule, F32, 16, agree=2.0)
    for x, bad in ((t.target, -0.25), (t.draft, -0.125)):
        x[:, :, 3::5] = bad
    for x in (want.target, want.draft):
        x[:, :, 3::5] = 0.0
    want.check(t.run())
    t.target[:, :, 4::50], want.target[:, :, 4::50] = float("nan"), 0.0
    t.draft[:, :, 4::50], want.draft[:, :, 4::50] = float("nan"), 0.0
    want.check(t.run())


@pytest.mark.parametrize("rule", ["drawn", "distinct"])
def test_equal_rows_leave_nothing(rule):
    """Target and draft are the same: whatever is turned down by a number that is none leaves the residual as it was."""
    t = Tree(6, 5, 700, rule, F32, 12, agree=0.0)
    t.draft = t.target.clone()
    t.uniform[:, 1:] = 1.0
    t.check(t.run())


def test_frequencies_of_the_next_token():
    """20000 sequences of one row: how often each token comes (5 standard deviations)."""
    r = np.random.default_rng(13)
    V, B = 6, 20000
    row = r.dirichlet(np.full(V, 0.7))
    q = r.dirichlet(np.full(V, 0.7))
    target = torch.from_numpy(row).float().to(DEV).expand(B, 3, V)
    draft = torch.from_numpy(q).float().to(DEV).expand(B, 3, V)
    tokens = r.choice(V, (B, 3), p=q)
    out = [torch.zeros((B, 3), dtype=torch.int32, device=DEV)] + [torch.zeros((B,), dtype=torch.int32, device=DEV) for _ in range(2)]
    vk.tree_verify(target, i32(tokens), torch.from_numpy(r.random((B, 3)).astype(np.float32)).to(DEV), *out,
                   vk.alloc_bytes(vk.tree_verify_workspace_bytes(B, 3, V), DEV), draft=draft, parents=i32(np.tile([-1, 0, 0], (B, 1))))
    path, accepted, token = (x.cpu().numpy() for x in out)
    first = np.where(accepted > 1, tokens[np.arange(B), np.maximum(path[:, 1], 0)], token)
    got = np.bincount(first, minlength=V) / B
    assert (np.abs(got - row) < 5 * np.sqrt(row * (1 - row) / B) + 1e-6).all()


def test_large_vocabulary():
    for rule, V in (("certain", 1 << 22), ("drawn", 150001)):
        t = Tree(1, 3, V, rule, F16 if V > 200000 else F32, 14, branch=2, spread=2.0)
        t.check(t.run())


def test_rows_beyond_32_bits():
    """Probabilities of 2.4e9 entries, 4.8 GB: the rows that a path goes by lie at both ends."""
    B, n, V = 40, 100, 600000
    target = torch.zeros((B, n, V), dtype=F16, device=DEV)
    tokens, parents = np.zeros((B, n), int), np.full((B, n), -1)
    parents[:, 50:52], parents[:, 99] = 0, 51
    tokens[:, 50], tokens[:, 51], tokens[:, 99] = 7, 599999, 300000
    target[:, 0, 599999] = 1.0
    target[:, 51, 300000] = 1.0
    target[:, 99, 123456] = 0.5
    target[:, 99, 599998] = 0.5
    u = np.full((B, n), 0.25, np.float32)
    u[1::2, 0] = 0.75
    out = [torch.zeros((B, n), dtype=torch.int32, device=DEV)] + [torch.zeros((B,), dtype=torch.int32, device=DEV) for _ in range(2)]
    vk.tree_verify(target, i32(tokens), torch.from_numpy(u).to(DEV), *out, vk.alloc_bytes(vk.tree_verify_workspace_bytes(B, n, V), DEV),
                   parents=i32(parents))
    path, accepted, token = (x.cpu().numpy() for x in out)
    assert (accepted == 3).all() and (path[:, :4] == [0, 51, 99, -1]).all()
    assert (token[::2] == 123456).all() and (token[1::2] == 599998).all()
