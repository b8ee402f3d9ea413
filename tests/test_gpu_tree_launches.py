"""Verification over vocabularies whose passes are launches of their own (more than 32768 tokens): what one launch leaves for the next.
Up to four launches take a pass each; trees that ask for fewer end before the last one, with the sums of an earlier one; what more they
ask for is left to the last launch.  Chains have one such launch.  Paths and tokens have to be those of oracle/tree.py."""
import numpy as np
import pytest
import torch

from oracle import tree as O
from paper_2503_16257_amd import binding as vk
from test_gpu_tree_verify import Tree, i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
RULES = ("certain", "drawn", "distinct")


def from_near_to_far(B, most):
    """How far the draft is from the target, by sequence: from equal rows on."""
    return np.linspace(0.0, most, B)[:, None, None]


def turned_down(t, b, count, parents=True):
    """Children that the walk of sequence b tries and turns down."""
    up = t.parents[b] if parents else np.arange(len(t.tokens[b])) - 1
    path, _ = O.verify(t.target[b].double().numpy(), None if t.draft is None else t.draft[b].double().numpy(), t.tokens[b], up, count,
                       t.uniform[b].astype(np.float64), t.rule == "distinct")
    return sum(1 for i in range(1, count) if up[i] in path and i not in path and
               (path.index(up[i]) + 1 == len(path) or i < path[path.index(up[i]) + 1]))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("B,n,V,branch", [(9, 3, 33001, 2), (9, 6, 40961, 3), (6, 24, 33001, 3), (3, 65, 32769, 8)])
def test_trees(B, n, V, branch, rule, dtype):
    print(f"[case] verify in launches B={B} n={n} V={V} {rule} {dtype}", flush=True)
    t = Tree(B, n, V, rule, dtype, n + V, branch, agree=from_near_to_far(B, 3.0))
    t.check(t.run())
    counts = [(5 * b) % (n + 2) for b in range(B)]               # 0 first, all and more among them
    t.check(t.run(counts), counts)
    t.uniform[::2, 1:] = 0.9999
    t.check(t.run())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rule", ["drawn", "distinct"])
def test_no_child_turned_down_to_many(rule, dtype):
    """All behind node 0: none, one, two and so on turned down, more than the launches that take a pass each."""
    print(f"[case] verify, children turned down, {rule} {dtype}", flush=True)
    B, n, V = 60, 12, 33001
    t = Tree(B, n, V, rule, dtype, 17, branch=n, agree=from_near_to_far(B, 5.0), spread=2.0)
    t.parents[:, 1:] = 0
    t.uniform[1::2, 1:] = np.float32(0.99999)
    counts = [n - b % 12 for b in range(B)]                      # 12 .. 1
    seen = {turned_down(t, b, c) for b, c in enumerate(counts)} | {turned_down(t, b, n) for b in range(B)}
    assert {0, 1, 2, 3, 4, 5} <= seen and max(seen) > 5, seen
    t.check(t.run())
    t.check(t.run(counts), counts)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("rule", RULES)
@pytest.mark.parametrize("V", [33001, 150001])
def test_chains(V, rule, dtype):
    """Drafted tokens in a row, the call without parents: one launch in front of the last."""
    print(f"[case] verify, chains V={V} {rule} {dtype}", flush=True)
    B, n = 10, 6
    t = Tree(B, n, V, rule, dtype, 23, branch=1, agree=from_near_to_far(B, 2.0))
    t.parents[:] = np.arange(n) - 1
    lengths = t.check(t.run(parents=False), parents=False)
    if rule != "certain":                                        # (a flat target's most probable token seldom stands)
        assert len(set(lengths)) > 2, lengths
        assert {turned_down(t, b, n, False) for b in range(B)} == {0, 1}
    counts = [0, 1, 2, 3, 4, 5, 6, 7, -1, 0]
    t.check(t.run(counts, parents=False), counts, parents=False)
    t.check(t.run())                                             # the same with their parents given


@pytest.mark.parametrize("rule", RULES)
def test_a_captured_call_replayed(rule):
    """New numbers and counts for every replay, a workspace of anything: the results are those of eager calls."""
    B, n, V = 8, 10, 33001
    t = Tree(B, n, V, rule, F32, 29, branch=4, agree=from_near_to_far(B, 4.0))
    target, draft = t.target.to(DEV), None if t.draft is None else t.draft.to(DEV)
    tokens, parents, uniform, count = i32(t.tokens), i32(t.parents), torch.from_numpy(t.uniform).to(DEV), i32([n] * B)
    out = [torch.full((B, n), -7, dtype=torch.int32, device=DEV)] + [torch.full((B,), -7, dtype=torch.int32, device=DEV) for _ in range(2)]
    ws = vk.alloc_bytes(vk.tree_verify_workspace_bytes(B, n, V), DEV)

    def call():
        vk.tree_verify(target, tokens, uniform, *out, ws, draft=draft, parents=parents, count=count, distinct=rule == "distinct")
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    r = np.random.default_rng(5)
    for turn in range(5):
        t.uniform[:] = r.random((B, n))
        if turn % 2:
            t.uniform[:, 1:] = 0.9999
        counts = r.integers(0, n + 1, B).tolist()
        uniform.copy_(torch.from_numpy(t.uniform))
        count.copy_(i32(counts))
        ws.fill_(17 * turn + 1)
        graph.replay()
        (target.float() ** 2).sum().item()
        t.check([x.cpu().numpy() for x in out], counts)
