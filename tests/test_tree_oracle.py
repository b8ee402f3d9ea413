"""The trees of drafted tokens in float64 (CPU): masks by hand and by matrix powers, attention against torch, and the
verification's promise - that a token comes out with the target's probability - by summing over everything that can happen."""
import itertools

import numpy as np
import pytest
import torch

from oracle import tree as O


def test_masks_by_hand():
    #       0
    #      1 2
    #     3   4
    sees, depth = O.masks(6, [-1, 0, 0, 1, 2, -1], 5)
    want = {0: [0], 1: [0, 1], 2: [0, 2], 3: [0, 1, 3], 4: [0, 2, 4], 5: []}
    assert [list(np.flatnonzero(r)) for r in sees] == list(want.values())
    assert depth.tolist() == [0, 1, 1, 2, 2, 0]
    assert O.words(sees)[:, 0].tolist() == [1, 3, 5, 11, 21, 0]


def test_masks_are_the_powers_of_the_parents():
    r = np.random.default_rng(3)
    n = 90
    parents = [-1] + [int(r.integers(0, i)) for i in range(1, n)]
    step = np.eye(n) + np.array([[float(parents[i] == j) for j in range(n)] for i in range(n)])
    assert (O.masks(n, parents, n)[0] == (np.linalg.matrix_power(step, n) > 0)).all()
    w = O.words(O.masks(n, parents, n)[0])
    assert w.shape == (n, 2) and all((int(w[i, j // 64]) >> (j % 64)) & 1 == (j in (i, parents[i]) or O.masks(n, parents, n)[0][i, j])
                                     for i, j in ((89, 89), (89, 70), (70, 64), (5, 0)))


def test_parents_that_are_no_earlier_node_are_none():
    sees, depth = O.masks(4, [3, 0, 2, -7], 9)
    assert [list(np.flatnonzero(x)) for x in sees] == [[0], [0, 1], [2], [3]] and depth.tolist() == [0, 1, 0, 0]
    assert [list(np.flatnonzero(x)) for x in O.masks(3, None, 3)[0]] == [[0], [0, 1], [0, 1, 2]]


def test_attention_against_torch():
    r = np.random.default_rng(4)
    q, K, V = r.standard_normal((5, 128)), r.standard_normal((20, 128)), r.standard_normal((20, 128))
    sees = r.random((5, 20)) < 0.5
    sees[2] = False
    out, W = O.attention(q, K, V, 0.1, sees)
    ref = torch.nn.functional.scaled_dot_product_attention(*(torch.from_numpy(x)[None] for x in (q, K, V)), scale=0.1,
                                                           attn_mask=torch.from_numpy(sees)[None])[0].numpy()
    keep = [0, 1, 3, 4]
    assert np.abs(out[keep] - ref[keep]).max() < 1e-14 and (out[2] == 0).all() and (W >= np.abs(out) - 1e-15).all()


def probability_of_each(P, Q, children, distinct):
    """Of the tokens behind a node: that a child stands with it, or that it is the next token, over the uniform numbers."""
    out = np.zeros(P.size)
    R, q, alive, had = P.copy(), Q, 1.0, set()
    for x in children:
        if x in had and (Q is None or distinct):
            continue
        had.add(x)
        stands, after, q_after = O.turned_down(R, q, x, distinct)
        out[x] += alive * stands
        alive *= 1.0 - stands
        R, q = after, q_after
    return out + alive * (R / R.sum() if R.sum() > 0 else 0.0)


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("k", [1, 2, 3])
@pytest.mark.parametrize("rule", ["certain", "drawn", "distinct"])
def test_tokens_come_out_with_the_targets_probabilities(rule, k, seed):
    r = np.random.default_rng(100 * k + seed)
    V = 4
    P, Q = r.dirichlet(np.full(V, 0.6)), r.dirichlet(np.full(V, 0.6))
    if rule == "certain":
        total = probability_of_each(P, None, list(r.integers(0, V, k)), False)
    else:
        total = np.zeros(V)
        for drawn in itertools.product(range(V), repeat=k):
            left, chance = Q.copy(), 1.0
            for x in drawn:
                chance *= left[x] / left.sum() if left.sum() > 0 else 0.0
                if rule == "distinct":
                    left[x] = 0.0
            if chance > 0:
                total += chance * probability_of_each(P, Q, drawn, rule == "distinct")
    assert np.abs(total - P).max() < 1e-12


@pytest.mark.parametrize("rule", ["certain", "drawn", "distinct"])
def test_verify_takes_these_steps(rule):
    """The walk over many uniform numbers: every decision's rate is the probability of that step (4 standard deviations)."""
    r = np.random.default_rng(7)
    V, n, runs = 5, 4, 20000
    P = r.dirichlet(np.full(V, 0.8), n)
    Q = None if rule == "certain" else r.dirichlet(np.full(V, 0.8), n)
    tokens, parents = [0, 1, 3, 2], [-1, 0, 0, 1]
    got = np.zeros(V)
    for _ in range(runs):
        path, token = O.verify(P, Q, tokens, parents, n, r.random(n), rule == "distinct")
        got[tokens[path[1]] if len(path) > 1 else token] += 1
    want = probability_of_each(P[0], None if Q is None else Q[0], [1, 3], rule == "distinct")
    assert (np.abs(got / runs - want) < 4 * np.sqrt(want * (1 - want) / runs) + 1e-9).all()


def test_the_closed_form_of_the_residual():
    """R_k = max(P - a_k Q, 0) / b_k with a' = a + b s, b' = sum max(P - a' Q, 0): what the kernels go by."""
    r = np.random.default_rng(9)
    for distinct in (False, True):
        for _ in range(20):
            P, Q = r.dirichlet(np.full(30, 0.5)), r.dirichlet(np.full(30, 0.5))
            R, q, a, b, used = P, Q, 0.0, 1.0, 0.0
            for x in r.choice(30, 4, replace=False):
                stands, after, q_after = O.turned_down(R, q, x, distinct)
                s = 1.0 / (1.0 - used) if distinct else 1.0
                if R[x] > s * Q[x]:
                    break                                       # (never turned down)
                a2 = a + b * s
                w = np.maximum(P - a2 * Q, 0.0)
                if not w.sum() > 1e-9:
                    break
                a, b, used, R, q = a2, w.sum(), used + Q[x], after, q_after
                if distinct:
                    assert w[x] == 0.0
                assert np.abs(w / b - R).max() < 1e-10


def test_edges():
    P = np.array([[0.0, 0.5, 0.5, 0.0]])
    assert O.verify(P, None, [0], None, 0, [0.3]) == ([], -1)
    assert O.verify(P, None, [0], None, 1, [0.0]) == ([0], 1)
    assert O.verify(P, None, [0], None, 1, [0.5]) == ([0], 2)
    assert O.verify(P, None, [0], None, 1, [np.nextafter(np.float32(1), 0)]) == ([0], 2)
    assert O.verify(0 * P, None, [0], None, 1, [0.5]) == ([0], -1)
    # the token has all of the row and is turned down by a number that is none: the row again
    one = np.array([[0.0, 1.0], [0.5, 0.5]])
    assert O.verify(one, None, [0, 1], None, 2, [0.5, 1.0]) == ([0], 1)
