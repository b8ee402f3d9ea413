"""Children drawn without putting back from rows in 16 bits (CPU): what a row whose entries were rounded does to the verification's
promise that tokens come out with the target's probabilities.

A draft row as it is stored sums to S.  A child that is drawn from it has x with Q(x) / S, so what stands is min(P, Q) / S and not
min(P, Q); with one child, and where no other is tried, what comes out is off by |1 - 1/S| of a token's probability at most
(M = sum min(P, Q): M (1 - 1/S) / (1 - M) of max(P - Q, 0), whose sum is 1 - M).  Orders that begin with a token of little
weight come as seldom as it, and add |1 - S| of that."""
import itertools

import numpy as np
import pytest
import torch

from oracle import tree as O

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def stored(row, dtype):
    return torch.tensor(row, dtype=torch.float64).to(dtype).double().numpy()


def chances(P, Q, children):
    """Of the tokens behind node 0, whose children these are, in verify()'s own rule: that a child stands with it, or that it is the
    next token.  Each decision is asked of verify() with a uniform number on either side of its border."""
    V, n = P.size, len(children) + 1
    target, draft = np.tile(P, (n, 1)), np.tile(Q, (n, 1))
    tokens, parents = [0, *children], [-1] + [0] * len(children)
    out, alive = np.zeros(V), 1.0

    def goes(u):
        return O.verify(target, draft, tokens, parents, n, u, True)

    for i in range(1, n):
        def stands(x, i=i):                                      # with the children before turned down, those behind not reached
            u = np.full(n, 1.0)
            u[0], u[i] = 0.5, x
            return goes(u)[0][1:2] == [i]
        lo, hi = 0.0, 1.0                                        # the largest number that lets it stand
        if not stands(0.0):
            continue
        if not stands(1.0 - 2.0 ** -40):
            for _ in range(45):
                mid = (lo + hi) / 2
                lo, hi = (mid, hi) if stands(mid) else (lo, mid)
        else:
            lo = 1.0
        out[children[i - 1]] += alive * lo
        alive *= 1.0 - lo
    if alive > 0.0:                                              # the next token behind all of them turned down, over its number
        u = np.full(n, 1.0)
        grid = (np.arange(4096) + 0.5) / 4096
        for x in grid:
            u[0] = x
            out[goes(u)[1]] += alive / grid.size
    return out


def total(P, Q, k):
    out = np.zeros(P.size)
    for drawn in itertools.permutations(range(P.size), k):
        left, chance = Q.copy(), 1.0
        for x in drawn:
            chance *= left[x] / left.sum() if left.sum() > 0 else 0.0
            left[x] = 0.0
        if chance > 0:
            out += chance * chances(P, Q, list(drawn))
    return out


# rows whose first entry is 1 in the type
NEARLY_CERTAIN = [([0.5, 0.1, 0.4], [0.9985, 0.00125, 0.00025], BF16), ([0.2, 0.7, 0.1], [0.99985, 0.0001, 0.00005], F16),
                  ([0.05, 0.05, 0.9], [0.9981, 0.0018, 0.0001], BF16)]


@pytest.mark.parametrize("k", [1, 2, 3])
@pytest.mark.parametrize("P,Q,dtype", NEARLY_CERTAIN)
def test_no_child_is_tried_where_nothing_is_left_of_the_draft(P, Q, dtype, k):
    """Once the tried tokens have all of the row, a sibling cannot have come from what is left of it: its chance is not known, and
    letting it stand whatever its number is gives it the others' probability."""
    P, Q = np.array(P), stored(Q, dtype)
    assert Q[0] == 1.0
    off = np.abs(total(P, Q, k) - P).max()
    assert off <= abs(1 - 1 / Q.sum()) + 1 / 4096, off           # (the grid's step)


def test_the_walk_ends_there():
    P = np.array([[0.0, 0.1, 0.9]] * 4)
    Q = np.array([[1.0, 0.0, 0.0]] * 4)
    assert O.verify(P, Q, [0, 0, 1, 2], [-1, 0, 0, 0], 4, [0.05, 0.5, 0.0, 0.0], True) == ([0], 1)
    assert O.verify(P, Q, [0, 0, 1, 2], [-1, 0, 0, 0], 4, [0.5, 0.5, 0.0, 0.0], True) == ([0], 2)
    # the sum of the tried tokens is what counts, not that of one
    Q = np.array([[0.25, 0.75, 0.0]] * 4)
    P = np.array([[0.0, 0.0, 1.0]] * 4)
    assert O.verify(P, Q, [0, 0, 1, 2], [-1, 0, 0, 0], 4, [0.5, 0.5, 0.5, 0.0], True) == ([0], 2)
    # drawn independently, each comes from the whole row
    assert O.verify(P, Q, [0, 0, 1, 2], [-1, 0, 0, 0], 4, [0.5, 0.5, 0.5, 0.0], False) == ([0, 3], 2)


def draft_rows(dtype):
    """Rows as a softmax in the type leaves them, from flat ones to nearly certain ones (their first entry below 1)."""
    r = np.random.default_rng(31)
    for top in (0.3, 0.7, 0.93, 0.985, 0.994):
        rest = r.dirichlet(np.full(3, 0.8)) * (1.0 - top)
        yield r.dirichlet(np.full(4, 0.7)), stored([top, *rest], dtype)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_what_a_row_that_does_not_sum_to_one_is_off_by(dtype):
    """Two children: the first |e| / S of a token's probability at most, S = 1 + e; the second, behind x, is compared with
    Q / (1 - Q(x)) and was drawn from Q / (S - Q(x)), a row of the sum (S - Q(x)) / (1 - Q(x)): |e| / (S - Q(x))."""
    for P, Q in draft_rows(dtype):
        S = Q.sum()
        e = abs(S - 1.0)
        off = np.abs(total(P, Q, 2) - P).max()
        assert off <= e / S + sum(q / S * e / (S - q) for q in Q) + 1 / 4096, (Q, off)


@pytest.mark.parametrize("dtype", [F16, BF16])
def test_rows_divided_by_their_sums_in_float32_keep_the_promise(dtype):
    """The same rows, converted and divided: what is left is float32's rounding, 2^-24 of each entry against the 2^-8 that is left of
    the most certain row."""
    for P, Q in [*draft_rows(dtype), (np.array([0.5, 0.1, 0.4]), stored([0.9985, 0.00125, 0.00025], dtype))]:
        Q = (torch.from_numpy(Q).float() / torch.from_numpy(Q).float().sum()).double().numpy()
        assert np.abs(total(P, Q, 2) - P).max() <= 1 / 4096 + 2.0 ** -14
