"""Trees of drafted tokens in float64, from their definitions.  Plain numpy; nothing here is shared with the library.

Node 0 is the last token that was sampled; node i > 0 is a drafted token behind node parents[i] < i."""
from __future__ import annotations

import numpy as np


def parent_of(parents, i):
    """The node that node i is behind, or -1.  parents None: a chain."""
    up = i - 1 if parents is None else int(parents[i])
    return up if 0 <= up < i else -1


def masks(n, parents, count):
    """sees [n, n] bool and the number of ancestors [n] of one sequence's nodes; nothing for nodes from count on."""
    sees, depth = np.zeros((n, n), bool), np.zeros(n, np.int64)
    for i in range(min(max(count, 0), n)):
        j = i
        while j >= 0:
            sees[i, j] = True
            j = parent_of(parents, j)
        depth[i] = sees[i].sum() - 1
    return sees, depth


def words(sees):
    """Rows of bits as uint64 words: bit j % 64 of word j / 64."""
    n, m = sees.shape
    out = np.zeros((n, -(-m // 64)), np.uint64)
    for j in range(m):
        out[:, j // 64] |= sees[:, j].astype(np.uint64) << np.uint64(j % 64)
    return out


def taken(x, top):
    """Elements as an 8-bit block takes them: NaN as zero, held to +-top."""
    return np.clip(np.where(np.isnan(x), 0.0, x), -top, top)


def attention(q, K, V, scale, sees):
    """One head's q [n, 128] over K, V [T, 128]; sees [n, T].  -> out, and sum_t w_t |V_t| of each row."""
    out, W = np.zeros(q.shape), np.zeros(q.shape)
    for i in range(q.shape[0]):
        t = np.flatnonzero(sees[i])
        if t.size:
            x = scale * (K[t] @ q[i])
            p = np.exp(x - x.max())
            p /= p.sum()
            out[i], W[i] = p @ V[t], p @ np.abs(V[t])
    return out, W


def turned_down(R, Q, x, distinct):
    """(probability that token x stands, what R becomes if it does not, what Q becomes).  Q None: x is no random token."""
    if Q is None:
        left = R.copy()
        left[x] = 0.0
        rest = 1.0 - R[x]
        return R[x], (left / rest if rest > 0 else left), None
    q = Q[x]
    stands = 1.0 if R[x] > 0 and q <= 0 else 0.0 if q <= 0 else min(1.0, R[x] / q)
    left = np.maximum(R - Q, 0.0)
    z = left.sum()
    after = Q
    if distinct:
        after = Q.copy()
        after[x] = 0.0
        after = after / (1.0 - q) if q < 1.0 else np.zeros_like(Q)
    return stands, (left / z if z > 0 else R), after


def verify(target, draft, tokens, parents, count, uniform, distinct=False):
    """(path, next token) of one sequence: target, draft [n, vocab] float64."""
    n, V = target.shape
    count = min(max(count, 0), n)
    if count == 0:
        return [], -1
    row = lambda x, u: np.where(x[u] > 0, x[u], 0.0)  # noqa: E731
    u, path, R, Q, had = 0, [0], row(target, 0), None if draft is None else row(draft, 0), set()
    tried = 0.0                                                # the row's probability of the tokens that were turned down
    for i in range(1, count):
        x = int(tokens[i])
        if parent_of(parents, i) != u or not 0 <= x < V:
            continue
        if x in had and (draft is None or distinct):
            continue
        if distinct and tried >= 1.0:
            break                                              # nothing is left of Q that a further child could have come from
        had.add(x)
        stands = uniform[i] * (1.0 if Q is None else Q[x]) < R[x]
        if not stands and Q is not None and not (R > Q).any():
            break                                              # nothing would be left: R stays, no further child is tried
        _, after, q_after = turned_down(R, Q, x, distinct)
        if stands:
            u, had, tried = i, set(), 0.0
            path.append(i)
            R, Q = row(target, i), None if draft is None else row(draft, i)
        else:
            tried += 0.0 if draft is None else row(draft, u)[x]
            R, Q = after, q_after
    if not R.sum() > 0:
        R = row(target, u)
    total = np.cumsum(R)
    some = np.flatnonzero(R > 0)
    if not some.size:
        return path, -1
    over = np.flatnonzero((total > uniform[0] * total[-1]) & (R > 0))
    return path, int(over[0] if over.size else some[-1])
