"""Plain fp64 statements of steps over several drafted tokens: attention of a tree of them over a cache, verification from given
random numbers, and what an accepted path's attention adds to the scores.

TEST INFRASTRUCTURE ONLY: numpy, no product code.
"""
from __future__ import annotations

import numpy as np


def ancestors(parent, i):
    """Node i and its ancestors, ascending.  A parent that is no earlier node is none."""
    seen = [i]
    while 0 <= parent[seen[-1]] < seen[-1]:
        seen.append(int(parent[seen[-1]]))
    return seen[::-1]


def tree_attention(K, V, k, v, q, parent):
    """One query head: live rows K, V [n, D], drafted rows k, v and queries q [N, D].  Returns (out, lse in log2 units, sum of weight
    times |v|, largest sum of |q_d k_d| / sqrt(D) over the seen keys) of every node."""
    N, D = q.shape
    out, mass = np.zeros((N, D)), np.zeros((N, D))
    lse, big = np.zeros(N), np.zeros(N)
    for i in range(N):
        seen = ancestors(parent, i)
        kk, vv = np.concatenate([K, k[seen]]), np.concatenate([V, v[seen]])
        s = kk @ q[i] / np.sqrt(D)
        top = s.max()
        e = np.exp(s - top)
        p = e / e.sum()
        out[i], mass[i] = p @ vv, p @ np.abs(vv)
        lse[i] = (top + np.log(e.sum())) * np.log2(np.e)
        big[i] = (np.abs(kk) @ np.abs(q[i])).max() / np.sqrt(D)
    return out, lse, mass, big


def weights(x, T):
    """What softmax(x / T) is proportional to, the largest 1; T not above 0: all on the first of the largest.  NaN counts as -inf,
    inf as the largest fp32 number.  (Sums of equal weights are whole numbers, so that borders between them are exact.)"""
    x = np.array(x, dtype=np.float64)
    x[np.isnan(x)] = -np.inf
    x = np.minimum(x, float(np.finfo(np.float32).max))
    p = np.zeros(len(x))
    if x.max() == -np.inf:
        return p
    if not T > 0:
        p[int(np.argmax(x))] = 1.0
        return p
    return np.exp((x - x.max()) / T)


def distribution(x, T):
    w = weights(x, T)
    return w / w.sum() if w.sum() > 0 else w


def verify(logits, token, parent, u, T=1.0, draft=None):
    """One sequence: logits [N, V], token, parent, u [N], draft [N, V] or None.  Returns (path, next token)."""
    N, V = logits.shape
    if N == 0:
        return [], -1
    path, w = [0], weights(logits[0], T)
    for i in range(1, N):
        t = token[i]
        if parent[i] != path[-1] or not 0 <= t < V:
            continue
        r = w / w.sum() if w.sum() > 0 else w
        drafted = draft is not None and T > 0
        q = distribution(draft[i], T) if drafted else None
        if float(u[i]) * (q[t] if drafted else 1.0) < r[t]:
            path.append(i)
            w = weights(logits[i], T)
            continue
        if drafted:
            rest = np.maximum(r - q, 0.0)
        else:
            rest = w.copy()
            rest[t] = 0.0
        if rest.sum() > 0:
            w = rest
    live = np.flatnonzero(w > 0)
    if len(live) == 0:
        return path, -1
    c = np.cumsum(w)
    over = np.flatnonzero((c > float(u[0]) * c[-1]) & (w > 0))
    return path, int(over[0]) if len(over) else int(live[-1])


def path_scores(K, q, lse, n):
    """What the path's attention adds to the scores of K [n + P, D], of which the last P are the path's rows: q [P, G, D], lse [P, G] in
    log2 units.  Also returns the largest sum of |q_d k_d| / sqrt(D)."""
    P, G, D = q.shape
    add, big = np.zeros(len(K)), 0.0
    for t in range(P):
        for g in range(G):
            s = K[:n + t + 1] @ q[t, g] / np.sqrt(D)
            add[:n + t + 1] += np.exp2(s * np.log2(np.e) - lse[t, g])
            big = max(big, (np.abs(K) @ np.abs(q[t, g])).max() / np.sqrt(D))
    return add, big
