"""Pins of the fp64 statements of steps over drafted tokens (oracle/draft_oracle.py)."""
import numpy as np
import pytest

from oracle import baklava_oracle as O
from oracle import draft_oracle as DO
from oracle import operators_oracle as OP


def test_a_chain_is_the_prompt_behind_its_prefix():
    rng = np.random.default_rng(1)
    n, N, D = 9, 5, 16
    K, V, k, v, q = (rng.standard_normal((m, D)) for m in (n, n, N, N, N))
    got = DO.tree_attention(K, V, k, v, q, [-1, 0, 1, 2, 3])
    want = OP.prompt_attention(q, np.concatenate([K, k]), np.concatenate([V, v]))
    for x, y in zip(got, want):
        np.testing.assert_allclose(x, y, rtol=1e-12)


def test_branches_are_chains_of_their_own():
    rng = np.random.default_rng(2)
    n, D = 4, 8
    parent = [-1, 0, 0, 1, 2, 7, -3]
    N = len(parent)
    K, V, k, v, q = (rng.standard_normal((m, D)) for m in (n, n, N, N, N))
    out, lse, _, _ = DO.tree_attention(K, V, k, v, q, parent)
    for seen in ([0], [0, 1], [0, 2], [0, 1, 3], [0, 2, 4], [5], [6]):  # (a parent that is no earlier node is none)
        i = seen[-1]
        assert DO.ancestors(parent, i) == seen
        o, z, _, _ = OP.prompt_attention(q[i:i + 1], np.concatenate([K, k[seen]]), np.concatenate([V, v[seen]]))
        np.testing.assert_allclose(out[i], o[0], rtol=1e-12)
        np.testing.assert_allclose(lse[i], z[0], rtol=1e-12)


def test_a_node_alone_gets_its_own_value():
    q = np.ones((1, 4))
    out, lse, _, _ = DO.tree_attention(np.zeros((0, 4)), np.zeros((0, 4)), q, 3 * q, q, [-1])
    assert out.tolist() == [[3.0] * 4] and abs(lse[0] - 2 * np.log2(np.e)) < 1e-12


def test_scores_are_those_of_steps_one_by_one():
    rng = np.random.default_rng(3)
    n, P, G, D = 6, 3, 2, 8
    K, V, q = rng.standard_normal((n + P, D)), rng.standard_normal((n + P, D)), rng.standard_normal((P, G, D))
    lse, want = np.zeros((P, G)), np.zeros(n + P)
    for t in range(P):
        for g in range(G):
            s = K[:n + t + 1] @ q[t, g] / np.sqrt(D)
            lse[t, g] = np.log2(np.exp(s).sum())
            want[:n + t + 1] += np.exp(s) / np.exp(s).sum()
    got, _ = DO.path_scores(K, q, lse, n)
    np.testing.assert_allclose(got, want, rtol=1e-12)
    assert abs(got.sum() - P * G) < 1e-10


def test_greedy_walk():
    x = np.full((4, 5), 0.0)
    x[0, 2] = x[0, 4] = 1.0      # the first of the largest: 2
    x[1, 3] = 1.0
    x[2, 0] = 1.0
    assert DO.verify(x, [9, 4, 2, 0], [-1, 0, 0, 2], [0.0] * 4, T=0.0) == ([0, 2, 3], 0)
    assert DO.verify(x, [9, 4, 3, 0], [-1, 0, 0, 2], [0.5] * 4, T=0.0) == ([0], 2)


def test_hand_worked_acceptances():
    p = np.log(np.array([[0.5, 0.25, 0.25], [1.0, 1.0, 2.0]]))
    d = np.log(np.array([[1.0, 1.0, 1.0], [0.75, 0.125, 0.125]]))
    # 0.6 * 0.75 < 0.5 stands; 0.7 * 0.75 > 0.5 does not, and what is left of (0.5, 0.25, 0.25) - (0.75, ...) is (0, 1/2, 1/2)
    assert DO.verify(p, [0, 0], [-1, 0], [0.49, 0.6], draft=d) == ([0, 1], 1)
    assert DO.verify(p, [0, 0], [-1, 0], [0.49, 0.7], draft=d) == ([0], 1)
    assert DO.verify(p, [0, 0], [-1, 0], [0.51, 0.7], draft=d) == ([0], 2)
    # point masses: 0.4 < 0.5; then the rest without token 0
    assert DO.verify(p, [0, 0], [-1, 0], [0.0, 0.4])[0] == [0, 1]
    assert DO.verify(p, [0, 0], [-1, 0], [0.0, 0.6]) == ([0], 1)
    # two children: the second is measured against what the first left: 0.45 < 0.5
    q = np.concatenate([p, p[:1]])
    assert DO.verify(q, [0, 0, 1], [-1, 0, 0], [0.0, 0.6, 0.45])[0] == [0, 2]
    assert DO.verify(q, [0, 0, 1], [-1, 0, 0], [0.0, 0.6, 0.55]) == ([0], 2)


@pytest.mark.parametrize("children", [1, 2, 3])
@pytest.mark.parametrize("drafted", [True, False])
def test_tokens_are_distributed_as_the_target_says(children, drafted):
    """Over all drafts and random numbers the token behind node 0 has the target's distribution."""
    rng = np.random.default_rng(children)
    V, steps = 3, 24 if children < 3 else 12
    x = rng.standard_normal((children + 1, V))
    d = np.tile(rng.standard_normal(V), (children + 1, 1)) + 0.3 * rng.standard_normal((children + 1, V))
    p = DO.distribution(x[0], 1.0)
    got = np.zeros(V)
    grid = (np.arange(steps) + 0.5) / steps
    for tokens in np.ndindex(*[V] * children):
        weight = np.prod([DO.distribution(d[i + 1], 1.0)[t] for i, t in enumerate(tokens)]) if drafted else 1.0 / V ** children
        for us in np.ndindex(*[steps] * children):
            u = [0.0] + [grid[k] for k in us]
            path, _ = DO.verify(x, [0, *tokens], [-1] + [0] * children, u, draft=d if drafted else None)
            if len(path) > 1:
                got[tokens[path[1] - 1]] += weight / steps ** children
                continue
            for u0 in grid:
                u[0] = u0
                got[DO.verify(x, [0, *tokens], [-1] + [0] * children, u, draft=d if drafted else None)[1]] += weight / steps ** (children + 1)
    # each of the children + 1 draws from the grid is off by at most one step of 1 / steps
    np.testing.assert_allclose(got, p, atol=(children + 1) / steps)
    assert abs(got.sum() - 1) < 1e-9


def test_rows_without_a_distribution():
    none = np.full((2, 4), -np.inf)
    assert DO.verify(none, [0, 1], [-1, 0], [0.5, 0.0]) == ([0], -1)
    assert DO.verify(np.full((2, 4), np.nan), [0, 1], [-1, 0], [0.5, 0.0]) == ([0], -1)
    assert DO.verify(np.zeros((0, 4)), [], [], []) == ([], -1)
    x = np.array([[0.0, np.inf, np.nan, -np.inf]])
    assert DO.verify(x, [0], [-1], [0.999]) == ([0], 1)
