"""GPU parity: verification of drafted tokens where siblings take nearly all of a distribution's weight, or all of it: what is left by them has
to be as exact as a whole distribution.  Paths and tokens exactly those of fp64."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from test_gpu_verify import expect, inputs, run, same

pytestmark = pytest.mark.gpu

LAST = 1 - 2.0 ** -24  # the largest random number


def star(rows, tokens, u, dtype, V):
    """Sequences of a root and as many children as tokens: rows [batch, len(tokens) or more] logits of tokens 0 .., -inf behind them."""
    batch, n = tokens.shape
    x = torch.full((batch, n + 1, V), float("-inf"), dtype=dtype)
    x[:, 0, :rows.shape[1]] = torch.from_numpy(rows).to(dtype)
    x[:, 1:, :3] = 0.0
    parent = torch.zeros((batch, n + 1), dtype=torch.int32)
    parent[:, 0] = -1
    token = torch.cat([torch.zeros((batch, 1), dtype=torch.int32), torch.from_numpy(tokens).int()], 1)
    return dict(logits=x, token=token, parent=parent, u=torch.from_numpy(np.asarray(u, dtype=np.float32)), draft_logits=None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_one_row_whose_tokens_are_all_drafted(dtype):
    """Children that draft all tokens a row has, every random number the largest: the last child has all that is left, and stands."""
    for row in ([0, -0.0078125, -12], [0, -1.1328875, -11.610435], [3, 3, 3, 3], [0, -16, -16.5], [0, -9, -18, -27, -36], [0, -17, -34, -51, -68]):
        n = len(row)
        t = star(np.array([row], dtype=np.float64), np.arange(n)[None], [[0.3] + [LAST] * n], dtype, 40)
        got = run(t)
        same(got, expect(t))
        assert int(got[1][0]) == 2 and int(got[2][0]) >= 0
    t = star(np.array([[0, -1.1328875, -11.610435]]), np.arange(3)[None], [[.3, .87818307, .9999719, .9993186]], dtype, 3)
    same(run(t), expect(t))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [9, 700, 20001])
@pytest.mark.parametrize("few", [3, 4, 5])
def test_rows_of_few_tokens_that_are_drafted(dtype, V, few):
    """Rows of three to five tokens (anywhere in the vocabulary, the others -inf or the type's lowest value), all of them or all but one
    drafted, random numbers at random or the largest."""
    batch = 120
    rng = np.random.default_rng(few + V)
    n = np.where(np.arange(batch) % 2, few, few - 1)  # children
    x = torch.full((batch, few + 1, V), float("-inf"), dtype=dtype)
    x[batch // 2:, 0] = torch.finfo(dtype).min
    x[:, 1:, :3] = 0.0
    tokens = np.stack([rng.choice(V, few, replace=False) for _ in range(batch)])
    logits = -np.sort(rng.exponential(6.0, (batch, few)), 1)
    for b in range(batch):
        x[b, 0, tokens[b]] = torch.from_numpy(logits[b]).to(dtype)
    parent = torch.zeros((batch, few + 1), dtype=torch.int32)
    u = rng.random((batch, few + 1)).astype(np.float32).clip(max=LAST)
    u[rng.random(u.shape) < 0.7] = LAST
    t = dict(logits=x, token=torch.cat([torch.zeros((batch, 1)), torch.from_numpy(tokens)], 1).int(), parent=parent, u=torch.from_numpy(u), draft_logits=None)
    count = torch.from_numpy(n + 1).int()
    got = run(t, n_nodes=count)
    assert (got[2] >= 0).all()
    same(got, expect(t, n_nodes=count))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("V", [300, 9000])
def test_random_numbers_beside_a_siblings_threshold(dtype, V):
    """Peaked rows, the likeliest tokens drafted: u of the k-th child is the fp32 number next below what it has of the rest, then the one next
    above it, u of those before it the largest.  fp64 sums of V terms, an exponential to 2^-47 and its argument (at most 100, half a step of
    2^-53 relative) leave a threshold within 1e-11: nearer random numbers are not asked for."""
    batch, n = 64, 5
    rng = np.random.default_rng(V)
    x = (rng.choice([2.0, 5.0, 9.0], (batch, 1)) * rng.standard_normal((batch, V)))
    row = torch.from_numpy(x).to(dtype)
    tokens = np.argsort(-row.double().numpy(), 1, kind="stable")[:, :n].copy()
    asked = 0
    for k in range(n):
        w = np.stack([DO.weights(r, 1.0) for r in row.double().numpy()])
        for b in range(batch):
            w[b, tokens[b, :k]] = 0.0
        r = w[np.arange(batch), tokens[:, k]] / w.sum(1)
        near = r.astype(np.float32)
        below = np.where(near.astype(np.float64) < r, near, np.nextafter(near, np.float32(0)))
        above = np.nextafter(below, np.float32(1))
        clear = (r - below > 1e-11) & (above - r > 1e-11) & (above <= LAST)
        for u_k in (below, above):
            u = np.full((batch, n + 1), LAST, dtype=np.float32)
            u[:, 0] = rng.random(batch)
            u[:, k + 1] = np.where(clear, u_k, 0.5)
            t = star(np.zeros((batch, 1)), tokens, u, dtype, V)
            t["logits"][:, 0] = row
            same(run(t), expect(t))
            asked += int(clear.sum())
    assert asked > 6 * batch


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tree,batch,N,V", [("tree", 6, 30, 400), ("star", 8, 12, 60), ("star", 3, 200, 256), ("tree", 2, 256, 8193)])
@pytest.mark.parametrize("temp", [None, 0.3])
def test_trees_with_large_random_numbers(dtype, tree, batch, N, V, temp):
    """Half of the random numbers the largest: many siblings fail, tokens come up twice, paths go on behind them."""
    for seed in range(3):
        t = inputs(batch, N, V, tree, dtype, False, 300 + seed, likely=0.9)
        rng = np.random.default_rng(seed)
        t["u"][torch.from_numpy(rng.random((batch, N)) < 0.5)] = LAST
        again = torch.from_numpy(rng.random((batch, N)) < 0.2)
        t["token"] = torch.where(again, t["token"].roll(1, 1), t["token"])
        T = None if temp is None else torch.full((batch,), temp)
        same(run(t, temperature=T), expect(t, T))


def test_a_star_over_a_whole_vocabulary():
    """255 children, all tokens but one: r of every child counts what is left by all before it."""
    V = 256
    rng = np.random.default_rng(4)
    for dtype in (torch.bfloat16, torch.float32):
        row = np.sort(rng.standard_normal((4, V)) * 3)[:, ::-1].copy()
        u = np.full((4, V), LAST)
        u[1, 1:] = rng.random(255) * 0.05 + 0.95
        u[2, 200:] = 0.0
        u[:, 0] = (0.0, 0.5, 0.9, LAST)
        t = star(row, np.tile(np.arange(255), (4, 1)), u.clip(max=LAST), dtype, V)
        same(run(t), expect(t))
