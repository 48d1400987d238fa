"""GPU parity: verification of drafted tokens (baklava_verify_draft); paths and tokens exactly those of fp64."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from paper_2502_13176_amd import binding as B

pytestmark = pytest.mark.gpu


def parents(kind, batch, N, rng):
    p = np.full((batch, N), -1, dtype=np.int32)
    for i in range(1, N):
        p[:, i] = i - 1 if kind == "chain" else 0 if kind == "star" else (rng.random(batch) ** 2 * i).astype(np.int32)
    return p


def inputs(batch, N, V, tree, dtype, drafts, seed, likely=0.8):
    """Logits whose likely tokens are in part the drafted ones, so that paths of all lengths come up."""
    rng = np.random.default_rng(seed)
    x = 2 * rng.standard_normal((batch, N, V))
    parent = parents(tree, batch, N, rng)
    token = rng.integers(0, V, (batch, N))
    for b in range(batch):
        for i in range(1, N):
            if 0 <= parent[b, i] < i and rng.random() < likely:
                x[b, parent[b, i], token[b, i]] += np.log(V) + 2 + 2 * rng.random()
    d = None
    if drafts:
        d = np.stack([x[np.arange(batch), np.maximum(parent[:, i], 0)] + 0.8 * rng.standard_normal((batch, V)) for i in range(N)], 1)
        for b in range(batch):
            for i in range(1, N):
                token[b, i] = rng.choice(V, p=DO.distribution(d[b, i], 1.0))
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    to = lambda t: torch.from_numpy(np.ascontiguousarray(t))
    u = torch.from_numpy(rng.random((batch, N)).astype(np.float32)).clamp(max=1 - 2.0 ** -24)
    return dict(logits=to(x).to(dt), token=to(token).int(), parent=to(parent), u=u, draft_logits=None if d is None else to(d).to(dt))


def run(t, **kw):
    args = {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in (t | kw).items()}
    return [x.cpu() for x in B.verify_draft(**args)]


def expect(t, temperature=None, n_nodes=None):
    batch, N = t["parent"].shape
    V = t["logits"].shape[-1]
    x = t["logits"].reshape(batch, N, V).double().numpy()
    d = t["draft_logits"].reshape(batch, N, V).double().numpy() if t["draft_logits"] is not None else None
    path, count, token = np.full((batch, N), -1), np.zeros(batch, int), np.zeros(batch, int)
    for b in range(batch):
        n = N if n_nodes is None else min(max(int(n_nodes[b]), 0), N)
        T = 1.0 if temperature is None else float(temperature[b])
        p, token[b] = DO.verify(x[b, :n], t["token"][b].tolist(), t["parent"][b].tolist(), t["u"][b].tolist(), T, None if d is None else d[b, :n])
        path[b, :len(p)], count[b] = p, len(p)
    return path, count, token


def same(got, want):
    for g, w, name in zip(got, want, ("path", "n_path", "next_token")):
        assert g.dtype == torch.int32 and np.array_equal(g.numpy(), w), (name, g.tolist(), w.tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("drafts", [False, True])
@pytest.mark.parametrize("tree,batch,N,V", [("chain", 3, 1, 40), ("chain", 5, 6, 1000), ("tree", 4, 20, 333), ("star", 6, 9, 64), ("tree", 2, 70, 129),
                                            ("tree", 1, 256, 50), ("chain", 2, 200, 8), ("tree", 3, 7, 8192), ("tree", 3, 7, 8193), ("star", 3, 5, 20001),
                                            ("chain", 2, 3, 1), ("star", 9, 4, 2)])
def test_against_fp64(dtype, drafts, tree, batch, N, V):
    for seed in range(3):
        t = inputs(batch, N, V, tree, dtype, drafts, seed * 100 + N)
        same(run(t), expect(t))
        rng = np.random.default_rng(seed)
        temp = torch.tensor(rng.choice([0.0, 0.5, 1.0, 2.0, -1.0], batch), dtype=torch.float32)
        n = torch.tensor(rng.integers(-1, N + 2, batch), dtype=torch.int32)
        same(run(t, temperature=temp, n_nodes=n), expect(t, temp, n))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_draws_of_a_large_vocabulary(dtype):
    """200 sequences, one node each: the next token alone, whose borders are some 1e-5 apart."""
    t = inputs(200, 1, 100003, "chain", dtype, False, 5)
    same(run(t), expect(t))


def test_random_numbers_on_borders():
    """Probabilities that are powers of two, random numbers that equal them: strictly less stands; the sum has to exceed."""
    V = 8
    for dtype in (torch.bfloat16, torch.float32):
        x = torch.zeros((1, 2, V), dtype=dtype)
        t = dict(logits=x, token=torch.tensor([[0, 3]]).int(), parent=torch.tensor([[-1, 0]]).int(), u=torch.tensor([[0.5, 0.125]]), draft_logits=None)
        got = run(t)
        assert got[0].tolist() == [[0, -1]] and got[2].tolist() == [4]  # seven tokens are left: 3 / 7 up to token 2, 4 / 7 up to token 4
        t["u"] = torch.tensor([[0.5, 0.125 - 2.0 ** -27]])
        got = run(t)
        assert got[0].tolist() == [[0, 1]] and got[2].tolist() == [4]   # c(3) = 0.5 does not exceed 0.5
        t["u"] = torch.tensor([[0.0, 0.0]])
        assert run(t)[2].tolist() == [0]
        t["u"] = torch.tensor([[1 - 2.0 ** -24, 0.0]])
        assert run(t)[2].tolist() == [V - 1]


def test_values_that_are_not_finite():
    V = 300
    inf, nan = float("inf"), float("nan")
    x = torch.full((7, 2, V), -inf)
    x[1, 0, 7] = 0.0
    x[2, 0, 7], x[2, 0, 9] = inf, inf
    x[3, 0], x[3, 0, 250] = nan, -3.0
    x[4] = 0.0
    x[4, 0, ::2] = nan
    x[5, 0, 299] = 3.4028234663852886e38
    x[6, 0, 3], x[6, 1, 4] = 1.0, 2.0
    t = dict(logits=x, token=torch.tensor([[0, 7]] * 6 + [[0, 3]]).int(), parent=torch.tensor([[-1, 0]] * 7).int(),
             u=torch.full((7, 2), 0.75), draft_logits=None)
    for temp in (None, torch.zeros(7), torch.full((7,), 0.25)):
        same(run(t, temperature=temp), expect(t, temp))
    t["draft_logits"] = x.roll(1, 0)
    same(run(t), expect(t))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("drafts", [False, True])
@pytest.mark.parametrize("temp", [None, 0.7, 1e-3, 1e-30, 1e-42, 1e30, float("inf")])
def test_lowest_and_largest_values_beside_ordinary_ones(dtype, drafts, temp):
    """Tokens masked with the type's lowest value, rows with an infinity, temperatures at the ends of their range."""
    B_, N, V = 6, 7, 300
    for tree in ("chain", "tree"):
        t = inputs(B_, N, V, tree, dtype, drafts, 11)
        low = torch.finfo(t["logits"].dtype).min
        keep = torch.rand((B_, N, V), generator=torch.Generator().manual_seed(5)) < 0.6
        for b in range(B_):
            for i in range(1, N):
                keep[b, max(int(t["parent"][b, i]), 0), int(t["token"][b, i])] = True
        t["logits"] = t["logits"].masked_fill(~keep, low)
        if temp is None or temp < 1e30:
            t["logits"][4, 0, 17] = float("inf")
            t["logits"][5, 1, 3], t["logits"][5, 1, 5] = -low, -low
        same(run(t, temperature=None if temp is None else torch.full((B_,), temp)), expect(t, None if temp is None else torch.full((B_,), temp)))


def test_tokens_that_are_none_and_parents_that_are_none():
    t = inputs(4, 8, 50, "star", "f32", False, 1)
    want = expect(t)
    t["parent"][:, 0] = torch.tensor([0, 5, -9, 99]).int()  # (the root's is not looked at)
    same(run(t), want)
    t["token"][0, 1], t["token"][1, 2], t["token"][2, 3] = -1, 50, 1 << 30
    t["parent"][3, 4], t["parent"][3, 5] = 5, 5
    same(run(t), expect(t))
    d = inputs(4, 8, 50, "star", "f32", True, 2)
    d["token"][0, 1], d["token"][1, 2] = -1, 50
    same(run(d), expect(d))


def test_the_same_token_twice():
    """Siblings that repeat a token: its weight is taken off once."""
    x = torch.tensor([[[2.0, 1.0, 0.0, 0.0]] * 4])
    for u in ([0.3, 0.9, 0.0, 0.4], [0.99, 0.9, 0.0, 0.99], [0.0, 0.1, 0.5, 0.5]):
        t = dict(logits=x, token=torch.tensor([[0, 0, 0, 1]]).int(), parent=torch.tensor([[-1, 0, 0, 0]]).int(), u=torch.tensor([u]), draft_logits=None)
        same(run(t), expect(t))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_and_rows_at_any_element(dtype):
    V = 1001
    for drafts in (False, True):
        t = inputs(3, 5, V, "tree", dtype, drafts, 11)
        want = expect(t)
        dt = t["logits"].dtype
        for pad, front in ((1, 0), (7, 3), (24, 1)):
            s = dict(t)
            for n in ("logits", "draft_logits"):
                if t[n] is not None:
                    wide = torch.full((15, V + pad + front), float("nan"), dtype=dt, device="cuda")
                    wide[:, front:front + V] = t[n].reshape(15, V).cuda()
                    s[n] = wide[:, front:front + V]
                    pad += 3
            same([x.cpu() for x in B.verify_draft(**{n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in s.items()})], want)


def test_drawn_tokens_follow_the_target():
    """4000 sequences with the same two-token choice: counts within four standard deviations."""
    n, V = 4000, 5
    rng = np.random.default_rng(3)
    row = rng.standard_normal(V)
    d = rng.standard_normal(V)
    p, q = DO.distribution(row, 1.0), DO.distribution(d, 1.0)
    token = np.stack([np.zeros(n, int), rng.choice(V, n, p=q)], 1)
    u = rng.random((n, 2)).astype(np.float32)
    u = np.minimum(u, 1 - 2.0 ** -24).astype(np.float32)
    t = dict(logits=torch.from_numpy(np.broadcast_to(row, (n, 2, V)).copy()).float(), draft_logits=torch.from_numpy(np.broadcast_to(d, (n, 2, V)).copy()).float(),
             token=torch.from_numpy(token).int(), parent=torch.tensor([[-1, 0]] * n).int(), u=torch.from_numpy(u))
    path, count, nxt = run(t)
    behind_root = np.where(count.numpy() > 1, token[:, 1], nxt.numpy())
    got = np.bincount(behind_root, minlength=V)
    assert (np.abs(got - n * p) <= 4 * np.sqrt(n * p * (1 - p))).all(), (got, n * p)


def test_vocabularies_of_more_parts_than_are_held():
    V = 3 * (1 << 18) + 5
    for drafts in (False, True):
        t = inputs(2, 3, V, "chain", "bf16", False, 3)
        if drafts:
            t["draft_logits"] = (t["logits"].float().roll(1, 1) + 0.5 * torch.randn(t["logits"].shape, generator=torch.Generator().manual_seed(1))).bfloat16()
        for u0 in (0.0, 0.37, 1 - 2.0 ** -24):
            t["u"][:, 0] = u0
            same(run(t), expect(t))


def test_two_calls_at_once_and_other_streams():
    sets = [inputs(4, 12, 5000, "tree", "f32", False, 1), inputs(6, 5, 20000, "chain", "bf16", True, 2)]
    sets = [{n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in t.items()} for t in sets]
    want = [B.verify_draft(**t) for t in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda._sleep(5_000_000)
    for _ in range(5):
        got = [B.verify_draft(**t, stream=s) for t, s in zip(sets, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for gs, ws in zip(got, want) for x, y in zip(gs, ws))


def test_captured_and_replayed():
    for drafts in (False, True):
        t = {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in inputs(3, 9, 4000, "tree", "bf16", drafts, 7).items()}
        B.verify_draft(**t)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            res = B.verify_draft(**t)
        for seed in range(4):
            new = inputs(3, 9, 4000, "tree", "bf16", drafts, 20 + seed)
            for n, x in new.items():
                if isinstance(x, torch.Tensor):
                    t[n].copy_(x)
            graph.replay()
            torch.cuda.synchronize()
            same([x.cpu() for x in res], expect(new))
            torch.randn((500, 500), device="cuda").sum().item()


def test_refusals_on_the_gpu():
    t = {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in inputs(2, 3, 50, "chain", "f32", False, 1).items()}
    f = torch.zeros((2, 3, 50), device="cuda")
    for bad in (dict(logits=f.double()), dict(logits=f[:, :2]), dict(logits=f.cpu()), dict(logits=f.transpose(0, 1).contiguous().transpose(0, 1)),
                dict(logits=torch.zeros((2, 3, 100), device="cuda")[..., ::2]), dict(draft_logits=f.bfloat16()), dict(draft_logits=f[..., :49]),
                dict(temperature=torch.ones(3, device="cuda")), dict(temperature=torch.ones(2, device="cuda").double()), dict(n_nodes=torch.ones(2, device="cuda")),
                dict(u=t["u"].cpu()), dict(u=t["u"].double())):
        with pytest.raises(ValueError):
            B.verify_draft(**(t | bad))
