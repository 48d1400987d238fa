"""GPU parity: attention of drafted trees over the caches (baklava_tree_attn) against fp64."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from oracle import operators_oracle as OP
from paper_2502_13176_amd import binding as B

pytestmark = pytest.mark.gpu


def stored(x, dtype):
    """What a cache holds of rows x [..., D], in fp64."""
    x = np.asarray(x.double().cpu())
    if dtype == "mxfp4":
        code, s = OP.mx_round(x)
        return OP.mx_values(OP.mx_pack(code), s)
    return x


def make(dtype, D, G, Hkv, batch, L, lens, room=8, seed=0, track=False):
    """An arena of random rows: lens [L * batch * Hkv] live ones; places behind them are NaN.  Also its rows in fp64."""
    cap = np.asarray(lens).reshape(L, batch, Hkv).max(1).reshape(-1) + room
    a = B.Arena(L, G * Hkv, Hkv, D, batch, dtype, cap.tolist(), 0, 0, 0, track_scores=track, workspace_fill=0xFF)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(seed)
    K, V = (torch.randn((a.total_tokens, D), generator=g).to(dt) for _ in range(2))
    for plane, x, at in ((a.k, K, 0), (a.v, V, D // 32)):
        if dtype == "mxfp4":
            code, s = OP.mx_round(x.double().numpy())
            plane.copy_(torch.from_numpy(OP.mx_pack(code)))
            a.kv_scale[:, at:at + D // 32] = torch.from_numpy(s).cuda()
        else:
            plane.copy_(x)
    for c, n in enumerate(lens):
        dead = slice(int(a.off_host[c]) + n, int(a.off_host[c]) + int(a.cap_host[c]))
        if dtype == "mxfp4":
            a.kv_scale[dead] = 255
        else:
            a.k[dead], a.v[dead] = float("nan"), float("nan")
    a.score.zero_()
    a.set_lengths(lens)
    return a, stored(K, dtype), stored(V, dtype)


def parents(kind, batch, N, seed=0):
    rng = np.random.default_rng(seed)
    p = np.full((batch, N), -1, dtype=np.int32)
    for b in range(batch):
        for i in range(1, N):
            p[b, i] = i - 1 if kind == "chain" else 0 if kind == "star" else -1 if kind == "apart" else rng.integers(max(-1, i - 9), i)
    return p


def nodes(layout, n_seq, N, H, D, dt, g):
    x = torch.randn((n_seq * N, H, D), generator=g)
    if layout == "fused":
        return torch.randn((n_seq * N, H + 3, D), generator=g).to(dt).cuda()[:, 2:2 + H]
    if layout == "padded":
        return torch.randn((n_seq, H, N + 2, D), generator=g).to(dt).cuda()[:, :, :N]
    return x.to(dt).cuda()


def check(a, K, V, k, v, q, parent, n_nodes, out, lse, layers, dtype, only=None):
    """out within rounding of fp64.  A weight's relative error: its logit's absolute one (D products and as many additions in fp32, each
    off by half a step of 2^-24 of what has been summed, and the product with the scale), 2^-22 of the exponential and, bf16 rows, half
    a step of bf16, 2^-8.  Sums of n terms in fp32: n half steps at most.  The output is rounded once, in its own type.  Weights below
    2^-126 of the largest one count as zero (the largest is at least 1 before the division by the sum, and fp32 ends there): n + N
    of them lose (n + N) 2^-126 max |v| at most."""
    batch, N, Hkv, D = a.batch, parent.shape[1], a.Hkv, a.D
    G = a.Hq // Hkv
    half = 2.0 ** -24 if dtype == "f32" else 2.0 ** -8
    kd, vd = stored(k, dtype), stored(v, dtype)
    qd = q.double().cpu().numpy()
    o, z = out.double().cpu().numpy(), lse.double().cpu().numpy() if lse is not None else None
    lens = a.len.cpu().numpy()
    for c in range(layers[0] * batch * Hkv, (layers[0] + layers[1]) * batch * Hkv):
        if only is not None and c not in only:
            continue
        s, h = c // Hkv - layers[0] * batch, c % Hkv
        b = s % batch
        m = N if n_nodes is None else min(max(int(n_nodes[b]), 0), N)
        at, n = int(a.off_host[c]), int(lens[c])
        pick = lambda t, i: t[s, i, :m] if t.ndim == 4 else t[s * N:s * N + m, i]
        for g in range(G):
            hq = h * G + g
            want, wl, mass, big = DO.tree_attention(K[at:at + n], V[at:at + n], pick(kd, h), pick(vd, h), pick(qd, hq), parent[b])
            e = 2 * (D + 2) * 2.0 ** -24 * big + (n + N) * 2.0 ** -23 + 2.0 ** -20
            tiny = (n + N + 1) * 2.0 ** -126 * max(1.0, np.abs(V[at:at + n]).max(initial=0), np.abs(pick(vd, h)).max(initial=0))
            tol = half * np.abs(want) + (half + e)[:, None] * mass + tiny
            got = pick(o, hq)
            assert (np.abs(got - want) <= tol).all(), (c, g, float((np.abs(got - want) / tol).max()))
            if z is not None:
                gl = z[s, hq, :m] if z.ndim == 3 else z[hq, s * N:s * N + m]
                assert (np.abs(gl - wl) <= 1.45 * e + np.abs(wl) * 2.0 ** -23).all(), (c, g)


CASES = [  # dtype, D, G, N, tree, layout, lens of (2 sequences, 2 heads), n_nodes
    ("bf16", 128, 1, 1, "chain", "packed", (0, 1, 63, 64), None),
    ("bf16", 128, 4, 8, "chain", "fused", (65, 127, 128, 129), None),
    ("bf16", 128, 4, 13, "tree", "padded", (300, 0, 31, 700), (13, 5)),
    ("bf16", 128, 7, 33, "tree", "packed", (257, 3, 1, 90), (7, 33)),
    ("bf16", 128, 16, 5, "star", "fused", (1000, 64, 2, 0), (5, 0)),
    ("bf16", 128, 3, 70, "tree", "packed", (130, 5, 0, 200), None),
    ("bf16", 128, 2, 256, "tree", "fused", (40, 129, 64, 0), (256, 200)),
    ("bf16", 64, 1, 3, "apart", "packed", (0, 0, 0, 5), None),
    ("bf16", 64, 5, 6, "tree", "padded", (64, 65, 66, 500), (1, 6)),
    ("bf16", 64, 8, 20, "tree", "fused", (128, 256, 0, 33), None),
    ("bf16", 64, 2, 130, "tree", "packed", (10, 600, 127, 0), (130, 64)),
    ("f32", 128, 1, 2, "chain", "packed", (0, 1, 64, 63), None),
    ("f32", 128, 4, 12, "tree", "padded", (65, 200, 0, 129), (12, 3)),
    ("f32", 128, 8, 17, "tree", "fused", (333, 1, 64, 0), None),
    ("f32", 64, 2, 9, "tree", "packed", (127, 128, 129, 0), (9, 9)),
    ("f32", 64, 7, 8, "star", "fused", (500, 2, 65, 31), None),
    ("f32", 64, 3, 66, "tree", "padded", (100, 0, 1, 64), (20, 66)),
    ("mxfp4", 128, 1, 1, "chain", "packed", (0, 1, 63, 64), None),
    ("mxfp4", 128, 4, 16, "tree", "fused", (65, 0, 129, 400), (16, 2)),
    ("mxfp4", 128, 16, 9, "tree", "padded", (128, 127, 5, 0), None),
    ("mxfp4", 128, 8, 65, "tree", "packed", (200, 64, 0, 33), None),
    ("mxfp4", 64, 4, 7, "tree", "packed", (66, 1, 0, 500), (7, 1)),
    ("mxfp4", 64, 16, 12, "chain", "fused", (128, 130, 0, 3), None),
    ("mxfp4", 64, 2, 140, "tree", "padded", (64, 65, 300, 0), (100, 140)),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_fp64(case):
    dtype, D, G, N, tree, layout, lens, count = CASES[case]
    a, K, V = make(dtype, D, G, 2, 2, 1, lens, seed=case)
    g = torch.Generator().manual_seed(100 + case)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    q, k, v = nodes(layout, 2, N, 2 * G, D, dt, g), nodes(layout, 2, N, 2, D, dt, g), nodes(layout, 2, N, 2, D, dt, g)
    parent = parents(tree, 2, N, case)
    n_nodes = torch.tensor(count, dtype=torch.int32).cuda() if count is not None else None
    out = torch.full(q.shape, 77.0, dtype=dt, device="cuda")
    lse = torch.full((2, 2 * G, N) if layout == "padded" else (2 * G, 2 * N), 77.0, device="cuda")
    before = a.score.clone(), a.len.clone()
    for t in (k, v, q):  # rows of absent nodes are not looked at
        for b in range(2):
            if count is not None:
                (t[b, :, count[b]:] if t.dim() == 4 else t[b * N + count[b]:(b + 1) * N]).fill_(float("nan"))
    a.tree_attn(0, 1, k, v, torch.from_numpy(parent).cuda(), q, n_nodes=n_nodes, out=out, lse=lse)
    check(a, K, V, k, v, q, parent, count, out, lse, (0, 1), dtype)
    for b in range(2):  # ... nor written
        m = N if count is None else count[b]
        assert ((out[b, :, m:] if out.dim() == 4 else out[b * N + m:(b + 1) * N]) == 77).all()
        assert ((lse[b, :, m:] if layout == "padded" else lse[:, b * N + m:(b + 1) * N]) == 77).all()
    assert torch.equal(a.score, before[0]) and torch.equal(a.len, before[1])


@pytest.mark.parametrize("dtype,D,G,N", [("bf16", 128, 4, 6), ("bf16", 64, 4, 24), ("f32", 128, 2, 7), ("mxfp4", 128, 7, 11)])
def test_long_and_ragged_caches_over_layers(dtype, D, G, N):
    """Caches of many work items beside short ones, layers in one call and one by one, one odd batch."""
    L, batch, Hkv = 3, 3, 2
    rng = np.random.default_rng(D + N)
    lens = np.repeat(rng.choice([70, 900, 5000, 20000], L * Hkv).reshape(L, 1, Hkv), batch, 1)
    lens = (lens - rng.integers(0, 60, lens.shape)).reshape(-1).tolist()
    a, K, V = make(dtype, D, G, Hkv, batch, L, lens, seed=N)
    g = torch.Generator().manual_seed(N)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    q, k, v = (nodes("packed", L * batch, N, h, D, dt, g) for h in (G * Hkv, Hkv, Hkv))
    parent = parents("tree", batch, N, 5)
    p = torch.from_numpy(parent).cuda()
    out, lse = a.tree_attn(0, L, k, v, p, q, want_lse=True)
    check(a, K, V, k, v, q, parent, None, out, lse, (0, L), dtype, only=range(0, L * batch * Hkv, 3))
    again, lse2 = a.tree_attn(0, L, k, v, p, q, want_lse=True)
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    per = batch * N
    for layer in range(L):
        at = slice(layer * per, (layer + 1) * per)
        one, z = a.tree_attn(layer, 1, k[at], v[at], p, q[at], want_lse=True)
        check(a, K, V, k[at], v[at], q[at], parent, None, one, z, (layer, 1), dtype, only=[layer * batch * Hkv + 1])


@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("bf16", 64), ("f32", 64), ("mxfp4", 128)])
def test_infinite_and_nan_rows_of_nodes_that_are_not_seen(dtype, D):
    """Siblings that hold infinities or NaN leave a node's bits as they are; those that see them get them."""
    N, G = 9, 2
    a, K, V = make(dtype, D, G, 1, 1, 1, [100], seed=3)
    g = torch.Generator().manual_seed(4)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    q, k, v = nodes("packed", 1, N, G, D, dt, g), nodes("packed", 1, N, 1, D, dt, g), nodes("packed", 1, N, 1, D, dt, g)
    parent = torch.tensor([[-1, 0, 0, 1, 2, 3, 4, 0, 7]], dtype=torch.int32).cuda()
    want, wl = a.tree_attn(0, 1, k, v, parent, q, want_lse=True)
    sees2, sees7 = [2, 4, 6], [7, 8]
    for plane in ("k", "v"):
        kk, vv = k.clone(), v.clone()
        t = kk if plane == "k" else vv
        t[2, 0, 5], t[7, 0, 40] = float("inf"), float("nan")
        got, gl = a.tree_attn(0, 1, kk, vv, parent, q, want_lse=True)
        clear = [i for i in range(N) if i not in sees2 + sees7]
        assert torch.equal(got[clear], want[clear]) and torch.equal(gl[:, clear], wl[:, clear])
        if plane == "v":
            if dtype == "mxfp4":  # all 32 elements of the scale
                assert got[sees2][:, :, :32].isnan().all() and torch.equal(got[sees2][:, :, 32:], want[sees2][:, :, 32:])
            else:
                assert (got[sees2][:, :, 5] == float("inf")).all() and got[sees7][:, :, 40].isnan().all()
                other = [d for d in range(D) if d != 5]
                assert torch.equal(got[sees2][:, :, other], want[sees2][:, :, other])
            assert torch.equal(gl, wl)
        else:
            assert got[sees7].isnan().all()


@pytest.mark.parametrize("dtype,D,G,N", [("bf16", 128, 4, 6), ("bf16", 128, 8, 8), ("bf16", 128, 4, 40), ("bf16", 64, 1, 1), ("bf16", 64, 3, 90),
                                         ("f32", 128, 2, 3), ("f32", 128, 2, 20), ("f32", 64, 4, 16), ("f32", 64, 4, 60)])
def test_infinite_values_of_the_last_live_row(dtype, D, G, N):
    """An infinity in the last row of a cache, anywhere in a tile, is one in that element of every output, and nothing else changes."""
    a, K, V = make(dtype, D, G, 2, 3, 1, (1, 31, 33, 70, 128, 600), seed=3)
    last = [int(a.off_host[c]) + int(a.len[c]) - 1 for c in range(6)]
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(4)
    k, v = (nodes("packed", 3, N, 2, D, dt, g) for _ in range(2))
    q, parent = nodes("packed", 3, N, 2 * G, D, dt, g), torch.from_numpy(parents("tree", 3, N)).cuda()
    want, lse = a.tree_attn(0, 1, k, v, parent, q, want_lse=True)
    a.v[last, 5], a.v[last, D - 1] = float("inf"), float("-inf")
    got, again = a.tree_attn(0, 1, k, v, parent, q, want_lse=True)
    want[..., 5], want[..., D - 1] = float("inf"), float("-inf")
    assert torch.equal(got, want) and torch.equal(again, lse)


def test_logits_far_apart():
    """Queries whose logits spread over thousands: one key takes everything, in any tile, and the running maximum follows."""
    for dtype in ("bf16", "f32", "mxfp4"):
        a, K, V = make(dtype, 128, 2, 1, 1, 1, [3000], seed=8)
        g = torch.Generator().manual_seed(9)
        dt = torch.float32 if dtype == "f32" else torch.bfloat16
        q = (200 * torch.randn((5, 2, 128), generator=g)).to(dt).cuda()
        k, v = nodes("packed", 1, 5, 1, 128, dt, g), nodes("packed", 1, 5, 1, 128, dt, g)
        parent = parents("tree", 1, 5, 1)
        out, lse = a.tree_attn(0, 1, k, v, torch.from_numpy(parent).cuda(), q, want_lse=True)
        check(a, K, V, k, v, q, parent, None, out, lse, (0, 1), dtype)


def test_a_path_gets_what_steps_get():
    """Nodes of a chain against append_decode_attn over the same tokens one by one."""
    for dtype in ("bf16", "f32", "mxfp4"):
        N, G, D, Hkv, batch = 6, 4, 128, 2, 2
        a, K, V = make(dtype, D, G, Hkv, batch, 1, [700, 33, 128, 5], room=N, seed=6)
        g = torch.Generator().manual_seed(7)
        dt = torch.float32 if dtype == "f32" else torch.bfloat16
        q, k, v = (nodes("packed", batch, N, h, D, dt, g) for h in (G * Hkv, Hkv, Hkv))
        parent = parents("chain", batch, N)
        out = a.tree_attn(0, 1, k, v, torch.from_numpy(parent).cuda(), q)
        step = torch.empty((batch, G * Hkv, D), device="cuda")
        for t in range(N):
            at = torch.arange(batch, device="cuda") * N + t
            a.append_decode_attn(0, 1, k[at].contiguous(), v[at].contiguous(), t, q[at].contiguous(), step)
            # both are within rounding of the exact result: half a step of the output and of the weights in bf16, fp32 otherwise
            tol = 2.0 ** -18 if dtype == "f32" else 2.0 ** -7
            far = (out[at].float() - step).abs()
            assert (far <= tol * (step.abs() + 1)).all(), (dtype, t, float(far.max()))


def test_parents_that_are_no_earlier_node():
    a, K, V = make("bf16", 128, 1, 1, 1, 1, [20])
    g = torch.Generator().manual_seed(1)
    q, k, v = (nodes("packed", 1, 6, 1, 128, torch.bfloat16, g) for _ in range(3))
    odd = torch.tensor([[5, 0, 2, 99, -7, 1]], dtype=torch.int32).cuda()
    plain = torch.tensor([[-1, 0, -1, -1, -1, 1]], dtype=torch.int32).cuda()
    assert torch.equal(a.tree_attn(0, 1, k, v, odd, q), a.tree_attn(0, 1, k, v, plain, q))
    for n in (-4, 0, 3, 6, 1000):
        out = torch.zeros_like(q)
        a.tree_attn(0, 1, k, v, plain, q, n_nodes=torch.tensor([n], dtype=torch.int32).cuda(), out=out)
        m = min(max(n, 0), 6)
        assert (out[m:] == 0).all() and (m == 0 or (out[:m] != 0).any())


def test_offsets_beyond_32_bits():
    """A cache whose rows end behind 2^32 bytes of its plane."""
    n = (1 << 24) + 77
    a = B.Arena(1, 2, 1, 128, 2, "bf16", [n], 4, 0, 0)
    a.k.fill_(0.25), a.v.zero_()
    last = int(a.off_host[1]) + n - 1
    for r in (int(a.off_host[1]), last - 5, last):
        a.v[r] = float(1 << 20)
    a.set_lengths([0, n])
    g = torch.Generator().manual_seed(1)
    q, k, v = (nodes("packed", 2, 3, h, 128, torch.bfloat16, g) for h in (2, 1, 1))
    k.fill_(0.25), v.zero_(), q.fill_(0.5)
    out, lse = a.tree_attn(0, 1, k, v, torch.from_numpy(parents("chain", 2, 3)).cuda(), q, want_lse=True)
    for i in range(3):  # equal weights: 3 of the n + i + 1 rows hold 2^20
        want = 3.0 * (1 << 20) / (n + i + 1)
        assert (out[3 + i].double() - want).abs().max() <= 2.0 ** -7 * want + 1e-30
        wl = np.log2(n + i + 1) + 128 * 0.125 / np.sqrt(128) * np.log2(np.e)
        assert (lse[:, 3 + i].double() - wl).abs().max() <= 1e-4  # (sums of 2^24 terms: within 2^-14)


@pytest.mark.parametrize("dtype,G,N", [("bf16", 7, 50), ("bf16", 16, 40), ("f32", 8, 30), ("mxfp4", 4, 31), ("mxfp4", 8, 100)])
def test_many_query_rows_behind_long_caches(dtype, G, N):
    """Several workgroups for the query rows of a work item, several work items for a cache, trees of different sizes."""
    lens = [9000, 40, 3000, 129]
    a, K, V = make(dtype, 128, G, 2, 2, 1, lens, seed=N)
    g = torch.Generator().manual_seed(N)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    q, k, v = (nodes("packed", 2, N, h, 128, dt, g) for h in (2 * G, 2, 2))
    parent, count = parents("tree", 2, N, 7), (N, N // 3)
    out, lse = torch.zeros_like(q), torch.zeros((2 * G, 2 * N), device="cuda")
    a.tree_attn(0, 1, k, v, torch.from_numpy(parent).cuda(), q, n_nodes=torch.tensor(count, dtype=torch.int32).cuda(), out=out, lse=lse)
    check(a, K, V, k, v, q, parent, count, out, lse, (0, 1), dtype)


@pytest.mark.parametrize("dtype,N", [("bf16", 3), ("bf16", 40), ("f32", 2), ("mxfp4", 5)])
@pytest.mark.parametrize("L,batch,Hkv", [(3, 8, 4), (5, 9, 16)])
def test_more_caches_than_a_workgroup_has_threads(dtype, N, L, batch, Hkv):
    """96 caches, and 720, some of them long, some empty, sequences without nodes among them."""
    rng = np.random.default_rng(L)
    lens = rng.integers(0, 150, (L, batch, Hkv))
    lens[1, 2, :] = 0
    lens[0, 1, 1], lens[L - 1, batch - 1, Hkv - 1] = 5000, 2500
    a, K, V = make(dtype, 64, 2, Hkv, batch, L, lens.reshape(-1).tolist(), seed=9)
    g = torch.Generator().manual_seed(L)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    q, k, v = (nodes("packed", L * batch, N, h, 64, dt, g) for h in (2 * Hkv, Hkv, Hkv))
    parent = parents("tree", batch, N, 2)
    count = rng.integers(0, N + 1, batch)
    count[2], count[3] = N, 0
    out, lse = torch.zeros_like(q), torch.zeros((2 * Hkv, L * batch * N), device="cuda")
    a.tree_attn(0, L, k, v, torch.from_numpy(parent).cuda(), q, n_nodes=torch.from_numpy(count).int().cuda(), out=out, lse=lse)
    some = sorted({1 * Hkv + 1, a.n_caches - 1} | set(rng.choice(a.n_caches, 40, replace=False).tolist()))
    check(a, K, V, k, v, q, parent, count, out, lse, (0, L), dtype, only=some)


def test_refusals():
    a, K, V = make("bf16", 128, 2, 2, 2, 2, [10] * 8, track=True)
    g = torch.Generator().manual_seed(1)
    N = 4
    q, k, v = (nodes("packed", 4, N, h, 128, torch.bfloat16, g) for h in (4, 2, 2))
    p = torch.from_numpy(parents("chain", 2, N)).cuda()
    n = torch.tensor([1, 2], dtype=torch.int32).cuda()
    a.tree_attn(0, 2, k, v, p, q)
    for bad in (dict(parent=p.long()), dict(parent=p[:1]), dict(parent=p.cpu()), dict(parent=p[:, ::2]), dict(n_nodes=n[:1]), dict(n_nodes=n.float()),
                dict(n_nodes=n.cpu()), dict(q=q.float()), dict(q=q[:-1]), dict(k=k[:, :1]), dict(v=v[..., :64]), dict(q=q.cpu()), dict(out=q.float()),
                dict(lse=torch.zeros((4, 4 * N), device="cuda").half()), dict(lse=torch.zeros((3, 4 * N), device="cuda")), dict(q=q.clone().requires_grad_())):
        with pytest.raises(ValueError):
            a.tree_attn(0, 2, **(dict(k=k, v=v, parent=p, q=q) | bad))
    for first, count in ((0, 3), (-1, 1), (2, 1), (1, 0)):
        with pytest.raises((B.BaklavaError, ValueError)):
            a.tree_attn(first, count, k, v, p, q)
    big = torch.zeros((2, 257), dtype=torch.int32).cuda()
    wide = [torch.zeros((4 * 257, h, 128), dtype=torch.bfloat16, device="cuda") for h in (2, 2, 4)]
    with pytest.raises(B.BaklavaError) as e:
        a.tree_attn(0, 2, wide[0], wide[1], big, wide[2])
    assert e.value.status == B.EINVAL
    # misaligned rows, outputs that overlap, a workspace that is too small
    odd = torch.zeros(4 * N * 4 * 128 + 8, dtype=torch.bfloat16, device="cuda")[4:4 + 4 * N * 4 * 128].view(4 * N, 4, 128)
    for bad in (dict(q=odd), dict(out=odd), dict(out=q[:1].expand(4 * N, 4, 128))):
        with pytest.raises(B.BaklavaError) as e:
            a.tree_attn(0, 2, **(dict(k=k, v=v, parent=p, q=q) | bad))
        assert e.value.status == B.EINVAL
    lib, rows = B.lib(), B._Rows(torch)
    at = [rows.add(t, "t", 4, 4 * N, N, t.shape[1], 128, torch.bfloat16) for t in (q, k, v)]
    need = lib.baklava_tree_workspace_bytes(a.ctx, 2, N)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    call = lambda nbytes, at_ws: lib.baklava_tree_attn(a.ctx, 0, 2, at[1], at[2], N, p.data_ptr(), None, at[0], at[0], None, at_ws, nbytes, None)
    assert call(need - 1, ws.data_ptr()) == B.ECAPACITY and call(need, ws.data_ptr() + 64) == B.EINVAL and call(need, None) == B.EINVAL
    assert lib.baklava_tree_workspace_bytes(a.ctx, 3, N) == lib.baklava_tree_workspace_bytes(a.ctx, 0, N) == lib.baklava_tree_workspace_bytes(a.ctx, 1, 257) == 0


def test_two_calls_at_once():
    """Calls on two streams over the same caches, each with outputs and a workspace of its own."""
    a, K, V = make("bf16", 128, 4, 2, 2, 1, [4000, 300, 2000, 9000])
    g = torch.Generator().manual_seed(5)
    sets = [[nodes("packed", 2, N, h, 128, torch.bfloat16, g) for h in (8, 2, 2)] + [torch.from_numpy(parents("tree", 2, N)).cuda()] for N in (5, 40)]
    want = [a.tree_attn(0, 1, k, v, p, q, want_lse=True) for q, k, v, p in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        got = [a.tree_attn(0, 1, k, v, p, q, want_lse=True, stream=s) for (q, k, v, p), s in zip(sets, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for gs, ws in zip(got, want) for x, y in zip(gs, ws))
