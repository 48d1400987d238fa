"""GPU parity: the accepted path's rows and scores into the caches (baklava_append_accepted), and the three calls of a step over
drafted tokens as they are used: behind prompts, steps and evictions, captured and replayed."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as DO
from oracle import operators_oracle as OP
from paper_2502_13176_amd import binding as B
from test_gpu_tree import make, nodes, parents, stored

pytestmark = pytest.mark.gpu


def expected_scores(K, lens_of, kd, qd, lse, path, n_path, c, Hkv, batch, N, G, D, at):
    """What cache c's scores gain, [n + P], and how far fp32 may be off: a weight by its logit's absolute error (as for the attention),
    2^-22 of the exponential and half a step of lse; sums of P G weights and the addition to the plane by as many half steps."""
    s, h = c // Hkv, c % Hkv
    b, n = s % batch, lens_of[c]
    P = int(n_path[b])
    pick = lambda t, i: t[s, i] if t.ndim == 4 else t[s * N:(s + 1) * N, i]
    zl = lambda i: lse[s, i] if lse.ndim == 3 else lse[i, s * N:(s + 1) * N]
    nodes_ = [int(x) for x in path[b][:P]]
    q = np.stack([pick(qd, h * G + g)[nodes_] for g in range(G)], 1)
    z = np.stack([zl(h * G + g)[nodes_] for g in range(G)], 1)
    add, big = DO.path_scores(np.concatenate([K[at:at + n], pick(kd, h)[nodes_]]), q, z, n)
    e = 2 * (D + 2) * 2.0 ** -24 * big + 2.0 ** -22 + np.abs(z).max(initial=0) * 2.0 ** -23 + (P * G + 2) * 2.0 ** -24
    return add, e


CASES = [  # dtype, D, G, N, layout, lens of (2 layers, 2 sequences, 2 heads), paths
    ("bf16", 128, 4, 8, "packed", (65, 0, 129, 700, 1, 31, 32, 33), ([0, 2, 5], [0])),
    ("bf16", 128, 1, 1, "fused", (0, 1, 2, 300, 63, 64, 127, 128), ([0], [0])),
    ("bf16", 128, 16, 40, "padded", (200, 5, 0, 1000, 90, 1, 4, 7), (list(range(40)), [0, 3, 39])),
    ("bf16", 128, 7, 30, "packed", (400, 31, 3, 77, 0, 0, 9, 256), (list(range(0, 30, 2)), [])),
    ("bf16", 64, 8, 12, "fused", (129, 2, 600, 0, 5, 96, 97, 160), ([0, 1, 2, 3], [0, 11])),
    ("bf16", 64, 2, 256, "packed", (50, 1, 64, 0, 7, 8, 9, 300), (list(range(0, 256)), [0, 255])),
    ("f32", 128, 8, 6, "padded", (130, 0, 33, 500, 2, 64, 65, 1), ([0, 1, 2, 3, 4, 5], [0, 2])),
    ("f32", 128, 3, 20, "packed", (30, 31, 0, 222, 4, 4, 4, 4), (list(range(0, 20, 1)), [0])),
    ("f32", 64, 4, 9, "fused", (700, 1, 95, 96, 0, 12, 13, 14), ([0, 8], [0, 4, 5])),
    ("mxfp4", 128, 4, 16, "packed", (65, 0, 129, 700, 1, 31, 32, 33), ([0, 2, 5, 15], [0])),
    ("mxfp4", 128, 16, 11, "fused", (64, 300, 2, 0, 95, 1, 128, 5), (list(range(11)), [])),
    ("mxfp4", 64, 5, 7, "padded", (127, 1, 0, 450, 33, 34, 35, 36), ([0, 3], [0, 1, 2, 3, 4, 5, 6])),
]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("track", [False, True])
def test_against_fp64(case, track):
    dtype, D, G, N, layout, lens, paths = CASES[case]
    L, batch, Hkv = 2, 2, 2
    a, K, V = make(dtype, D, G, Hkv, batch, L, lens, room=N + 3, seed=case, track=track)
    g = torch.Generator().manual_seed(50 + case)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    q, k, v = (nodes(layout, L * batch, N, h, D, dt, g) for h in (G * Hkv, Hkv, Hkv))
    a.score.copy_(torch.rand((a.total_tokens,), generator=g)), a.pos.fill_(-7)
    n_path = [len(p) for p in paths]
    path = np.full((batch, N), -1, dtype=np.int32)
    for b, p in enumerate(paths):
        path[b, :len(p)] = p
    # normalisers of queries that see everything up to themselves
    lse = torch.full((L * batch, G * Hkv, N) if layout == "padded" else (G * Hkv, L * batch * N), float("nan"))
    kd, vd, qd = stored(k, dtype), stored(v, dtype), q.double().cpu().numpy()
    pick = lambda t, s, i: t[s, i] if t.ndim == 4 else t[s * N:(s + 1) * N, i]
    for c, n in enumerate(lens):
        s, h, at = c // Hkv, c % Hkv, int(a.off_host[c])
        for t, i in enumerate(paths[s % batch]):
            kk = np.concatenate([K[at:at + n], pick(kd, s, h)[paths[s % batch][:t + 1]]])
            for hq in range(h * G, (h + 1) * G):
                z = np.log2(np.exp2(kk @ pick(qd, s, hq)[i] * np.log2(np.e) / np.sqrt(D)).sum())
                if layout == "padded":
                    lse[s, hq, i] = z
                else:
                    lse[hq, s * N + i] = z
    before = [x.clone() for x in (a.k, a.v, a.score, a.pos)]
    pos0 = torch.tensor([1000, 2000], dtype=torch.int32).cuda()
    a.append_accepted(0, L, k, v, torch.from_numpy(path).cuda(), torch.tensor(n_path, dtype=torch.int32).cuda(), pos0,
                      q=q if track else None, lse=lse.cuda() if track else None)
    a.sync_lengths()
    want_len = [n + n_path[c // Hkv % batch] for c, n in enumerate(lens)]
    assert a.lengths().tolist() == want_len
    score, pos, ln = a.score.double().cpu().numpy(), a.pos.cpu().numpy(), lse.double().numpy()
    old = before[2].double().cpu().numpy()
    k2, v2 = a.read_rows(0, L, N)
    for c, n in enumerate(lens):
        s, h, at = c // Hkv, c % Hkv, int(a.off_host[c])
        P, p = n_path[s % batch], paths[s % batch]
        rows = slice(at + n, at + n + P)
        assert pos[rows].tolist() == [1000 * (s % batch + 1) + t for t in range(P)]
        for got, x in ((k2, kd), (v2, vd)):
            assert np.array_equal(got[c, N - P:].double().cpu().numpy(), pick(x, s, h)[p]), c
        if track:
            add, e = expected_scores(K, lens, kd, qd, ln, path, n_path, c, Hkv, batch, N, G, D, at)
            want = np.concatenate([old[at:at + n], np.zeros(P)]) + add
            far = np.abs(score[at:at + n + P] - want)
            assert (far <= e * add + np.abs(want) * 2.0 ** -23).all(), (c, float((far / (e * add + np.abs(want) * 2.0 ** -23 + 1e-300)).max()))
        else:
            assert np.array_equal(score[at:at + n], old[at:at + n]) and (score[rows] == 0).all()
        # nothing else has changed
        for now, was in ((a.k, before[0]), (a.v, before[1]), (a.pos, before[3]), (a.score, before[2])):
            end = at + int(a.cap_host[c])
            bits = lambda x: x.contiguous().view(torch.uint8)
            assert torch.equal(bits(now[at + n + P:end]), bits(was[at + n + P:end]))
            if now is not a.score:
                assert torch.equal(bits(now[at:at + n]), bits(was[at:at + n]))


@pytest.mark.parametrize("dtype", ["bf16", "f32", "mxfp4"])
def test_caches_without_room_stay_as_they_are(dtype):
    a, K, V = make(dtype, 128, 2, 2, 1, 2, [10, 40, 40, 7], room=0, track=True)
    a.set_lengths([10 - 3, 40 - 2, 40 - 3, 7])
    g = torch.Generator().manual_seed(1)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    q, k, v = (nodes("packed", 2, 5, h, 128, dt, g) for h in (4, 2, 2))
    lse = torch.full((4, 10), 9.0).cuda()
    path, n = torch.tensor([[0, 1, 2, -1, -1]], dtype=torch.int32).cuda(), torch.tensor([3], dtype=torch.int32).cuda()
    before = a.score.clone(), a.pos.clone()
    a.append_accepted(0, 2, k, v, path, n, n, q=q, lse=lse)
    with pytest.raises(B.BaklavaError) as e:
        a.sync_lengths()
    assert e.value.status == B.ECAPACITY and a.lengths().tolist() == [10, 38, 40, 7]
    for c, full in ((1, True), (3, True), (0, False), (2, False)):
        at = slice(int(a.off_host[c]), int(a.off_host[c]) + int(a.cap_host[c]))
        assert torch.equal(a.score[at], before[0][at]) == full and torch.equal(a.pos[at], before[1][at]) == full
    a.sync_lengths()  # reported once


def test_paths_that_end_early():
    """n_path beyond N, entries that are no node: the path ends there."""
    for p, count, want in (([0, 2, 9, 1, -1], 5, 2), ([0, 1, 2, 3, 4], 99, 5), ([-1, 0, 0, 0, 0], 3, 0), ([0, 1, 1, 0, 4], 4, 4), ([0, 1, 2, 3, 4], -3, 0)):
        a, K, V = make("bf16", 64, 1, 1, 1, 1, [20], room=9)
        g = torch.Generator().manual_seed(1)
        k, v = nodes("packed", 1, 5, 1, 64, torch.bfloat16, g), nodes("packed", 1, 5, 1, 64, torch.bfloat16, g)
        a.append_accepted(0, 1, k, v, torch.tensor([p], dtype=torch.int32).cuda(), torch.tensor([count], dtype=torch.int32).cuda(),
                          torch.tensor([5], dtype=torch.int32).cuda())
        a.sync_lengths()
        assert a.lengths().tolist() == [20 + want]
        if want:
            assert torch.equal(a.read_rows(0, 1, want)[0][0], k[p[:want], 0])


@pytest.mark.parametrize("dtype,D,G", [("bf16", 128, 4), ("bf16", 64, 2), ("f32", 128, 2), ("mxfp4", 128, 4)])
def test_drafted_steps_are_steps(dtype, D, G):
    """Several steps over drafted trees, with tracked scores, an eviction between them, beside an arena that takes the accepted tokens one
    by one: the same rows, positions and lengths, scores and outputs within rounding."""
    L, batch, Hkv, N, V = 2, 2, 2, 7, 50
    lens = [150, 90, 150, 90, 60, 200, 60, 200]
    pair = []
    for _ in range(2):
        a, _, _ = make(dtype, D, G, Hkv, batch, L, [n + 30 for n in lens], room=40, seed=4, track=True)
        budgets = [lens[0], lens[1], lens[4], lens[5]]
        b = B.Arena(L, G * Hkv, Hkv, D, batch, dtype, budgets, 70, 4, 16, B.POLICY_SCORE, True, workspace_fill=0xFF)
        for c in range(len(lens)):
            src, dst = int(a.off_host[c]), int(b.off_host[c])
            for x, y in ((a.k, b.k), (a.v, b.v), (a.kv_scale, b.kv_scale)):
                if x is not None:
                    y[dst:dst + lens[c]] = x[src:src + lens[c]]
            b.pos[dst:dst + lens[c]] = torch.arange(lens[c], dtype=torch.int32, device="cuda")
        b.set_lengths(lens)
        pair.append(b)
    spec, plain = pair
    g = torch.Generator().manual_seed(11)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    rng = np.random.default_rng(2)
    at_pos = torch.tensor([500, 800], dtype=torch.int32).cuda()
    for step in range(6):
        q, k, v = (nodes("packed", L * batch, N, h, D, dt, g) for h in (G * Hkv, Hkv, Hkv))
        parent = torch.from_numpy(parents("tree", batch, N, step)).cuda()
        parent[:, 1] = 0
        logits = 3 * torch.randn((batch, N, V), generator=g).cuda()
        token = logits.argmax(2).gather(1, parent.clamp(min=0).long()).int()  # every node is its parent's likeliest token
        u = (0.5 * torch.rand((batch, N), generator=g)).cuda()
        out, lse = torch.empty_like(q), torch.empty((G * Hkv, L * batch * N), device="cuda")
        for layer in range(L):
            sl = slice(layer * batch * N, (layer + 1) * batch * N)
            spec.tree_attn(layer, 1, k[sl], v[sl], parent, q[sl], out=out[sl], lse=lse[:, sl])
        path, n_path, nxt = B.verify_draft(logits, token, parent, u)
        spec.append_accepted(0, L, k, v, path, n_path, at_pos, q=q, lse=lse)
        spec.sync_lengths()
        # one by one: sequences of different paths take turns; one that is done takes steps of its own elsewhere
        P, counts = path.cpu().numpy(), n_path.cpu().numpy()
        for t in range(counts.max()):
            on = [b for b in range(batch) if t < counts[b]]
            keep = {c: int(plain.lengths()[c]) for c in range(len(lens))}
            rows = torch.tensor([[(l * batch + b) * N + int(P[b][min(t, counts[b] - 1)]) for b in range(batch)] for l in range(L)]).cuda()
            plain.flush_scores(0, L)
            was = plain.score.clone()
            got = torch.empty((L, batch, G * Hkv, D), device="cuda")
            plain.append_decode_attn(0, L, k[rows].contiguous(), v[rows].contiguous(), 0, q[rows].contiguous(), got)
            plain.flush_scores(0, L)
            now = plain.lengths().tolist()
            for c in range(len(lens)):
                b = c // Hkv % batch
                base = int(plain.off_host[c])
                if b not in on:  # taken back
                    now[c] = keep[c]
                    plain.score[base:base + int(plain.cap_host[c])] = was[base:base + int(plain.cap_host[c])]
                else:
                    plain.pos[base + keep[c]] = int(at_pos[b]) + t
            plain.set_lengths(now)
            for l in range(L):
                for b in on:
                    x, y = out[rows[l, b]].float(), got[l, b]
                    tol = 2.0 ** -18 if dtype == "f32" else 2.0 ** -7
                    assert ((x - y).abs() <= tol * (y.abs() + 1)).all(), (step, t, l, b)
        at_pos = at_pos + n_path
        assert spec.lengths().tolist() == plain.lengths().tolist()
        for c, n in enumerate(spec.lengths()):
            x = slice(int(spec.off_host[c]), int(spec.off_host[c]) + int(n))
            for p1, p2 in ((spec.k, plain.k), (spec.v, plain.v), (spec.pos, plain.pos)):
                assert torch.equal(p1[x], p2[x]), (step, c)
            assert ((spec.score[x] - plain.score[x]).abs() <= 2.0 ** -14 * (plain.score[x] + 2.0 ** -10)).all(), (step, c)
        if step % 2:
            plain.score.copy_(spec.score)  # (an eviction ranks by bits)
            for a in pair:
                a.compact(0, L)
            assert spec.lengths().tolist() == plain.lengths().tolist()


@pytest.mark.parametrize("dtype", ["bf16", "f32", "mxfp4"])
def test_captured_step_replays_with_new_trees(dtype):
    """Attention, verification and appending captured once and replayed with other trees, tokens and lengths, eager work in between."""
    L, batch, Hkv, G, D, N, V = 2, 2, 2, 2, 128, 6, 300
    lens = [40, 3, 200, 64, 0, 9, 30, 31]
    arenas = [make(dtype, D, G, Hkv, batch, L, lens, room=60, seed=1, track=True)[0] for _ in range(2)]
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(3)

    def inputs(step):
        q, k, v = (nodes("packed", L * batch, N, h, D, dt, g) for h in (G * Hkv, Hkv, Hkv))
        parent = torch.from_numpy(parents(["tree", "chain", "star"][step % 3], batch, N, step)).cuda()
        logits = 3 * torch.randn((batch, N, V), generator=g).cuda()
        token = logits.argmax(2).gather(1, parent.clamp(min=0).long()).int()
        return [q, k, v, parent, logits, token, torch.rand((batch, N), generator=g).cuda(), torch.full((batch,), 7 * step, dtype=torch.int32).cuda(),
                torch.tensor([N, N - step % 3], dtype=torch.int32).cuda()]

    def step_of(a, x):
        q, k, v, parent, logits, token, u, pos0, n = x
        out, lse = a.tree_attn(0, L, k, v, parent, q, n_nodes=n, want_lse=True)
        path, n_path, nxt = B.verify_draft(logits, token, parent, u, n_nodes=n)
        a.append_accepted(0, L, k, v, path, n_path, pos0, q=q, lse=lse)
        return out, lse, path, n_path, nxt

    static = inputs(0)
    warm = make(dtype, D, G, Hkv, batch, L, lens, room=60, seed=1, track=True)[0]
    step_of(warm, static)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = step_of(arenas[0], static)
    for step in range(1, 6):
        x = inputs(step)
        for dst, src in zip(static, x):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in res]
        want = step_of(arenas[1], x)
        valid = torch.arange(N).expand(batch, N) < x[-1].cpu().unsqueeze(1)
        on = valid.reshape(-1).repeat(L).cuda()
        assert torch.equal(got[0][on], want[0][on]) and torch.equal(got[1][:, on], want[1][:, on])
        assert all(torch.equal(s, t) for s, t in zip(got[2:], want[2:]))
        for a in arenas:
            a.sync_lengths()
        assert arenas[0].lengths().tolist() == arenas[1].lengths().tolist()
        for c, n in enumerate(arenas[0].lengths()):
            r = slice(int(arenas[0].off_host[c]), int(arenas[0].off_host[c]) + int(n))
            for p in ("k", "v", "score", "pos"):
                assert torch.equal(getattr(arenas[0], p)[r], getattr(arenas[1], p)[r]), (step, c, p)
        torch.randn((1000, 1000), device="cuda").sum().item()


def test_another_stream_while_the_current_one_is_busy():
    a, K, V = make("bf16", 128, 2, 2, 1, 1, [500, 300], room=20, track=True)
    g = torch.Generator().manual_seed(2)
    N = 5
    q, k, v = (nodes("packed", 1, N, h, 128, torch.bfloat16, g) for h in (4, 2, 2))
    parent = torch.from_numpy(parents("tree", 1, N)).cuda()
    logits, token, u = torch.randn((1, N, 900), generator=g).cuda(), torch.randint(0, 900, (1, N), generator=g).int().cuda(), torch.rand((1, N), generator=g).cuda()
    want = a.tree_attn(0, 1, k, v, parent, q, want_lse=True)
    told = B.verify_draft(logits, token, parent, u)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    torch.cuda._sleep(20_000_000)
    got = a.tree_attn(0, 1, k, v, parent, q, want_lse=True, stream=s)
    path, n_path, nxt = B.verify_draft(logits, token, parent, u, stream=s)
    a.append_accepted(0, 1, k, v, path, n_path, n_path, q=q, lse=got[1], stream=s)
    a.sync_lengths(stream=s)
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and all(torch.equal(x, y) for x, y in zip((path, n_path, nxt), told))
    assert a.lengths().tolist() == [500 + int(n_path[0]), 300 + int(n_path[0])]
    torch.cuda.synchronize()


def test_refusals():
    a, K, V = make("bf16", 128, 2, 2, 1, 2, [10] * 4, room=20, track=True)
    g = torch.Generator().manual_seed(1)
    q, k, v = (nodes("packed", 2, 5, h, 128, torch.bfloat16, g) for h in (4, 2, 2))
    lse = torch.full((4, 10), 9.0).cuda()
    path, n = torch.zeros((1, 5), dtype=torch.int32).cuda(), torch.ones(1, dtype=torch.int32).cuda()
    with pytest.raises(B.BaklavaError) as e:  # scores are tracked
        a.append_accepted(0, 2, k, v, path, n, n)
    assert e.value.status == B.EINVAL
    good = dict(k=k, v=v, path=path, n_path=n, pos0=n, q=q, lse=lse)
    for bad in (dict(path=path.long()), dict(path=path[0]), dict(path=path.cpu()), dict(n_path=torch.ones(2, dtype=torch.int32).cuda()), dict(pos0=n.float()),
                dict(q=None), dict(lse=None), dict(k=k.float()), dict(v=v[:-1]), dict(q=q[:, :2]), dict(lse=lse.double()), dict(lse=lse[:, :9])):
        with pytest.raises(ValueError):
            a.append_accepted(0, 2, **(good | bad))
    for first, count in ((0, 3), (-1, 1), (2, 1)):
        with pytest.raises((B.BaklavaError, ValueError)):
            a.append_accepted(first, count, **good)
    a.sync_lengths()
    assert a.lengths().tolist() == [10] * 4
    a.set_option(B.OPT_TRACK_SCORES, 0)  # paused: they are not looked at
    before = a.score.clone()
    a.append_accepted(0, 2, k, v, path, n, n)
    a.sync_lengths()
    for c in range(4):
        o = int(a.off_host[c])
        assert torch.equal(a.score[o:o + 10], before[o:o + 10])
    assert a.lengths().tolist() == [11] * 4


@pytest.mark.parametrize("dtype", ["bf16", "mxfp4"])
def test_pending_calls_and_accepted_paths_add_up(dtype):
    """Tracked steps that are still on record, a path behind them, steps behind that: the scores an eviction finds hold all of them."""
    L, Hkv, G, D, N = 1, 2, 4, 128, 5
    a, K, V = make(dtype, D, G, Hkv, 1, L, [200, 77], room=40, seed=1, track=True)
    g = torch.Generator().manual_seed(4)
    steps = [[nodes("packed", 1, 1, h, D, torch.bfloat16, g) for h in (G * Hkv, Hkv, Hkv)] for _ in range(7)]
    q, k, v = (nodes("packed", 1, N, h, D, torch.bfloat16, g) for h in (G * Hkv, Hkv, Hkv))
    out = torch.empty((1, G * Hkv, D), device="cuda")
    for t, (qs, ks, vs) in enumerate(steps[:3]):
        a.append_decode_attn(0, 1, ks, vs, t, qs, out)
    parent = torch.from_numpy(parents("chain", 1, N)).cuda()
    _, lse = a.tree_attn(0, 1, k, v, parent, q, want_lse=True)
    path, n, pos = torch.arange(N, dtype=torch.int32).view(1, N).cuda(), torch.tensor([N], dtype=torch.int32).cuda(), torch.tensor([3], dtype=torch.int32).cuda()
    a.append_accepted(0, 1, k, v, path, n, pos, q=q, lse=lse)
    a.sync_lengths()
    for t, (qs, ks, vs) in enumerate(steps[3:]):
        a.append_decode_attn(0, 1, ks, vs, 3 + N + t, qs, out)
    a.flush_scores(0, 1)
    for c, n0 in enumerate((200, 77)):
        o, total = int(a.off_host[c]), n0 + 7 + N
        score = a.score[o:o + total].double().cpu()
        # every query's weights add up to 1 a head: 2^-10 of it is far more than fp32 loses
        assert abs(float(score.sum()) - G * (7 + N)) <= 2.0 ** -10 * G * (7 + N)
        rows = [stored(ks, dtype)[0, c] for _, ks, _ in steps[:3]] + [stored(k, dtype)[i, c] for i in range(N)] + [stored(ks, dtype)[0, c] for _, ks, _ in steps[3:]]
        all_k = np.concatenate([K[o:o + n0], np.stack(rows)])
        qd = [s[0][0, c * G:(c + 1) * G] for s in steps[:3]] + [q[i, c * G:(c + 1) * G] for i in range(N)] + [s[0][0, c * G:(c + 1) * G] for s in steps[3:]]
        want = np.zeros(total)
        for t, x in enumerate(qd):
            for y in x.double().cpu().numpy():
                s = all_k[:n0 + t + 1] @ y / np.sqrt(D)
                e = np.exp(s - s.max())
                want[:n0 + t + 1] += e / e.sum()
        assert np.abs(score.numpy() - want).max() <= 2e-3 * max(1.0, want.max())


def test_many_caches_and_a_long_one():
    """720 caches of which some take no path, and one of 40000 rows, in one call."""
    L, batch, Hkv, G, D, N = 5, 9, 16, 2, 64, 6
    rng = np.random.default_rng(1)
    lens = rng.integers(0, 90, (L, batch, Hkv))
    lens[2, 4, 3] = 40000
    a, K, V = make("bf16", D, G, Hkv, batch, L, lens.reshape(-1).tolist(), room=N, seed=2, track=True)
    g = torch.Generator().manual_seed(3)
    q, k, v = (nodes("packed", L * batch, N, h, D, torch.bfloat16, g) for h in (G * Hkv, Hkv, Hkv))
    parent = torch.from_numpy(parents("chain", batch, N)).cuda()
    _, lse = a.tree_attn(0, L, k, v, parent, q, want_lse=True)
    n_path = rng.integers(0, N + 1, batch)
    n_path[4] = 5
    path = np.full((batch, N), -1, dtype=np.int32)
    for b in range(batch):
        path[b, :n_path[b]] = np.arange(n_path[b])
    n = torch.from_numpy(n_path).int().cuda()
    a.append_accepted(0, L, k, v, torch.from_numpy(path).cuda(), n, n, q=q, lse=lse)
    a.sync_lengths()
    assert a.lengths().tolist() == (lens + n_path.reshape(1, -1, 1)).reshape(-1).tolist()
    score, kd, qd, ln = a.score.double().cpu().numpy(), stored(k, "bf16"), q.double().cpu().numpy(), lse.double().cpu().numpy()
    flat = lens.reshape(-1)
    for c in sorted({(2 * batch + 4) * Hkv + 3} | set(rng.choice(a.n_caches, 60, replace=False).tolist())):
        P, o = int(n_path[c // Hkv % batch]), int(a.off_host[c])
        add, e = expected_scores(K, flat, kd, qd, ln, path, n_path, c, Hkv, batch, N, G, D, o)
        got = score[o:o + flat[c] + P]
        assert (np.abs(got - add[:len(got)]) <= e * add[:len(got)] + add[:len(got)] * 2.0 ** -23).all(), c
