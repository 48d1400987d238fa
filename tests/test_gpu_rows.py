"""GPU parity: baklava_append_prompt and baklava_read_rows, and the whole way of a prompt through the library."""
import numpy as np
import pytest
import torch

from oracle import baklava_oracle as O
from oracle import operators_oracle as OP
from paper_2502_13176_amd import binding as B

pytestmark = pytest.mark.gpu


def arena(dtype, D=64, L=2, batch=3, Hkv=2, cap=200, **kw):
    a = B.Arena(L, 2 * Hkv, Hkv, D, batch, dtype, [cap] * (L * Hkv), 0, 0, 0, **kw)
    a.score.fill_(-5.0), a.pos.fill_(-7)
    a.k.fill_(3), a.v.fill_(3)
    return a


def stored(x, dtype):
    """What a cache holds of rows x [..., D]."""
    x = x.double().cpu().numpy()
    if dtype == "mxfp4":
        code, s = OP.mx_round(x)
        return OP.mx_values(OP.mx_pack(code), s)
    return x


def rows(dtype, layout, lens, H, D, g):
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    n = sum(lens)
    if layout == "packed":
        return torch.randn((n, H, D), generator=g).to(dt).cuda()
    if layout == "fused":
        return torch.randn((n, H + 3, D), generator=g).to(dt).cuda()[:, 1:1 + H]
    if layout == "heads":
        return torch.randn((H, n, D), generator=g).to(dt).cuda().transpose(0, 1)
    return torch.randn((len(lens), H, max(lens) + 2, D), generator=g).to(dt).cuda()


def of_sequence(t, b, lens):
    return t[b, :, :lens[b]] if t.dim() == 4 else t[sum(lens[:b]):sum(lens[:b + 1])].transpose(0, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32", "mxfp4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", ["packed", "fused", "heads", "padded"])
@pytest.mark.parametrize("with_scores", [False, True])
def test_prompts_into_caches_and_back(dtype, D, layout, with_scores):
    a = arena(dtype, D)
    g = torch.Generator().manual_seed(D)
    H, batch = 2, 3
    want = {}
    live = np.zeros((2, batch), dtype=int)
    for call, (layer, lens) in enumerate([(0, [5, 0, 130]), (1, [1, 64, 65]), (0, [63, 129, 0]), (1, [0, 3, 70])]):
        k, v = (rows(dtype, layout, lens, H, D, g) for _ in range(2))
        sc = None
        if with_scores:
            sc = torch.rand((batch, H, max(lens)) if layout == "padded" else (H, sum(lens)), generator=g).cuda()
        pos0 = [10 * call + b for b in range(batch)] if call != 1 else None
        a.append_prompt(layer, k, v, lens, pos0, scores=sc)
        for b in range(batch):
            for h in range(H):
                w = want.setdefault((layer, b, h), ([], [], [], []))
                for i, t in enumerate((k, v)):
                    w[i].append(stored(of_sequence(t, b, lens)[h], dtype))
                s = np.zeros(lens[b]) if sc is None else (sc[b, h, :lens[b]] if layout == "padded" else sc[h, sum(lens[:b]):sum(lens[:b + 1])]).cpu().numpy()
                w[2].append(s)
                w[3].append(np.arange(lens[b]) + (pos0[b] if pos0 else 0))
            live[layer, b] += lens[b]
    torch.cuda.synchronize()
    assert np.array_equal(a.lengths(), np.repeat(live.reshape(-1), H)) and np.array_equal(a.len.cpu().numpy(), a.lengths())
    kr, vr = a.read_rows(0, 2, 205)
    one = a.read_rows(1, 1, 4)
    sc, ps = a.score.cpu().numpy(), a.pos.cpu().numpy()
    for (layer, b, h), w in want.items():
        c = (layer * batch + b) * H + h
        n, o = live[layer, b], int(a.off_host[c])
        for t, parts, last in ((kr, w[0], one[0]), (vr, w[1], one[1])):
            x = np.concatenate(parts)
            assert np.array_equal(t[c, 205 - n:].double().cpu().numpy(), x) and not t[c, :205 - n].any()
            if layer == 1:
                y = np.vstack([np.zeros((4, D)), x])[-4:]
                assert np.array_equal(last[c - batch * H].double().cpu().numpy(), y)
        assert np.array_equal(sc[o:o + n], np.concatenate(w[2]).astype(np.float32)) and np.array_equal(ps[o:o + n], np.concatenate(w[3]))
        assert (sc[o + n:o + 200] == -5).all() and (ps[o + n:o + 200] == -7).all()   # rows behind stay as they were
        if dtype != "mxfp4":
            assert (a.k[o + n:o + 200] == 3).all() and (a.v[o + n:o + 200] == 3).all()


@pytest.mark.parametrize("batch,Hkv", [(130, 1), (150, 4), (3, 600), (1, 1)])
def test_more_sequences_and_heads_than_a_launch_holds(batch, Hkv):
    a = arena("bf16", 64, 1, batch, Hkv, cap=9)
    rng = np.random.default_rng(batch)
    lens = [int(x) for x in rng.integers(0, 6, batch)]
    lens[-1] = 4
    k = torch.randn((sum(lens), Hkv, 64)).bfloat16().cuda()
    v = torch.randn((sum(lens), Hkv, 64)).bfloat16().cuda()
    a.append_prompt(0, k, v, lens, list(range(batch)))
    kr, vr = a.read_rows(0, 1, 6)
    kr, vr = kr.view(batch, Hkv, 6, 64), vr.view(batch, Hkv, 6, 64)
    for b in range(batch):
        at = sum(lens[:b])
        assert torch.equal(kr[b, :, 6 - lens[b]:], k[at:at + lens[b]].transpose(0, 1))
        assert torch.equal(vr[b, :, 6 - lens[b]:], v[at:at + lens[b]].transpose(0, 1)) and not kr[b, :, :6 - lens[b]].any()
    assert np.array_equal(a.lengths(), np.repeat(lens, Hkv)) and np.array_equal(a.len.cpu().numpy(), a.lengths())


def test_refusals_leave_the_caches_as_they_are():
    a = arena("bf16", 64, 1, 2, 2, cap=10)
    k = torch.randn((12, 2, 64)).bfloat16().cuda()
    with pytest.raises(B.BaklavaError) as e:
        a.append_prompt(0, k, k, [1, 11])
    assert e.value.status == B.ECAPACITY and not a.lengths().any()
    a.append_prompt(0, k, k, [1, 9])
    for lens in ([10, 0], [0, 2]):
        with pytest.raises(B.BaklavaError) as e:
            a.append_prompt(0, k, k, lens)
        assert e.value.status == B.ECAPACITY
    for kw in (dict(lens=[1]), dict(lens=[1, 12]), dict(pos0=[1]), dict(scores=torch.zeros((2, 1)).cuda()), dict(k=k.cpu()), dict(k=k.float()),
               dict(k=k[:, :1])):
        with pytest.raises(ValueError):
            a.append_prompt(0, **{**dict(k=k, v=k, lens=[1, 1]), **kw})
    for layer, lens, pos0 in ((1, [1, 0], None), (-1, [1, 0], None), (0, [1, -1], None), (0, [2, 0], [2 ** 31 - 1, 0])):
        with pytest.raises((B.BaklavaError, ValueError)):
            a.append_prompt(layer, k, k, lens, pos0)
    a.append_prompt(0, k, k, [0, 0])                      # nothing to append
    with pytest.raises(B.BaklavaError):
        a.read_rows(0, 2, 1)
    with pytest.raises(ValueError):
        a.read_rows(0, 1, 0)
    torch.cuda.synchronize()
    assert a.lengths().tolist() == [1, 1, 9, 9] and a.len.cpu().tolist() == [1, 1, 9, 9]


def test_captured_prompt_replays_the_rows_of_its_capture():
    a = arena("mxfp4", 128, 1, 2, 2, cap=40)
    k = torch.randn((30, 2, 128)).bfloat16().cuda()
    v = torch.randn((30, 2, 128)).bfloat16().cuda()
    ko, vo = None, None
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        a.reset()
        a.append_prompt(0, k, v, [10, 20])
        ko, vo = a.read_rows(0, 1, 20)
    for _ in range(3):
        k.normal_(), v.normal_()
        g.replay()
        torch.cuda.synchronize()
        for t, x in ((ko, k), (vo, v)):
            want = stored(x[10:].transpose(0, 1), "mxfp4")
            assert np.array_equal(t[2:].double().cpu().numpy(), want)
        assert a.len.cpu().tolist() == [10, 10, 20, 20]
    assert a.lengths().tolist() == [10, 10, 20, 20]


@pytest.mark.parametrize("dtype", ["bf16", "mxfp4"])
def test_a_prompt_and_the_steps_behind_it(dtype):
    """A model's layer as it would use the library: norm and rotation, attention over the packed prompts, their scores, rows into the
    caches, eviction, and decode steps whose rows are normed and rotated too.  Every step against fp64 from what the device holds."""
    L, batch, Hq, Hkv, D, T = 1, 2, 8, 2, 128, 300
    G = Hq // Hkv
    lens = [300, 170]
    budget = [60, 200]
    a = B.Arena(L, Hq, Hkv, D, batch, dtype, budget, T - min(budget) + 8, 4, 16, B.POLICY_SCORE, True)
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((sum(lens), Hq + 2 * Hkv, D), generator=g).bfloat16().cuda()
    wq, wk = ((1 + 0.1 * torch.randn((D,), generator=g)).bfloat16().cuda() for _ in range(2))
    pos = torch.cat([torch.arange(n) for n in lens]).to(torch.int32).cuda()
    f = 10000.0 ** (-np.arange(D // 2) / (D // 2))
    q, k = B.qk_norm_rope(qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], pos, f, q_weight=wq, k_weight=wk)
    v = qkv[:, Hq + Hkv:]
    out, lse = B.prompt_attn(q, k, v, lens, want_lse=True)
    scores = torch.zeros((Hkv, sum(lens)), device="cuda")
    for b, n in enumerate(lens):
        at = slice(sum(lens[:b]), sum(lens[:b]) + n)
        one = torch.empty((Hkv * n,), device="cuda")
        B.prefill_scores(q[at].transpose(0, 1).contiguous(), k[at].transpose(0, 1).contiguous(), lse[:, at].contiguous(), one, 1, Hq, Hkv, n)
        scores[:, at] = one.view(Hkv, n)
    a.append_prompt(0, k, v, lens, scores=scores)
    kept = torch.full((a.total_tokens,), -1, dtype=torch.int32, device="cuda")
    a.compact(0, 1, kept)
    torch.cuda.synchronize()
    q64, k64, v64 = (t.double().cpu().numpy() for t in (q, k, v))
    caches = []
    for c in range(batch * Hkv):
        b, h = divmod(c, Hkv)
        at = slice(sum(lens[:b]), sum(lens[:b]) + lens[b])
        for i in (0, G - 1):
            want, _, mass, big = OP.prompt_attention(q64[at, h * G + i], k64[at, h], v64[at, h])
            tol = (2.0 ** -8 + 2.0 ** -16 * big + 2.0 ** -20)[:, None] * mass + 2.0 ** -8 * 1.02 * np.abs(want)
            assert (np.abs(out[at, h * G + i].double().cpu().numpy() - want) <= tol).all()
        want = O.prefill_scores(np.stack([q64[at, h * G + i] for i in range(G)]), k64[at, h])
        got = scores[h, at].cpu().numpy()
        assert (np.abs(got - want) <= 2e-5 * np.maximum(1, want)).all()
        idx = np.asarray(O.compact_select(got, lens[b], budget[h], 4, 16))
        o = int(a.off_host[c])
        assert np.array_equal(kept[o:o + len(idx)].cpu().numpy(), idx)
        caches.append([stored(k[at, h], dtype)[idx], stored(v[at, h], dtype)[idx], got[idx].astype(np.float64)])
    for t in range(4):
        x = torch.randn((batch, Hq + 2 * Hkv, D), generator=g).bfloat16().cuda()
        at = torch.tensor([lens[0] + t, lens[1] + t], dtype=torch.int32).cuda()
        qn, kn = B.qk_norm_rope(x[:, :Hq], x[:, Hq:Hq + Hkv], at, f, q_weight=wq, k_weight=wk)
        vn = x[:, Hq + Hkv:].contiguous()
        o = torch.empty((1, batch, Hq, D), device="cuda")
        a.append_decode_attn(0, 1, kn, vn, lens[0] + t, qn, o)
        torch.cuda.synchronize()
        for c, (K, V, S) in enumerate(caches):
            b, h = divmod(c, Hkv)
            K, V, S = np.vstack([K, stored(kn[b, h], dtype)]), np.vstack([V, stored(vn[b, h], dtype)]), np.append(S, 0.0)
            for i in range(G):
                row = qn[b, h * G + i].double().cpu().numpy()
                want, p = O.decode_attn(row[None], K, V)
                assert np.abs(o[0, b, h * G + i].double().cpu().numpy() - want).max() <= 2e-3
                S = S + np.asarray(p).reshape(-1)
            caches[c] = [K, V, S]
    a.flush_scores(0, 1)
    kr, vr = a.read_rows(0, 1, int(a.lengths().max()))
    for c, (K, V, S) in enumerate(caches):
        n, o = len(K), int(a.off_host[c])
        assert np.array_equal(kr[c, -n:].double().cpu().numpy(), K) and np.array_equal(vr[c, -n:].double().cpu().numpy(), V)
        assert (np.abs(a.score[o:o + n].cpu().numpy() - S) <= 2e-3).all()
