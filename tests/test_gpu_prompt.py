"""GPU parity: baklava_prompt_attn against fp64."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as OP
from paper_2502_13176_amd import binding as B

pytestmark = pytest.mark.gpu


def inputs(lens, kv, Hq, Hkv, D, layout, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)

    def rows(n, h, s=1.0):
        if layout == "packed":
            return (torch.randn((sum(n), h, D), generator=g) * s).bfloat16().cuda()
        if layout == "heads":                             # [H, tokens, D], handed over as [tokens, H, D]
            return (torch.randn((h, sum(n), D), generator=g) * s).bfloat16().cuda().transpose(0, 1)
        if layout == "fused":                             # keys and values of a wider buffer
            return (torch.randn((sum(n), h + 3, D), generator=g) * s).bfloat16().cuda()[:, 2:2 + h]
        if layout == "padded":
            return (torch.randn((len(n), h, max(n) + 3, D), generator=g) * s).bfloat16().cuda()
        return (torch.randn((len(n), max(n) + 1, h, D), generator=g) * s).bfloat16().cuda().transpose(1, 2)  # "padded tokens"
    return rows(lens, Hq, scale), rows(kv, Hkv), rows(kv, Hkv)


def of_sequence(t, b, lens):
    if t.dim() == 4:
        return t[b, :, :lens[b]]
    return t[sum(lens[:b]):sum(lens[:b + 1])].transpose(0, 1)


def check(q, k, v, out, lse, lens, kv, heads=None, tokens=None):
    """Weights enter the second product rounded to bf16, half a step of each at most: 2^-8 sum p |v|; the result is rounded once
    more, 2^-8 |o|.  fp32 logits: D products of fp32 sums, D 2^-24 of sum |q k| / sqrt(D) (times the logarithm's base in log2
    units), in every weight and once more in their sum; exponentials and the rest below 2^-20.  A weight below 2^-126 is no
    fp32 number and counts as zero: fewer than 2^14 rows of values below 2^4 make 2^-108 of them at most."""
    Hq, Hkv, D = q.shape[1], k.shape[1], q.shape[-1]
    G = Hq // Hkv
    worst = 0.0
    for b in range(len(lens)):
        if not lens[b]:
            continue
        qs, os = (of_sequence(t, b, lens).double().cpu().numpy() for t in (q, out))
        ks, vs = (of_sequence(t, b, kv).double().cpu().numpy() for t in (k, v))
        ls = (lse[b, :, :lens[b]] if lse.dim() == 3 else lse[:, sum(lens[:b]):sum(lens[:b + 1])]).double().cpu().numpy()
        for h in range(Hq) if heads is None else heads:
            at = np.arange(lens[b]) if tokens is None else np.unique(np.clip(tokens, 0, lens[b] - 1))
            if tokens is None:
                want, want_lse, mass, big = OP.prompt_attention(qs[h], ks[h // G], vs[h // G])
            else:
                parts = [OP.prompt_attention(qs[h, t:t + 1], ks[h // G, :max(0, kv[b] - lens[b] + t + 1)],
                                             vs[h // G, :max(0, kv[b] - lens[b] + t + 1)]) for t in at]
                want, want_lse, mass, big = (np.concatenate([x[i] for x in parts]) for i in range(4))
            logit = D * 2.0 ** -24 * big
            tol = (2.0 ** -8 + 2 * logit + 2.0 ** -20)[:, None] * mass + 2.0 ** -8 * (1 + 2.0 ** -6) * np.abs(want) + 2.0 ** -108
            err = np.abs(os[h, at] - want)
            assert (err <= tol).all(), (b, h, float((err - tol).max()))
            seen = np.isfinite(want_lse)
            assert np.array_equal(np.isneginf(ls[h, at]), ~seen)
            tol = 1.5 * logit[seen] + 2.0 ** -20 * (1 + np.abs(want_lse[seen]))
            assert (np.abs(ls[h, at][seen] - want_lse[seen]) <= tol).all()
            worst = max(worst, float(err.max()))
    return worst


def run(lens, kv=None, Hq=4, Hkv=2, D=128, layout="packed", seed=1, scale=1.0, **kw):
    kvl = lens if kv is None else kv
    q, k, v = inputs(lens, kvl, Hq, Hkv, D, layout, seed, scale)
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=q.device)
    lse = torch.full((len(lens), Hq, q.shape[2]) if q.dim() == 4 else (Hq, q.shape[0]), 7.0, device=q.device)
    B.prompt_attn(q, k, v, lens, kv_lens=kv, out=out, lse=lse)
    torch.cuda.synchronize()
    check(q, k, v, out, lse, lens, kvl, **kw)
    if q.dim() == 4:                                      # places past a sequence's length stay as they were
        for b, n in enumerate(lens):
            assert (out[b, :, n:] == 7).all() and (lse[b, :, n:] == 7).all()
    return q, k, v, out, lse


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 191, 200, 257, 320])
def test_one_sequence(n, D):
    run([n], D=D, seed=n)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", ["packed", "heads", "fused", "padded", "padded tokens"])
def test_several_sequences_and_layouts(layout, D):
    run([5, 130, 0, 1, 77], D=D, layout=layout, Hq=6, Hkv=2)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (7, 1), (8, 8), (14, 2), (16, 1), (20, 1), (9, 3)])
def test_head_counts(Hq, Hkv):
    run([70, 140], Hq=Hq, Hkv=Hkv, seed=Hq)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,kv", [([1], [300]), ([1], [64]), ([64], [128]), ([128], [256]), ([129], [1000]), ([5, 200, 1], [5, 263, 640]),
                                     ([40], [17]), ([200], [1]), ([150, 3], [60, 0]), ([3], [0])])
def test_prefixes_and_tokens_that_see_nothing(lens, kv, D):
    run(lens, kv, D=D, seed=lens[0])


@pytest.mark.parametrize("seqs", [64, 65, 128, 129, 300])
def test_many_sequences(seqs):
    rng = np.random.default_rng(seqs)
    run([int(x) for x in rng.integers(0, 9, seqs)], Hq=2, Hkv=1, D=64)


@pytest.mark.parametrize("scale", [30.0, 1000.0])
def test_steep_logits(scale):
    run([150, 90], scale=scale)


# Above, a call has at most one workgroup of 128 tokens for each of 256 compute units; these have one to two, and more.
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens,kv", [([257, 1, 130], None), ([300, 129, 64, 1, 500, 33], None), ([200, 640], [263, 641]), ([130, 300, 260], [60, 299, 1000]),
                                     ([1100], None)])
def test_more_workgroups_than_compute_units(lens, kv, D):
    run(lens, kv, Hq=60, Hkv=4, D=D, heads=[0, 14, 15, 59], layout="heads", seed=len(lens))


@pytest.mark.parametrize("D", [64, 128])
def test_more_workgroups_with_steep_logits_and_values_that_are_not_finite(D):
    lens = [300, 200]
    run(lens, Hq=64, Hkv=2, D=D, scale=40.0, heads=[5, 60])
    q, k, v = inputs(lens, lens, 64, 2, D, "packed", 8)
    want, want_lse = B.prompt_attn(q, k, v, lens, want_lse=True)
    v2 = v.clone()
    v2[250] = float("inf")
    v2[499] = float("nan")
    out, lse = B.prompt_attn(q, k, v2, lens, want_lse=True)
    clean = [t for t in range(500) if not 250 <= t < 300 and t != 499]
    assert torch.equal(out[clean], want[clean]) and torch.equal(lse, want_lse)
    assert torch.isinf(out[250:300]).all() and torch.isnan(out[499]).all()


def test_more_workgroups_of_many_padded_sequences():
    rng = np.random.default_rng(5)
    lens = [int(x) for x in rng.integers(0, 200, 150)]
    run(lens, [max(0, n + int(rng.integers(-5, 90))) for n in lens], Hq=4, Hkv=2, D=64, layout="padded", heads=[1, 2])


def test_tokens_far_apart():
    """Offsets of more than 2^31 elements, of tokens that are 2^20 elements apart."""
    n, w = 2100, 1 << 20
    far = torch.empty((n, w), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn((n, h, 64), generator=g).bfloat16().cuda() for h in (4, 2, 2))
    at = {}
    for name, x, i in (("q", q, 0), ("k", k, 4), ("v", v, 6), ("out", torch.zeros_like(q), 8), ("q_out", torch.zeros_like(q), 12)):
        at[name] = far[:, 64 * i:64 * (i + x.shape[1])].unflatten(1, (-1, 64))
        at[name].copy_(x)
    want, want_lse = B.prompt_attn(q, k, v, [n - 50, 50], want_lse=True)
    _, lse = B.prompt_attn(at["q"], at["k"], at["v"], [n - 50, 50], out=at["out"], want_lse=True)
    assert torch.equal(at["out"], want) and torch.equal(lse, want_lse)
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    f = [0.5 ** i for i in range(32)]
    B.qk_norm_rope(at["q"], None, pos, f, q_out=at["q_out"])
    assert torch.equal(at["q_out"], B.qk_norm_rope(q, None, pos, f)[0])
    for dtype in ("bf16", "mxfp4"):
        rows = []
        for x, y in ((k, v), (at["k"], at["v"])):
            a = B.Arena(1, 4, 2, 64, 2, dtype, [n] * 2, 0, 0, 0)
            a.append_prompt(0, x, y, [n - 50, 50])
            rows.append(a.read_rows(0, 1, n))
        assert torch.equal(rows[0][0], rows[1][0]) and torch.equal(rows[0][1], rows[1][1])


def test_rows_behind_the_last_sequence_and_shared_heads():
    """Tensors that hold more tokens than the lengths name, and keys of one head handed over as several."""
    lens = [50, 100]
    q, k, v = inputs([50, 100, 30], [50, 100, 30], 4, 1, 64, "packed", 12)
    k4, v4 = (t.expand(-1, 4, -1) for t in (k, v))
    out, lse = torch.full_like(q, 3.0), torch.full((4, 180), 3.0, device="cuda")
    B.prompt_attn(q, k4, v4, lens, out=out, lse=lse)
    assert (out[150:] == 3).all() and (lse[:, 150:] == 3).all()
    want, want_lse = B.prompt_attn(q[:150], k[:150], v[:150], lens, want_lse=True)
    assert torch.equal(out[:150], want) and torch.equal(lse[:, :150], want_lse)


@pytest.mark.parametrize("Hq", [2, 24])
def test_a_long_prompt_at_some_tokens(Hq):
    run([6000, 2049], Hq=Hq, Hkv=1, heads=[1], tokens=[0, 1, 63, 64, 127, 128, 2047, 2048, 4095, 5990, 5999])


def test_equal_rows_give_their_mean():
    k = torch.ones((100, 1, 64)).bfloat16().cuda()
    v = torch.arange(100).view(100, 1, 1).expand(100, 1, 64).bfloat16().cuda().contiguous()
    out, lse = B.prompt_attn(torch.zeros((100, 1, 64)).bfloat16().cuda(), k, v, [100], want_lse=True)
    want = torch.arange(100).double().cumsum(0) / torch.arange(1, 101)
    assert (out[:, 0].double().cpu() - want[:, None]).abs().le(want[:, None] * 2.0 ** -7).all()
    assert (lse[0].double().cpu() - torch.log2(torch.arange(1, 101).double())).abs().max() <= 1e-5


def test_values_behind_the_mask_do_not_matter():
    """Infinite and NaN keys and values of later tokens, of other sequences and of padded places."""
    lens = [70, 133]
    q, k, v, out, lse = run(lens, layout="padded")
    k2, v2 = k.clone(), v.clone()
    for t, bad in ((k2, float("nan")), (v2, float("inf"))):
        for b, n in enumerate(lens):
            t[b, :, n:] = bad
            t[b, :, n - 3:n] = bad
    out2, lse2 = B.prompt_attn(q, k2, v2, lens, want_lse=True)
    for b, n in enumerate(lens):
        assert torch.equal(out2[b, :, :n - 3], out[b, :, :n - 3]) and torch.equal(lse2[b, :, :n - 3], lse[b, :, :n - 3])
        assert torch.isnan(out2[b, :, n - 3:n]).all()     # they see the NaN keys
    k3, v3 = k.clone(), v.clone()
    for b, n in enumerate(lens):
        k3[b, :, n:] = float("nan")
        v3[b, :, n:] = float("nan")
    out3, lse3 = B.prompt_attn(q, k3, v3, lens, want_lse=True)
    for b, n in enumerate(lens):
        assert torch.equal(out3[b, :, :n], out[b, :, :n]) and torch.equal(lse3[b, :, :n], lse[b, :, :n])


@pytest.mark.parametrize("D", [64, 128])
def test_infinite_values_reach_the_tokens_that_see_them(D):
    n = 150
    q, k, v = inputs([n], [n], 2, 1, D, "packed", 8)
    v[100, 0, 5] = float("inf")
    v[101, 0, 7] = float("-inf")
    v[120, 0, 5] = float("-inf")
    v[130] = float("nan")
    out = B.prompt_attn(q, k, v, [n]).float().cpu()
    clean = v.clone()
    clean[100:, 0, 5], clean[101:, 0, 7], clean[130:] = 0, 0, 0
    ref = B.prompt_attn(q, k, clean, [n]).float().cpu()
    assert torch.equal(out[:100], ref[:100]) and torch.isinf(out[100:120, :, 5]).all() and (out[100:120, :, 5] > 0).all()
    assert torch.isnan(out[120:, :, 5]).all() and (out[101:130, :, 7] == float("-inf")).all()
    assert torch.isnan(out[130:]).all()
    other = [d for d in range(D) if d not in (5, 7)]
    assert torch.allclose(out[100:130][..., other], ref[100:130][..., other], rtol=2 ** -7, atol=2 ** -7)


def test_lse_feeds_the_prompt_scores():
    n, Hq, Hkv = 700, 8, 2
    q, k, v = inputs([n], [n], Hq, Hkv, 128, "padded", 3)
    q, k, v = (t[:, :, :n].contiguous() for t in (q, k, v))
    _, _, want = B.profile_similarity(q, k, v, want_lse=True)
    _, lse = B.prompt_attn(q, k, v, [n], want_lse=True)
    score = torch.empty((Hkv * n,), device="cuda")
    B.prefill_scores(q, k, lse, score, 1, Hq, Hkv, n)
    assert (lse - want).abs().max() <= 2e-4
    assert abs(float(score.sum()) - n * Hq) <= 1e-4 * n * Hq


def test_captured_replays_and_another_stream():
    lens = [90, 40]
    q, k, v = inputs(lens, lens, 4, 2, 128, "packed", 5)
    out, lse = torch.empty_like(q), torch.empty((4, 130), device="cuda")
    g = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        B.prompt_attn(q, k, v, lens, out=out, lse=lse)
    for _ in range(3):
        for t in (q, k, v):
            t.normal_()
        g.replay()
        torch.cuda.synchronize()
        want, want_lse = B.prompt_attn(q, k, v, lens, want_lse=True)
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    with torch.cuda.stream(s):
        other = B.prompt_attn(q, k, v, lens)
    s.synchronize()
    assert torch.equal(other, out)


def test_refusals_of_the_binding():
    q, k, v = inputs([9], [9], 4, 2, 64, "packed", 6)
    for bad in (dict(lens=[10]), dict(lens=[]), dict(lens=[-1]), dict(kv_lens=[10]), dict(kv_lens=[1, 2]), dict(out=q.float()),
                dict(lse=torch.empty((2, 9)).cuda()), dict(lse=torch.empty((4, 9)).cuda().half())):
        with pytest.raises(ValueError):
            B.prompt_attn(q, k, v, **{**dict(lens=[9]), **bad})
    for args in ((q.cpu(), k, v), (q.float(), k, v), (q, k, v[:, :1]), (q[..., :32], k, v), (q.transpose(1, 2), k, v)):
        with pytest.raises(ValueError):
            B.prompt_attn(*args, [9])
    with pytest.raises(B.BaklavaError):                   # three query heads over two caches
        B.prompt_attn(q[:, :3], k, v, [9])
    assert B.prompt_attn(q[:0], k[:0], v[:0], [0]).shape == (0, 4, 64)
