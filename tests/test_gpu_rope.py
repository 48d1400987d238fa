"""GPU parity: baklava_qk_norm_rope against fp64."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as OP
from paper_2502_13176_amd import binding as B

pytestmark = pytest.mark.gpu

# bf16: half a step of the result, 2^-8 |y|.  fp32 arithmetic in front of it, relative to the size R of the pair: 18 additions of
# squares (halved by the root), root, quotient, two products of the norm, angle and its sine and cosine (2 ulp each), three
# roundings of the turn: below 32 half steps, 2^-19 R.  fp32 results: that alone.
FP32 = 2.0 ** -19


def run(dtype="bf16", n=5, Hq=4, Hkv=2, D=128, rot=None, axes=1, interleaved=False, norm=(True, True), layout="fused", base=10000.0,
        far=1000, seed=1, in_place=False, axis=None):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rot = D if rot is None else rot
    g = torch.Generator().manual_seed(seed)
    if layout == "fused":                                 # [tokens, Hq + 2 Hkv, D]
        buf = torch.randn((n, Hq + 2 * Hkv, D), generator=g).to(dt).cuda()
        q, k = buf[:, :Hq], buf[:, Hq:Hq + Hkv]
    elif layout == "heads":                               # [H, tokens, D]
        q, k = (torch.randn((h, n, D), generator=g).to(dt).cuda().transpose(0, 1) for h in (Hq, Hkv))
    else:                                                 # [3, H, tokens, D]
        q, k = (torch.randn((3, h, n, D), generator=g).to(dt).cuda() for h in (Hq, Hkv))
    seqs = 3 if layout == "batch" else 1
    pos = torch.randint(0, far, (axes, seqs * n), generator=g).to(torch.int32)
    w = [(torch.randn((D,), generator=g).to(dt).cuda() if x else None) for x in norm]
    f = base ** (-np.arange(rot // 2) / max(1, rot // 2))
    axis = [i % axes for i in range(rot // 2)] if axis is None else axis
    if in_place:
        want_in = (q.double().cpu().numpy(), k.double().cpu().numpy())
    got = B.qk_norm_rope(q, k, pos.cuda(), f, q_weight=w[0], k_weight=w[1], eps=1e-5, axis_of_pair=axis, interleaved=interleaved,
                         q_out=q if in_place else None, k_out=k if in_place else None)
    torch.cuda.synchronize()
    src = want_in if in_place else (q.double().cpu().numpy(), k.double().cpu().numpy())
    for i, (x, y, wt) in enumerate(zip(src, got, w)):
        y = y.double().cpu().numpy()
        if layout == "batch":                             # -> [batch * tokens, H, D]
            x, y = (a.transpose(0, 2, 1, 3).reshape(-1, a.shape[1], D) for a in (x, y))
        want, size = OP.norm_rope(x, wt.double().cpu().numpy() if wt is not None else None, 1e-5, pos.numpy(), f, axis, interleaved)
        tol = FP32 * size + (2.0 ** -8 * np.abs(want) if dtype == "bf16" else 0.0)
        assert (np.abs(y - want) <= tol).all(), (i, float((np.abs(y - want) - tol).max()))
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", ["fused", "heads", "batch"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_types_sizes_and_layouts(dtype, D, layout, interleaved):
    run(dtype, 7, 6, 2, D, layout=layout, interleaved=interleaved, axes=3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot", [0, 2, 16, 22, 24, 48, 64, 126])
@pytest.mark.parametrize("interleaved", [False, True])
def test_part_of_a_row_rotated(dtype, rot, interleaved):
    run(dtype, 3, 4, 1, 128, rot=rot, interleaved=interleaved, seed=rot)


@pytest.mark.parametrize("n,Hq,Hkv", [(1, 1, 1), (1, 32, 8), (8, 28, 4), (129, 7, 7), (4095, 3, 1), (4099, 5, 1)])
def test_token_and_head_counts(n, Hq, Hkv):
    run("bf16", n, Hq, Hkv, 64, seed=n)


@pytest.mark.parametrize("Hq,Hkv", [(0, 3), (40, 1), (130, 2)])
def test_many_heads_and_none(Hq, Hkv):
    """More heads than a workgroup takes rows at a time; keys alone."""
    x = torch.randn((6, Hq + Hkv, 128)).bfloat16().cuda()
    pos = torch.arange(6, dtype=torch.int32).cuda()
    f = 10000.0 ** (-np.arange(64) / 64)
    q, k = B.qk_norm_rope(x[:, :Hq] if Hq else None, x[:, Hq:], pos, f)
    every = B.qk_norm_rope(x, None, pos, f)[0]
    assert torch.equal(k, every[:, Hq:]) and (q is None or torch.equal(q, every[:, :Hq]))
    want, _ = OP.norm_rope(x.double().cpu().numpy(), None, 0.0, pos.cpu().numpy()[None], f, [0] * 64, False)
    assert (np.abs(every.double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + FP32 * 8).all()


@pytest.mark.parametrize("far", [131072, 1 << 24, (1 << 31) - 1])
def test_far_positions(far):
    run("f32", 64, 2, 1, 128, far=far, base=500000.0)


@pytest.mark.parametrize("norm", [(False, False), (True, False), (False, True)])
def test_without_norms(norm):
    run("f32", 5, 3, 1, 64, norm=norm)


@pytest.mark.parametrize("kw", [dict(), dict(rot=24), dict(interleaved=True), dict(layout="heads"), dict(layout="batch")])
def test_in_place(kw):
    run("bf16", 9, 4, 2, 128, in_place=True, **kw)


def test_one_of_the_two_and_rows_around_them():
    """Only queries; the rows of the buffer that are not asked for stay as they are."""
    buf = torch.randn((6, 8, 128)).bfloat16().cuda()
    keep = buf.clone()
    pos = torch.arange(6, dtype=torch.int32).cuda()
    f = np.ones(64)
    q, k = B.qk_norm_rope(buf[:, 2:5], None, pos, f, q_out=buf[:, 2:5])
    torch.cuda.synchronize()
    assert k is None and torch.equal(buf[:, :2], keep[:, :2]) and torch.equal(buf[:, 5:], keep[:, 5:])
    only = B.qk_norm_rope(None, keep[:, 2:5], pos, f)[1]
    torch.cuda.synchronize()
    assert torch.equal(only, buf[:, 2:5])


def test_rows_that_are_not_finite_and_zero_rows():
    q = torch.zeros((4, 1, 64))
    q[1, 0, 3] = float("inf")
    q[2, 0, 5] = float("nan")
    q[3] = 1.0
    out, _ = B.qk_norm_rope(q.cuda(), None, torch.zeros(4, dtype=torch.int32).cuda(), np.ones(32), q_weight=torch.ones(64).cuda(), eps=1e-6)
    out = out.cpu()
    assert not out[0].any()                               # 0 / sqrt(eps)
    assert torch.isnan(out[1]).any() and torch.isnan(out[2]).all()
    assert torch.allclose(out[3], torch.full((1, 64), 1 / (1 + 1e-6) ** 0.5), atol=1e-6)


def test_sections_and_refusals_of_the_binding():
    q = torch.randn((5, 2, 64)).cuda()
    pos = torch.randint(0, 100, (3, 5), dtype=torch.int32).cuda()
    f = 100.0 ** (-np.arange(32) / 32)
    a = B.qk_norm_rope(q, None, pos, f, sections=[8, 12, 12])[0]
    b = B.qk_norm_rope(q, None, pos, f, axis_of_pair=[0] * 8 + [1] * 12 + [2] * 12)[0]
    assert torch.equal(a, b)
    for kw in (dict(sections=[8, 12]), dict(sections=[8, 8, 8, 8]), dict(axis_of_pair=[3] * 32), dict(axis_of_pair=[0]),
               dict(q_weight=torch.ones(32).cuda()), dict(q_weight=torch.ones(64)), dict(k_weight=torch.ones(64).cuda()),
               dict(q_out=torch.empty((5, 2, 32)).cuda())):
        with pytest.raises(ValueError):
            B.qk_norm_rope(q, None, pos, f, **kw)
    for x, p in ((q.cpu(), pos), (q, pos.cpu()), (q.double(), pos), (q, pos.long()), (q.transpose(1, 2), pos), (q, pos[:, :4])):
        with pytest.raises(ValueError):
            B.qk_norm_rope(x, None, p, f)
    assert B.qk_norm_rope(q[:0], None, pos, f)[0].shape == (0, 2, 64)


def test_captured_and_on_another_stream():
    n = 33
    q = torch.randn((n, 4, 128)).bfloat16().cuda()
    pos = torch.arange(n, dtype=torch.int32).cuda()
    out = torch.empty_like(q)
    f = 10000.0 ** (-np.arange(64) / 64)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        B.qk_norm_rope(q, None, pos, f, q_out=out)
    for i in range(3):
        q.normal_()
        pos += 1000
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, B.qk_norm_rope(q, None, pos, f)[0])
    with torch.cuda.stream(s):
        other = B.qk_norm_rope(q, None, pos, f)[0]
    s.synchronize()
    assert torch.equal(out, other) and torch.equal(B.qk_norm_rope(q, None, pos, f, stream=torch.cuda.current_stream())[0], out)
