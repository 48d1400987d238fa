"""GPU: baklava_qk_norm_rope over batches of sequences, as right and as fast as over the same tokens packed."""
import numpy as np
import pytest
import torch

from paper_2502_13176_amd import binding as B
from test_gpu_rope import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,kw", [(1366, dict()), (2053, dict(interleaved=True)), (1500, dict(rot=22)), (1367, dict(in_place=True))])
def test_several_tokens_of_a_workgroup_in_a_batch(dtype, n, kw):
    """Three sequences of fewer than 4096 tokens that have more together."""
    run(dtype, n, 2, 1, 64, axes=2, layout="batch", **kw)


def test_sequences_shorter_than_a_workgroup_takes_tokens():
    x = torch.randn((700, 2, 7, 64)).bfloat16().cuda()
    pos = torch.randint(0, 9000, (700 * 7,), dtype=torch.int32).cuda()
    f = 10000.0 ** (-np.arange(32) / 32)
    got = B.qk_norm_rope(x, None, pos, f)[0]
    for i in (0, 1, 350, 699):
        assert torch.equal(got[i:i + 1], B.qk_norm_rope(x[i:i + 1], None, pos[7 * i:7 * i + 7], f)[0])


def us(call):
    call()
    torch.cuda.synchronize()
    best = float("inf")
    for _ in range(5):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        for _ in range(10):
            call()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b) * 100)
    return best


def test_a_batch_takes_no_token_alone():
    """64 sequences of 2048 tokens, two heads: 10 times the packed call's time with a token for each workgroup, 1.0 with several."""
    x = torch.randn((64, 2, 2048, 64)).bfloat16().cuda()
    out, pos, f = torch.empty_like(x), torch.arange(64 * 2048, dtype=torch.int32).cuda(), 10000.0 ** (-np.arange(32) / 32)
    rows, rows_out = (t.view(64 * 2048, 2, 64) for t in (x, out))
    batch = us(lambda: B.qk_norm_rope(x, None, pos, f, q_out=out))
    packed = us(lambda: B.qk_norm_rope(rows, None, pos, f, q_out=rows_out))
    assert batch < 4 * packed, (batch, packed)


def test_more_tokens_than_a_launch_has_workgroups():
    """Rows so wide that every token takes a workgroup: 2^24 + 3 tokens of 25 fp32 heads, 107 GB written, from one row read again and again."""
    torch.cuda.empty_cache()
    n, H, D = (1 << 24) + 3, 25, 64
    one = torch.randn((1, H, D)).cuda()
    out = torch.full((n, H, D), float("nan"), device="cuda")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    f, w = 10000.0 ** (-np.arange(32) / 32), torch.ones(D, device="cuda")
    B.qk_norm_rope(one.expand(n, H, D), None, pos, f, q_weight=w, q_out=out)
    at = torch.tensor([0, 1, 255, (1 << 23) + 1, (1 << 24) - 2, (1 << 24) - 1, 1 << 24, n - 1]).cuda()
    want = B.qk_norm_rope(one.expand(len(at), H, D), None, pos[at].contiguous(), f, q_weight=w)[0]
    assert torch.equal(out[at], want)
    for i in range(0, n, 1 << 20):                        # every row is written
        assert not torch.isnan(out[i:i + (1 << 20), :, 0]).any()
    del out
    torch.cuda.empty_cache()


def test_more_sequences_than_a_launch_holds():
    x = torch.randn((65535 + 9, 1, 2, 64)).bfloat16().cuda()
    pos = torch.randint(0, 9000, (x.shape[0] * 2,), dtype=torch.int32).cuda()
    f = 10000.0 ** (-np.arange(32) / 32)
    got = B.qk_norm_rope(x, None, pos, f)[0]
    rows = B.qk_norm_rope(x.view(-1, 1, 64), None, pos, f)[0]
    assert torch.equal(got.view(-1, 1, 64), rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,Hq,Hkv", [(128, 6, 2), (128, 1, 1), (64, 7, 1)])
@pytest.mark.parametrize("kw", [dict(axes=3), dict(interleaved=True), dict(rot=24), dict(rot=22), dict(rot=24, interleaved=True), dict(layout="heads"),
                                dict(in_place=True), dict(in_place=True, rot=22), dict(in_place=True, layout="heads", interleaved=True)])
def test_several_tokens_of_a_workgroup(dtype, D, Hq, Hkv, kw):
    """4103 tokens: the last workgroup has fewer than the others (of 3 to 16, by the size of a token's rows)."""
    run(dtype, 4103, Hq, Hkv, D, far=100000, **kw)
