"""Calls on another stream than torch's current one: their outputs come from that stream's part of the caching allocator, where no
kernel of the current stream can still be at work on them, and are right while the current stream is busy."""
import numpy as np
import pytest
import torch

from paper_2502_13176_amd import binding as B

pytestmark = pytest.mark.gpu


def stream_of(t):
    """The stream whose part of the caching allocator holds t."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not in the caching allocator")


def rows(n, H, D=128):
    return torch.randn((n, H, D)).bfloat16().cuda()


def rope(n):
    x, pos, f = rows(n, 4), torch.arange(n, dtype=torch.int32).cuda(), 10000.0 ** (-np.arange(64) / 64)
    return lambda s: B.qk_norm_rope(x[:, :3], x[:, 3:], pos, f, stream=s)


def attention(n):
    q, k, v = rows(n, 4), rows(n, 2), rows(n, 2)
    return lambda s: B.prompt_attn(q, k, v, [n - 7, 7], want_lse=True, stream=s)


def cache_rows(n):
    a = B.Arena(1, 4, 2, 128, 1, "mxfp4", [n, n], 0, 0, 0)
    a.append_prompt(0, rows(n, 2), rows(n, 2), [n])
    return lambda s: a.read_rows(0, 1, n, stream=s)


def similarity(n):
    q, k, v = (torch.randn((1, h, n, 128)).bfloat16().cuda() for h in (4, 2, 2))
    return lambda s: B.profile_similarity(q, k, v, want_lse=True, stream=s)


def layers(n):
    x, y = (torch.randn((2, n, 512)).bfloat16().cuda() for _ in range(2))
    return lambda s: B.layer_similarity(x, y, stream=s)


@pytest.mark.parametrize("make", [rope, attention, cache_rows, similarity, layers])
def test_outputs_belong_to_the_stream_that_writes_them(make):
    call = make(200)
    want = call(None)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    assert all(stream_of(t) == torch.cuda.current_stream().cuda_stream for t in want)
    # Blocks of the outputs' sizes, dropped while a kernel that is still to write them waits on the current stream.
    dropped = [[torch.empty_like(t) for t in want] for _ in range(3)]
    torch.cuda.synchronize()
    torch.cuda._sleep(10_000_000)
    for ts in dropped:
        for t in ts:
            t.fill_(7)
    at = {t.data_ptr() for ts in dropped for t in ts}
    del dropped, ts, t
    got = call(s)
    assert all(stream_of(t) == s.cuda_stream and t.data_ptr() not in at for t in got)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


@pytest.mark.parametrize("make", [rope, attention, cache_rows, similarity, layers])
def test_outputs_dropped_while_the_current_stream_reads_them(make):
    """What the caller does with outputs on the current stream ends before their memory is handed out again."""
    call = make(200)
    s = torch.cuda.Stream()
    got = call(s)
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda._sleep(10_000_000)
    kept = [t.clone() for t in got]
    at = {t.data_ptr() for t in got}
    del got
    again = call(s)
    assert not at & {t.data_ptr() for t in again}
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(kept, again))


def test_given_outputs_are_used():
    q, k, v = rows(50, 4), rows(50, 2), rows(50, 2)
    want = B.prompt_attn(q, k, v, [50])
    s = torch.cuda.Stream()
    out = torch.empty_like(q)
    torch.cuda.synchronize()
    assert B.prompt_attn(q, k, v, [50], out=out, stream=s) is out
    s.synchronize()
    assert torch.equal(out, want)
