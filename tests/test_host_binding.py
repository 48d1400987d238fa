"""What the binding refuses before it calls the library, without a GPU."""
import array

import numpy as np
import pytest
import torch

from paper_2502_13176_amd import binding as B


def scores(**kw):
    a = dict(q=torch.zeros((2, 4, 6, 128), dtype=torch.bfloat16), k_plane=torch.zeros((2, 2, 6, 128), dtype=torch.bfloat16),
             lse=torch.zeros((2, 4, 6)), score_plane=torch.zeros((24,)), batch=2, Hq=4, Hkv=2, T=6)
    B.prefill_scores(**{**a, **kw})


@pytest.mark.parametrize("kw", [
    dict(k_plane=torch.zeros((24, 64), dtype=torch.uint8)),                           # the K plane of a 4-bit arena
    dict(k_plane=torch.zeros((24, 64), dtype=torch.uint8), row_off=torch.zeros((4,), dtype=torch.int64)),
    dict(k_plane=torch.zeros((5, 128), dtype=torch.bfloat16), row_off=torch.zeros((4,), dtype=torch.int64)),
    dict(k_plane=torch.zeros((48, 64), dtype=torch.bfloat16)), dict(k_plane=torch.zeros((24, 128))), dict(q=torch.zeros((2, 4, 6, 128))),
    dict(k_plane=torch.zeros((23, 128), dtype=torch.bfloat16)), dict(q=torch.zeros((2, 4, 5, 128), dtype=torch.bfloat16)),
    dict(q=torch.zeros((2, 6, 4, 128), dtype=torch.bfloat16).transpose(1, 2)), dict(lse=torch.zeros((2, 4, 6), dtype=torch.float64)),
    dict(lse=torch.zeros((4, 6))), dict(lse=torch.zeros((2, 4, 12))[:, :, ::2]), dict(score_plane=torch.zeros((23,))),
    dict(score_plane=torch.zeros((24,), dtype=torch.bfloat16)), dict(row_off=torch.zeros((3,), dtype=torch.int64)),
    dict(row_off=torch.zeros((4,), dtype=torch.int32))])
def test_prefill_scores_refuses(kw):
    with pytest.raises(ValueError):
        scores(**kw)


def test_caches_in_4_bits_take_no_codes():
    a = B.Arena.__new__(B.Arena)                          # (a context takes a GPU; the refusal comes before it is used)
    a.torch, a.dtype, a.mx, a.ctx = torch, "mxfp4", True, None
    row, codes, wide, out = (torch.zeros((1, 1, 2, n), dtype=t) for n, t in ((128, torch.bfloat16), (64, torch.uint8), (128, torch.float32),
                                                                             (128, torch.float32)))
    pos = torch.zeros((1,), dtype=torch.int32)
    for bad in (codes, wide):
        for k, v, q in ((bad, row, row), (row, bad, row), (row, row, bad)):
            with pytest.raises(ValueError):
                a.append_decode_attn(0, 1, k, v, 0, q, out)
            with pytest.raises(ValueError):
                a.append_decode_attn_replay(0, 1, k, v, pos, q, out)
        for k, v in ((bad, row), (row, bad)):
            with pytest.raises(ValueError):
                a.append(0, 1, k, v, 0)
        with pytest.raises(ValueError):
            a.decode_attn(0, 1, bad, out)


@pytest.mark.parametrize("which", range(3))
def test_prompt_attn_refuses_tensors_that_require_a_gradient(which):
    t = [torch.zeros((3, 2, 64), dtype=torch.bfloat16) for _ in range(3)]
    t[which].requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        B.prompt_attn(*t, [3])
    with torch.no_grad(), pytest.raises(ValueError, match="GPU"):  # refused for where it is alone
        B.prompt_attn(*t, [3])
    with pytest.raises(ValueError, match="GPU"):
        B.prompt_attn(*(x.detach() for x in t), [3])


@pytest.mark.parametrize("which", range(4))
def test_qk_norm_rope_refuses_tensors_that_require_a_gradient(which):
    t = [torch.zeros(s) for s in ((3, 2, 64), (3, 1, 64), (64,), (64,))]
    t[which].requires_grad_()
    pos = torch.zeros((3,), dtype=torch.int32)
    with pytest.raises(ValueError, match="gradient"):
        B.qk_norm_rope(t[0], t[1], pos, [1.0] * 32, q_weight=t[2], k_weight=t[3])
    with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
        B.qk_norm_rope(t[0], t[1], pos, [1.0] * 32, q_weight=t[2], k_weight=t[3])


@pytest.mark.parametrize("make", [list, tuple, np.array, lambda a: np.array(a, dtype=np.uint8), lambda a: array.array("i", a), torch.tensor, bytes])
def test_axes_of_pairs_in_any_sequence(make):
    axis = [0, 2, 1, 1, 0]
    assert B._axes(None, make(axis), 5, 3) == bytes(axis)
    assert B._axes(make([2, 0, 3]), None, 5, 3) == bytes([0, 0, 2, 2, 2])
    assert B._axes(make([5]), None, 5, 3) is None and B._axes(None, None, 5, 3) is None
    for sections, pairs in (([2, 2], None), ([2, 1, 1, 1], None), ([1, 4], axis), (None, axis[:4]), (None, [0, 3, 0, 0, 0])):
        with pytest.raises(ValueError):
            B._axes(make(sections) if sections else None, make(pairs) if pairs else None, 5, 3)


def test_rows_of_an_arena_on_another_gpu(monkeypatch):
    a = B.Arena.__new__(B.Arena)
    a.torch, a.dtype, a.mx, a.ctx, a.gpu, a.device = torch, "bf16", False, None, 1, torch.device("cpu")
    a.L, a.batch, a.Hkv, a.D = 1, 1, 2, 64
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "is_initialized", lambda: True)
    k = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="arena"):
        a.append_prompt(0, k, k, [3])
    with pytest.raises(ValueError, match="arena"):
        a.read_rows(0, 1, 1)
