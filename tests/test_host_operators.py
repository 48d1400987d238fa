"""What the entry points around the prompts refuse, without a GPU: every check comes before anything is enqueued."""
import ctypes as C

import numpy as np
import pytest

from paper_2502_13176_amd import binding as B

OKP = 0x10000                                             # never dereferenced: the calls fail on their arguments


class Rows(C.Structure):                                  # baklava_rows
    _fields_ = [("data", C.c_void_p), ("seq_stride", C.c_int64), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


def rows(data=OKP, seq=0, tok=1024, head=128):
    return Rows(data, seq, tok, head)


def ref(r):
    return C.addressof(r) if r is not None else None


def i32(*x):
    return (C.c_int32 * max(1, len(x)))(*x)


def rope(q=rows(), k=rows(), n_seq=1, T=4, Hq=4, Hkv=2, D=128, dtype=B.BF16, wq=OKP, wk=OKP, eps=1e-6, pos=OKP, axes=1, axis=None,
         freq=(1.0,) * 64, rot=128, qo=rows(), ko=rows()):
    f = (C.c_double * 64)(*freq) if freq is not None else None
    a = bytes(axis) if axis is not None else None
    return B.lib().baklava_qk_norm_rope(ref(q), ref(k), n_seq, T, Hq, Hkv, D, dtype, wq, wk, eps, pos, axes, a,
                                        f, rot, 0, ref(qo),
                                        ref(ko), None)


BAD_ROWS = [None, rows(data=None), rows(data=OKP + 8), rows(tok=1020), rows(head=124), rows(tok=-1024), rows(head=-128),
            rows(tok=1 << 24)]


@pytest.mark.parametrize("bad", range(len(BAD_ROWS)))
@pytest.mark.parametrize("arg", ["q", "k", "qo", "ko"])
def test_rope_refuses_rows(arg, bad):
    assert rope(**{arg: BAD_ROWS[bad]}) == B.EINVAL


@pytest.mark.parametrize("kw", [dict(n_seq=0), dict(T=0), dict(T=-1), dict(T=(1 << 26) + 1), dict(Hq=-1), dict(Hq=0, Hkv=0), dict(D=96), dict(dtype=2),
                                dict(dtype=7), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(rot=127), dict(rot=130),
                                dict(rot=-2), dict(pos=None), dict(pos=OKP + 2), dict(axes=0), dict(axes=9), dict(freq=None),
                                dict(freq=(float("nan"),) * 64), dict(freq=(float("inf"),) * 64), dict(axis=[1] * 64), dict(wq=OKP + 4),
                                dict(wk=OKP + 8), dict(qo=rows(tok=64)), dict(qo=rows(head=0)), dict(ko=rows(head=64)),
                                dict(n_seq=2, qo=rows(seq=64)), dict(n_seq=2, q=rows(seq=1004))])
def test_rope_refuses(kw):
    assert rope(**kw) == B.EINVAL


def attn(q=rows(), k=rows(), v=rows(), q_len=(4, 0, 7), kv_len=None, Hq=4, Hkv=2, D=128, dtype=B.BF16, out=rows(), lse=Rows(OKP, 0, 1, 11)):
    n = len(q_len) if q_len is not None else 3
    return B.lib().baklava_prompt_attn(ref(q), ref(k), ref(v), n, i32(*q_len) if q_len is not None else None,
                                       i32(*kv_len) if kv_len is not None else None, Hq, Hkv, D, dtype, ref(out), ref(lse), None)


@pytest.mark.parametrize("bad", range(len(BAD_ROWS)))
@pytest.mark.parametrize("arg", ["q", "k", "v", "out"])
def test_prompt_attn_refuses_rows(arg, bad):
    assert attn(**{arg: BAD_ROWS[bad]}) == B.EINVAL


@pytest.mark.parametrize("kw", [dict(q_len=None), dict(q_len=()), dict(q_len=(-1,)), dict(kv_len=(4, 0, -7)), dict(q_len=((1 << 29) + 1,)),
                                dict(q_len=(1 << 29,) * 4), dict(kv_len=(1 << 29, 1 << 29, (1 << 29) + 1)), dict(Hq=0), dict(Hkv=0), dict(Hq=3), dict(D=96), dict(dtype=B.F32),
                                dict(dtype=B.MXFP4), dict(lse=Rows(None, 0, 1, 11)), dict(lse=Rows(OKP + 2, 0, 1, 11)),
                                dict(lse=Rows(OKP, 0, 0, 11)), dict(lse=Rows(OKP, 0, 1, 0)), dict(lse=Rows(OKP, 0, 1, -11)),
                                dict(out=rows(tok=120)), dict(out=rows(head=0))])
def test_prompt_attn_refuses(kw):
    assert attn(**kw) == B.EINVAL


def test_prompt_attn_without_tokens_does_nothing():
    assert attn(q_len=(0, 0)) == B.OK
    assert attn(q_len=(0, 0), kv_len=(5, 9), q=None, k=None, v=None, out=None, lse=None) == B.OK


def test_calls_on_a_context_refuse_null():
    L = B.lib()
    assert L.baklava_append_prompt(None, 0, ref(rows()), ref(rows()), i32(1), None, None, None) == B.EINVAL
    assert L.baklava_read_rows(None, 0, 1, 1, OKP, OKP, None) == B.EINVAL


def mx_desc(Hq=4, Hkv=2, D=128):
    d = B.Desc()
    d.L, d.Hq, d.Hkv, d.D, d.batch, d.dtype = 1, Hq, Hkv, D, 1, B.MXFP4
    fake = 0x1000
    d.k = d.v = d.score = d.pos = d.off = d.cap = d.len = d.budget = d.workspace = d.kv_scale = fake
    d.workspace_bytes = 1 << 30
    return d


def create(d):
    b = np.asarray([64] * d.Hkv, dtype=np.int32)
    off, cap, _ = B.layout(b, 1, d.Hkv, 1, 0)
    ctx = C.c_void_p()
    return B.lib().baklava_create(C.byref(d), off.ctypes.data_as(C.POINTER(C.c_int64)), cap.ctypes.data_as(C.POINTER(C.c_int32)), None,
                                  b.ctypes.data_as(C.POINTER(C.c_int32)), C.byref(ctx))


def test_contexts_of_4_bit_rows_refuse():
    for scale in (None, 0x1004):
        d = mx_desc()
        d.kv_scale = scale
        assert create(d) == B.EINVAL
    for kw in (dict(D=96), dict(Hq=34, Hkv=2), dict(D=32)):
        assert create(mx_desc(**kw)) == B.EINVAL
    d = mx_desc()
    d.dtype = 3
    assert create(d) == B.EINVAL


def test_caches_of_4_bit_rows_have_a_most_length():
    i32p, i64p = C.POINTER(C.c_int32), C.POINTER(C.c_int64)
    budget = np.asarray([64, 64], dtype=np.int32)
    for more in (0, 1):
        cap = np.asarray([(1 << 25) + more, 64], dtype=np.int32)
        off = np.asarray([0, cap[0]], dtype=np.int64)
        d, ctx = mx_desc(), C.c_void_p()
        size = B.lib().baklava_workspace_bytes(C.byref(d), cap.ctypes.data_as(i32p), budget.ctypes.data_as(i32p))
        assert (size == 0) == bool(more)
        if more:
            assert B.lib().baklava_create(C.byref(d), off.ctypes.data_as(i64p), cap.ctypes.data_as(i32p), None,
                                          budget.ctypes.data_as(i32p), C.byref(ctx)) == B.EINVAL


def test_workspace_of_4_bit_rows_holds_records_of_bf16_queries():
    i32p = C.POINTER(C.c_int32)
    cap = np.full(2, 500, dtype=np.int32)
    for D in (64, 128):
        size = []
        for track in (0, 1):
            d = mx_desc(D=D)
            d.track_scores = track
            size.append(B.lib().baklava_workspace_bytes(C.byref(d), cap.ctypes.data_as(i32p), cap.ctypes.data_as(i32p)))
        assert size[0] > 0 and size[1] - size[0] == 2 * 32 * D * 2 + 2 * 32 * 2 * 4
