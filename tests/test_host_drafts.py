"""What the entry points of steps over drafted tokens refuse, without a GPU: every check comes before anything is enqueued."""
import ctypes as C

import pytest
import torch

from paper_2502_13176_amd import binding as B
from test_host_operators import OKP

WS = 0x100000


def verify(logits=OKP, row=100, draft=None, draft_row=0, dtype=B.BF16, n_seq=2, N=3, V=100, token=OKP, parent=OKP, nodes=None, temp=None, u=OKP,
           path=OKP, n_path=OKP, nxt=OKP, ws=WS, nbytes=1 << 30):
    return B.lib().baklava_verify_draft(logits, row, draft, draft_row, dtype, n_seq, N, V, token, parent, nodes, temp, u, path, n_path, nxt, ws, nbytes, None)


@pytest.mark.parametrize("kw", [dict(logits=None), dict(logits=OKP + 1), dict(dtype=B.F32, logits=OKP + 2), dict(draft=OKP + 1), dict(row=-1),
                                dict(row=1 << 62), dict(draft=OKP, draft_row=-5), dict(draft=OKP, draft_row=1 << 61), dict(dtype=2), dict(dtype=-1), dict(n_seq=0),
                                dict(n_seq=-2), dict(N=0), dict(N=257), dict(V=0), dict(V=(1 << 30) + 1), dict(n_seq=1 << 20, N=256), dict(V=1 << 30, N=200, n_seq=10),
                                dict(token=None), dict(token=OKP + 2), dict(parent=None), dict(parent=OKP + 1), dict(nodes=OKP + 3), dict(temp=OKP + 2),
                                dict(u=None), dict(u=OKP + 1), dict(path=None), dict(path=OKP + 2), dict(n_path=None), dict(n_path=OKP + 2), dict(nxt=None),
                                dict(nxt=OKP + 1), dict(ws=None), dict(ws=WS + 128)])
def test_verify_refuses(kw):
    assert verify(**kw) == B.EINVAL


def test_verify_asks_for_its_workspace():
    for draft in (None, OKP):
        need = B.lib().baklava_verify_workspace_bytes(2, 3, 100, int(draft is not None))
        assert need > 0 and verify(draft=draft, draft_row=100, nbytes=need - 1) == B.ECAPACITY
    size = B.lib().baklava_verify_workspace_bytes
    assert size(0, 3, 100, 0) == size(2, 0, 100, 0) == size(2, 257, 100, 0) == size(2, 3, 0, 0) == size(1 << 20, 256, 100, 0) == 0
    assert size(2, 3, 100, 1) > size(2, 3, 100, 0) and size(2, 3, 1 << 20, 0) > size(2, 3, 100, 0)


def test_calls_without_a_context():
    L = B.lib()
    assert L.baklava_tree_workspace_bytes(None, 1, 4) == 0
    assert L.baklava_tree_attn(None, 0, 1, OKP, OKP, 4, OKP, None, OKP, OKP, None, WS, 1 << 30, None) == B.EINVAL
    assert L.baklava_append_accepted(None, 0, 1, OKP, OKP, 4, OKP, OKP, OKP, None, None, None) == B.EINVAL


def test_binding_refuses_tensors_of_verify():
    f, i = torch.float32, torch.int32
    good = dict(logits=torch.zeros(2, 3, 50), token=torch.zeros(2, 3, dtype=i), parent=torch.zeros(2, 3, dtype=i), u=torch.zeros(2, 3))
    for name, bad in (("parent", torch.zeros(2, 3)), ("parent", torch.zeros(6, dtype=i)), ("parent", torch.zeros(2, 6, dtype=i)[:, ::2]), ("parent", torch.zeros(2, 0, dtype=i)),
                      ("token", torch.zeros(2, 4, dtype=i)), ("token", torch.zeros(2, 3, dtype=torch.int64)), ("u", torch.zeros(2, 3, dtype=torch.float64))):
        with pytest.raises(ValueError):
            B.verify_draft(**(good | {name: bad}))
    with pytest.raises(ValueError, match="current GPU"):  # (host tensors)
        B.verify_draft(**good)
