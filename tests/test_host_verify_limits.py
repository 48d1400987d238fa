"""The sizes that baklava_verify_draft takes, on both sides of its limits, without a GPU."""
import pytest
import torch

from paper_2502_13176_amd import binding as B
from test_host_drafts import verify
from test_host_operators import OKP

MOST = (1 << 21) - 1  # rows times parts of 8192 elements


@pytest.mark.parametrize("draft", [0, 1])
@pytest.mark.parametrize("n_seq,N,V", [(600000, 1, 1000), (MOST, 1, 1), (MOST, 1, 8192), (1 << 20, 1, 8192), (MOST // 2, 1, 8193), (MOST // 256, 256, 8192),
                                       (1, 15, 1 << 30), (15, 1, 1 << 30), (7, 1, (1 << 31) // 8), (1, 1, 1 << 30)])
def test_sizes_up_to_the_limit(n_seq, N, V, draft):
    need = B.lib().baklava_verify_workspace_bytes(n_seq, N, V, draft)
    assert need > 0
    # (a workspace that is too small is what is refused last)
    assert verify(n_seq=n_seq, N=N, V=V, row=V, draft=OKP if draft else None, draft_row=V, nbytes=need - 1) == B.ECAPACITY


@pytest.mark.parametrize("draft", [0, 1])
@pytest.mark.parametrize("n_seq,N,V", [(MOST + 1, 1, 1), (MOST // 2 + 1, 1, 8193), (1 << 20, 2, 5), (MOST // 256 + 1, 256, 8192), (1, 16, 1 << 30), (16, 1, 1 << 30),
                                       (1, 1, (1 << 30) + 1), (2147483647, 256, 1 << 30)])
def test_sizes_beyond_the_limit(n_seq, N, V, draft):
    assert B.lib().baklava_verify_workspace_bytes(n_seq, N, V, draft) == 0
    assert verify(n_seq=n_seq, N=N, V=V, row=V, draft=OKP if draft else None, draft_row=V) == B.EINVAL
