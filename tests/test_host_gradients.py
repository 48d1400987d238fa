"""Tensors that require a gradient at the calls of steps over drafted tokens, without a GPU: refused before anything else is looked at."""
import types

import pytest
import torch

from paper_2502_13176_amd import binding as B


@pytest.mark.parametrize("which", ["k", "v", "q", "lse"])
def test_append_accepted_refuses_tensors_that_require_a_gradient(which):
    t = {n: torch.zeros(3, 2, 128) for n in ("k", "v", "q")} | {"lse": torch.zeros(2, 3)}
    t[which].requires_grad_()
    path, n = torch.zeros(1, 3, dtype=torch.int32), torch.ones(1, dtype=torch.int32)
    call = lambda: B.Arena.append_accepted(types.SimpleNamespace(torch=torch), 0, 1, t["k"], t["v"], path, n, n, q=t["q"], lse=t["lse"])
    with pytest.raises(ValueError, match="gradient"):
        call()
    with torch.no_grad(), pytest.raises(Exception) as e:  # (what is wrong then is that there is no arena)
        call()
    assert "gradient" not in str(e.value)


def test_verify_draft_takes_logits_of_a_graph():
    """Paths and tokens are whole numbers: logits that require a gradient are refused for lying on the host, not for that."""
    z = torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="current GPU"):
        B.verify_draft(torch.zeros(1, 2, 9, requires_grad=True), z, z, torch.zeros(1, 2))
