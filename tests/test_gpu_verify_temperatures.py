"""GPU parity: verification of drafted tokens at the largest temperatures, where differences beyond fp32 count.  Paths and tokens exactly those of
fp64."""
import pytest
import torch

from test_gpu_verify import expect, inputs, run, same

pytestmark = pytest.mark.gpu

LAST = 1 - 2.0 ** -24  # the largest random number


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("drafts", [False, True])
@pytest.mark.parametrize("temp", [1e30, 3e38, float("inf")])
def test_an_infinity_beside_the_lowest_value_at_the_largest_temperatures(dtype, drafts, temp):
    """Differences beyond fp32 that such a temperature brings back: at an infinite one every token that is not -inf weighs the same."""
    batch, N, V = 6, 7, 300
    for tree in ("chain", "tree"):
        t = inputs(batch, N, V, tree, dtype, drafts, 11)
        low = torch.finfo(t["logits"].dtype).min
        for x in (t["logits"], t["draft_logits"]):
            if x is not None:
                keep = torch.rand((batch, N, V), generator=torch.Generator().manual_seed(5)) < 0.6
                x.masked_fill_(~keep, low)
                x[4, 0, 17], x[4, 1, 18] = float("inf"), float("inf")
                x[5, 1, 3], x[5, 1, 5], x[5, 0, 7] = -low, -low, float("inf")
        T = torch.full((batch,), temp)
        same(run(t, temperature=T), expect(t, T))
    # three tokens, one of them drafted: a third of the weight at an infinite temperature, whatever they are
    u = torch.linspace(0, LAST, 64).view(64, 1).expand(64, 2).contiguous()
    x = torch.zeros((64, 2, 3), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    x[:, 0, 0], x[:, 0, 1] = float("inf"), torch.finfo(x.dtype).min
    for token in range(3):
        s = dict(logits=x, token=torch.tensor([[0, token]] * 64).int(), parent=torch.tensor([[-1, 0]] * 64).int(), u=u, draft_logits=None)
        same(run(s, temperature=torch.full((64,), temp)), expect(s, torch.full((64,), temp)))
