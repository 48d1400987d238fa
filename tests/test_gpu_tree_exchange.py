"""GPU parity: values of 4-bit rows pass from lane to lane in LDS, slab after slab of a wavefront (baklava_tree_attn)."""
import pytest
import torch

from paper_2502_13176_amd import binding as B
from test_gpu_tree import nodes, parents

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,N", [(1, 1), (4, 3), (4, 8)])
def test_every_slab_of_a_wavefront_gives_its_own_rows(D, G, N):
    """Eight wavefronts take slabs of 32 rows in turn, so two slabs of a wavefront are 256 rows apart.  Every other 256 rows weigh nothing and
    have positive values, the others weigh the same and have negative ones: outputs are means of the latter, and a value that came from the slab
    before or behind shows."""
    n = 300001
    a = B.Arena(1, G, 1, D, 1, "mxfp4", [n], 8, 0, 0)
    g = torch.Generator(device="cuda").manual_seed(D + N)
    heavy = (torch.arange(a.total_tokens, device="cuda") // 256 % 2 == 0).view(-1, 1)
    a.k.copy_(torch.where(heavy, 0x22, 0xAA).to(torch.uint8).expand_as(a.k))  # 1 and -1 throughout
    code = torch.randint(0, 256, a.v.shape, generator=g, device="cuda", dtype=torch.uint8)
    a.v.copy_(torch.where(heavy, code | 0x88, code & 0x77))
    a.kv_scale.copy_(torch.randint(124, 131, a.kv_scale.shape, generator=g, device="cuda", dtype=torch.uint8))
    a.kv_scale[:, :D // 32] = 127
    a.set_lengths([n])
    cpu = torch.Generator().manual_seed(1)
    q, k, v = (nodes("packed", 1, N, h, D, torch.bfloat16, cpu) for h in (G, 1, 1))
    k.zero_(), v.zero_(), q.fill_(8.0)  # logits of 8 sqrt(D) and -8 sqrt(D); the nodes' own rows, at 0, weigh 2^-92 of a heavy one at most
    out = a.tree_attn(0, 1, k, v, torch.from_numpy(parents("chain", 1, N)).cuda(), q)
    x = a.read_rows(0, 1, n)[1][0].double()[heavy[:n, 0]]
    want, size = x.mean(0), x.abs().mean(0)
    assert (want < -0.5).all()
    # sums of len(x) terms in fp32 by 2048 wavefronts: len(x) / 2048 + 2048 half steps; the output's rounding
    tol = want.abs() * 2.0 ** -8 + size * (len(x) / 2048 + 2048 + 10) * 2.0 ** -24
    assert ((out.double() - want).abs() <= tol).all(), float(((out.double() - want).abs() / tol).max())
