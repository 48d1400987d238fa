"""GPU parity: a 4-bit cache of as many rows as one may have, 2^31 bytes of codes a plane, in the longest work items there are."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as OP
from paper_2502_13176_amd import binding as B

pytestmark = pytest.mark.gpu

CAP = 1 << 25
G, D = 16, 128


def grid(x):
    code, s = OP.mx_round(torch.from_numpy(x).bfloat16().double().numpy())
    return code, s, OP.mx_values(OP.mx_pack(code), s)


def test_the_longest_cache_in_the_longest_work_items():
    """All rows but a few, near the ends of the cache and of its eight work items, are zero: logit 0, which is the largest (queries are positive, the other
    keys negative), so that a zero row's weight is 1 before the division and sums of them are exact in fp32 (fewer than 2^24 a
    lane).  Values of the other rows are large, to be seen among 2^25.  Two calls fill a record: the third adds it, in a pass
    of its own, the flush what is left.  Tolerances as in test_gpu_mxfp4.py."""
    rng = np.random.default_rng(5)
    n = CAP - 5
    a = B.Arena(1, G, 1, D, 1, "mxfp4", [CAP - 64], 64, 4, 16, B.POLICY_SCORE, True)
    assert int(a.cap_host[0]) == CAP
    for o in (B.OPT_TARGET_ITEMS, B.OPT_TARGET_ITEMS_WHOLE):
        a.set_option(o, 1)
    assert all([i[2] for i in B.plan_schedule(a.off_host, a.cap_host, 1, 1, 256, w, target_items=1)] == [1 << 22] * 8 for w in (False, True))
    a.kv_scale.fill_(127)
    at = [0, 1, 300, (1 << 22) - 1, 1 << 22, (1 << 24) - 1, 1 << 24, (1 << 24) + 77, n - 257, n - 33, n - 32, n - 1]
    kc, ks, K = grid(-np.abs(rng.standard_normal((len(at), D))))
    vc, vs, V = grid(rng.standard_normal((len(at), D)) * 2.0 ** 20)
    i = torch.tensor(at).cuda()
    a.k[i], a.v[i] = torch.from_numpy(OP.mx_pack(kc)).cuda(), torch.from_numpy(OP.mx_pack(vc)).cuda()
    a.kv_scale[i] = torch.from_numpy(np.concatenate([ks, vs], 1)).cuda()
    a.set_lengths([n])
    zero = n - len(at)
    score, zero_score, off, zero_off = np.zeros(len(at)), 0.0, np.zeros(len(at)), 0.0
    for step in range(5):
        k, v = -np.abs(rng.standard_normal((1, D))), rng.standard_normal((1, D)) * 2.0 ** 20
        kd, vd = (torch.from_numpy(x).bfloat16().view(1, 1, 1, D).cuda() for x in (k, v))
        q = torch.from_numpy(np.abs(rng.standard_normal((1, 1, G, D)))).bfloat16()
        out = torch.full((1, 1, G, D), float("nan"), device="cuda")
        a.append_decode_attn(0, 1, kd, vd, n + step, q.cuda(), out)
        torch.cuda.synchronize()
        print("step", step, flush=True)
        K, V, at = np.vstack([K, grid(k)[2]]), np.vstack([V, grid(v)[2]]), at + [n + step]
        score, off = np.append(score, 0.0), np.append(off, 0.0)
        got = out[0, 0].double().cpu().numpy()
        for h in range(G):
            row = q[0, 0, h].double().numpy()
            e = np.exp(K @ row / np.sqrt(D))
            p, p0 = e / (zero + e.sum()), 1 / (zero + e.sum())
            rel = 2 * D * 2.0 ** -24 * (np.abs(K) @ row).max() / np.sqrt(D) + 2.0 ** -18
            assert (np.abs(got[h] - p @ V) <= rel * (p @ np.abs(V))).all(), (step, h)
            score, zero_score = score + p, zero_score + p0
            off, zero_off = off + rel * p, zero_off + rel * p0
    a.flush_scores(0, 1)
    torch.cuda.synchronize()
    assert a.len.cpu().tolist() == [CAP]
    sums = 2.0 ** -24 * (5 * (G + 1) + 1)
    sc = a.score[torch.tensor(at).cuda()].double().cpu().numpy()
    assert (np.abs(sc - score) <= off + sums * score).all()
    rest = torch.ones((CAP,), dtype=torch.bool, device="cuda")
    rest[torch.tensor(at).cuda()] = False
    low, high = (float(x) for x in torch.aminmax(a.score[rest]))
    assert abs(low - zero_score) <= zero_off + sums * zero_score and abs(high - zero_score) <= zero_off + sums * zero_score
    kr, vr = a.read_rows(0, 1, 40)
    for t, x in ((kr, K), (vr, V)):
        want = np.zeros((40, D))
        want[[r - (CAP - 40) for r in at if r >= CAP - 40]] = x[[j for j, r in enumerate(at) if r >= CAP - 40]]
        assert np.array_equal(t[0].double().cpu().numpy(), want)
    a.close()
