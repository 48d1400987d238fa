"""GPU parity: prompts that follow replayed decode steps, of which the host mirror of the lengths knows nothing until it is synchronised."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as OP
from paper_2502_13176_amd import binding as B

pytestmark = pytest.mark.gpu


def values(x, dtype):
    x = x.double().cpu().numpy()
    if dtype == "mxfp4":
        code, s = OP.mx_round(x)
        return OP.mx_values(OP.mx_pack(code), s)
    return x


class Run:
    """An arena, and the rows its caches should hold."""

    def __init__(self, dtype, cap, batch=2, Hkv=2, D=64, track=False):
        self.dtype, self.batch, self.Hkv, self.D = dtype, batch, Hkv, D
        self.t = torch.float32 if dtype == "f32" else torch.bfloat16
        self.a = B.Arena(1, 2 * Hkv, Hkv, D, batch, dtype, [cap] * Hkv, 0, 0, 0, B.POLICY_SCORE, track, workspace_fill=0xFF)
        self.a.score.fill_(-5.0), self.a.pos.fill_(-7)
        self.a.reset()
        self.K, self.V, self.pos = ([[] for _ in range(batch * Hkv)] for _ in range(3))
        self.kn, self.vn = (torch.zeros((1, batch, Hkv, D), dtype=self.t, device="cuda") for _ in range(2))
        self.q = torch.zeros((1, batch, 2 * Hkv, D), dtype=self.t, device="cuda")
        self.out = torch.zeros((1, batch, 2 * Hkv, D), device="cuda")
        self.at = torch.tensor([100], dtype=torch.int32, device="cuda")

    def prompt(self, lens, pos0, refused=()):
        k, v = (torch.randn((sum(lens), self.Hkv, self.D)).to(self.t).cuda() for _ in range(2))
        self.a.append_prompt(0, k, v, lens, pos0)
        for b, n in enumerate(lens):
            x = slice(sum(lens[:b]), sum(lens[:b]) + n)
            for h in range(self.Hkv):
                if b * self.Hkv + h not in refused:
                    self.keep(b * self.Hkv + h, values(k[x, h], self.dtype), values(v[x, h], self.dtype), pos0[b] + np.arange(n))

    def keep(self, c, k, v, pos):
        self.K[c].append(k), self.V[c].append(v), self.pos[c].append(pos)

    def step(self):
        self.a.append_decode_attn_replay(0, 1, self.kn, self.vn, self.at, self.q, self.out)

    def stepped(self):
        """The step's rows, after it ran."""
        for b in range(self.batch):
            for h in range(self.Hkv):
                c = b * self.Hkv + h
                self.keep(c, values(self.kn[0, b, h][None], self.dtype), values(self.vn[0, b, h][None], self.dtype), self.at.cpu().numpy())

    def new_rows(self, i):
        self.kn.normal_(), self.vn.normal_(), self.q.normal_()
        self.at.fill_(100 + i)

    def check(self, full=False):
        a = self.a
        torch.cuda.synchronize()
        if full:
            with pytest.raises(B.BaklavaError) as e:
                a.sync_lengths()
            assert e.value.status == B.ECAPACITY
        a.sync_lengths()
        n = [sum(len(x) for x in k) for k in self.K]
        assert a.lengths().tolist() == n and a.len.cpu().tolist() == n
        kr, vr = a.read_rows(0, 1, max(n))
        ps, sc = a.pos.cpu().numpy(), a.score.cpu().numpy()
        for c, m in enumerate(n):
            o = int(a.off_host[c])
            assert np.array_equal(kr[c, max(n) - m:].double().cpu().numpy(), np.concatenate(self.K[c]))
            assert np.array_equal(vr[c, max(n) - m:].double().cpu().numpy(), np.concatenate(self.V[c]))
            assert np.array_equal(ps[o:o + m], np.concatenate(self.pos[c]))
            end = o + int(a.cap_host[c])
            assert (ps[o + m:end] == -7).all() and (sc[o + m:end] == -5).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32", "mxfp4"])
@pytest.mark.parametrize("n", [1, 64, 65, 400])
def test_rows_go_behind_steps_the_mirror_does_not_know(dtype, n):
    r = Run(dtype, 1000)
    r.prompt([3, 90], [0, 5])
    for turn in range(2):
        for i in range(3):
            r.new_rows(10 * turn + i)
            r.step()
            r.stepped()
        r.prompt([n, max(0, n - 64)], [1000, 2000])
    r.check()


def test_rows_go_behind_replays_of_a_graph():
    r = Run("mxfp4", 9300, batch=1, Hkv=3, D=128, track=True)
    r.prompt([40], [0])
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        r.step()
    for turn, n in enumerate((8300, 130, 5)):             # more than 128 tiles, some, one
        for i in range(4):
            r.new_rows(10 * turn + i)
            g.replay()
            r.stepped()
        r.prompt([n], [5000 * turn])
        if turn == 1:
            r.a.flush_scores(0, 1)                        # (draws the same tickets)
    torch.cuda.synchronize()
    assert np.isfinite(r.a.score.cpu().numpy()).all()
    r.check()


@pytest.mark.parametrize("dtype", ["bf16", "mxfp4"])
def test_a_long_prompt_and_one_full_cache(dtype):
    """More tiles than draw tickets; the second sequence's caches have room on the device, the first one's have not."""
    r = Run(dtype, 9000, Hkv=3)
    r.prompt([500, 3], [0, 0])
    for i in range(2):
        r.new_rows(i)
        r.step()
        r.stepped()
    r.prompt([8500, 8990], [500, 600], refused=(0, 1, 2))
    r.check(full=True)
    r.prompt([8498, 5], [500, 600])
    r.check()


@pytest.mark.parametrize("dtype", ["bf16", "mxfp4"])
def test_a_cache_that_the_device_finds_full_stays_as_it_is(dtype):
    r = Run(dtype, 300)
    r.prompt([100, 10], [0, 0])
    for i in range(2):
        r.new_rows(i)
        r.step()
        r.stepped()
    r.prompt([199, 199], [500, 600], refused=(0, 1))      # 102 and 12 rows on the device, 100 and 10 in the mirror
    r.check(full=True)
    r.prompt([198, 88], [500, 600])                       # all that is left
    r.check()
    with pytest.raises(B.BaklavaError) as e:
        r.prompt([1, 0], [0, 0])
    assert e.value.status == B.ECAPACITY


def test_a_captured_prompt_keeps_its_rows():
    """... whatever the device's lengths are when it is replayed."""
    r = Run("bf16", 300, batch=1)
    r.prompt([70], [0])
    r.a.sync_lengths()
    k, v = (torch.randn((130, 2, 64)).bfloat16().cuda() for _ in range(2))
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(g, stream=s):
        r.a.append_prompt(0, k, v, [130], [70])
    for i in range(3):
        k.normal_(), v.normal_()
        g.replay()
        torch.cuda.synchronize()
        assert r.a.len.cpu().tolist() == [200, 200] and r.a.lengths().tolist() == [200, 200]
        kr, vr = r.a.read_rows(0, 1, 200)
        assert torch.equal(kr[:, 70:], k.transpose(0, 1)) and torch.equal(vr[:, 70:], v.transpose(0, 1))
        assert np.array_equal(kr[0, :70].double().cpu().numpy(), r.K[0][0])
