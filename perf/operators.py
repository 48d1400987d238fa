"""The operators around the ragged caches whose speed is measured: rows of queries and keys normed and
rotated, attention over whole prompts, prompts written into the caches, decode attention over caches held
in 4 bits.

Shapes are those of this repository's workloads (`paper_2502_13176_amd/synth.py`), with fewer layers where a
full stack would only repeat the same launches.  Where `own` is false everything is computed with elementary
torch operations in 32 bits; where it is true by the library's calls.

Caches in 4 bits: a row of D elements is D / 2 bytes of E2M1 codes (element 2 i in the low half of byte i) and
one E8M0 scale for every 32 elements; the scales of a row's key stand before those of its value.
"""
import math

import numpy as np
import torch

own = False

LOG2E = 1.4426950408889634
SINK, RECENT = 4, 16


def listed():
    return [
        # the queries and keys of one decode step of a serving batch, between two projections (launch latency)
        dict(name="rotate_step_b8", kind="rotate", dtype="bf16", n=8, Hq=32, Hkv=8, D=128, rot=128, axes=1, pairs=False, norm=True, far=32768),
        # a prompt with images: three position axes, fused projection in, odd length
        dict(name="rotate_axes_qwen_8k", kind="rotate", dtype="bf16", n=8191, Hq=28, Hkv=4, D=128, rot=128, axes=3, pairs=False, norm=True, far=8192),
        # a full-length prompt of one layer
        dict(name="rotate_llama_32k", kind="rotate", dtype="bf16", n=32768, Hq=32, Hkv=8, D=128, rot=128, axes=1, pairs=False, norm=True, far=32768),
        # short requests of a chat server, packed: heads of 64, from one token to two hundred
        dict(name="prompt_short_packed", kind="prompt", Hq=16, Hkv=8, D=64, seqs=16, T=200, least=1, prefix=0, padded=False),
        # requests of mixed length, packed
        dict(name="prompt_mixed_qwen", kind="prompt", Hq=28, Hkv=4, D=128, seqs=8, T=8192, least=128, prefix=0, padded=False),
        # one long prompt, heads in front of tokens
        dict(name="prompt_llama_16k", kind="prompt", Hq=32, Hkv=8, D=128, seqs=1, T=16384, least=16384, prefix=0, padded=True),
        # one layer's rows of a full-length prompt into caches in 4 bits
        dict(name="write_llama_32k_q4", kind="write", store="mxfp4", L=1, Hq=32, Hkv=8, D=128, batch=1, T=32768, least=32768, scores=True),
        # two layers of a small fp32 model, prompts of mixed length
        dict(name="write_mixed_f32", kind="write", store="f32", L=2, Hq=16, Hkv=8, D=64, batch=4, T=3001, least=500, scores=False),
        # one attention call of a single user over caches in 4 bits (latency)
        dict(name="attend_q4_llama_b1", kind="attend", L=1, Hq=32, Hkv=8, D=128, batch=1, ctx=8192, keep=50, sigma=1.0, lo=256, steps=1, whole=False),
        # heads of 64, tracked steps of a small batch
        dict(name="generate_q4_d64", kind="generate", L=2, Hq=16, Hkv=4, D=64, batch=4, ctx=16384, keep=50, sigma=1.0, lo=128, steps=4, whole=False),
        # the main path in 4 bits: tracked decode steps of a serving batch, one fused call per layer
        dict(name="generate_q4_llama_b8", kind="generate", L=4, Hq=32, Hkv=8, D=128, batch=8, ctx=32768, keep=30, sigma=1.5, lo=128, steps=8, whole=False),
        # contexts of up to 131072 rows, seven query heads, both layers in one call
        dict(name="generate_q4_long_whole", kind="generate", L=2, Hq=28, Hkv=4, D=128, batch=4, ctx=131072, keep=30, sigma=1.0, lo=256, steps=8, whole=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "prompt", "prompt", "write", "attend", "generate", "generate"])
    Hkv = rng.choice([1, 2, 4, 8])
    D = rng.choice([128, 128, 64])
    if kind == "rotate":
        Hq = Hkv * rng.choice([1, 2, 4, 7])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        rot = rng.choice([D, D, D // 2, 24])
        return dict(kind=kind, dtype=dtype, n=_log(rng, 1, 32768), Hq=Hq, Hkv=Hkv, D=D, rot=rot, axes=rng.choice([1, 1, 3]),
                    pairs=rng.random() < 0.3, norm=rng.random() < 0.8, far=_log(rng, 100, 1000000))
    if kind == "prompt":
        Hq = Hkv * rng.choice([1, 2, 4, 7])
        T = _log(rng, 1, 12000)
        most = max(1, min(32, int(4e9 // (Hq * T * T))))
        return dict(kind=kind, Hq=Hq, Hkv=Hkv, D=D, seqs=_log(rng, 1, most), T=T, least=rng.randint(1, T),
                    prefix=rng.choice([0, 0, _log(rng, 1, 2000)]), padded=rng.random() < 0.5)
    G = rng.choice([1, 2, 4, 7, 8, 16] if D == 128 else [1, 2, 4, 8])
    batch, L = _log(rng, 1, 16), rng.randint(1, 3)
    if kind == "write":
        T = _log(rng, 1, max(64, 500000 // (batch * Hkv * L)))
        return dict(kind=kind, store=rng.choice(["mxfp4", "mxfp4", "bf16", "f32"]), L=L, Hq=Hkv * min(G, 8), Hkv=Hkv, D=D, batch=batch, T=T,
                    least=rng.randint(0, T), scores=rng.random() < 0.5)
    ctx = _log(rng, 512, max(1024, min(131072, (1 << 22) // (batch * L * Hkv))))
    return dict(kind=kind, L=L, Hq=G * Hkv, Hkv=Hkv, D=D, batch=batch, ctx=ctx, keep=rng.choice([20, 30, 50]),
                sigma=rng.choice([0.5, 1.0, 1.5]), lo=64, steps=1 if kind == "attend" else rng.randint(1, 10), whole=rng.random() < 0.4)


# ---------------------------------------------------------------------------
# sizes that follow from a case alone
# ---------------------------------------------------------------------------

def _lengths(case, most):
    """Tokens of every sequence: the first has the most."""
    n = case["batch"] if case["kind"] == "write" else case["seqs"]
    rng = np.random.Generator(np.random.PCG64(n * 7919 + most))
    lens = rng.integers(case["least"], most + 1, n)
    lens[0] = most
    return [int(x) for x in lens]


def _budgets(case):
    """Rows of the cache of every layer and KV head, heavy-tailed, about keep percent of the context on average."""
    m = case["L"] * case["Hkv"]
    rng = np.random.Generator(np.random.PCG64(7))
    w = rng.lognormal(0.0, case["sigma"], m)
    b = case["ctx"] * case["keep"] / 100 * m * w / w.sum()
    return [int(x) for x in np.clip(b, min(case["lo"], case["ctx"]), case["ctx"])]


def _arena_lens(case):
    """Live rows of every cache, layer-major, then sequence, then KV head."""
    b = np.asarray(_budgets(case)).reshape(case["L"], 1, case["Hkv"])
    return np.broadcast_to(b, (case["L"], case["batch"], case["Hkv"])).reshape(-1).copy()


def _inv_freq(rot):
    return [500000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]


def _sections(case):
    """Pairs of every axis, in turn."""
    n = case["rot"] // 2
    if case["axes"] == 1:
        return [n]
    a = n // 4
    return [a, (n - a) // 2, n - a - (n - a) // 2]


def work(case):
    kind, D = case["kind"], case["D"]
    if kind == "rotate":
        es = 2 if case["dtype"] == "bf16" else 4
        rows = case["n"] * (case["Hq"] + case["Hkv"])
        return {"bytes": 2 * rows * D * es + 4 * case["axes"] * case["n"], "flops": rows * (4 * D + 3 * case["rot"])}
    if kind == "prompt":
        lens = _lengths(case, case["T"])
        pairs = sum(t * (t + 1) / 2 + t * case["prefix"] for t in lens) * case["Hq"]
        n, keys = sum(lens), sum(lens) + len(lens) * case["prefix"]
        return {"bytes": 4 * n * case["Hq"] * D + 4 * keys * case["Hkv"] * D + 4 * n * case["Hq"], "flops": 4.0 * D * pairs}
    if kind == "write":
        es = 4 if case["store"] == "f32" else 2
        stored = D // 2 + D // 32 if case["store"] == "mxfp4" else D * es
        rows = case["L"] * case["Hkv"] * sum(_lengths(case, case["T"]))
        # (reading the rows back is part of the pass)
        return {"bytes": rows * (2 * D * es + 4 * stored + 8 + (4 if case["scores"] else 0) + 2 * D * es), "flops": 0}
    rows, steps = int(_arena_lens(case).sum()), case["steps"]
    caches, heads = case["L"] * case["batch"] * case["Hkv"], case["L"] * case["batch"] * case["Hq"]
    seen = steps * rows + (caches * steps * (steps + 1) // 2 if kind == "generate" else 0)
    moved = seen * (D + D // 16) + steps * heads * D * 6
    if kind == "generate":
        moved += 8 * (rows + caches * steps) + caches * steps * D * 8
    return {"bytes": moved, "flops": 4.0 * D * seen * (case["Hq"] // case["Hkv"])}


# ---------------------------------------------------------------------------
# 4-bit rows, with elementary operations
# ---------------------------------------------------------------------------

def _quantized(x):
    """Codes (0 .. 15, one byte each) and E8M0 scale bytes of rows x [..., D] of finite values.  A block's scale is the
    power of two that puts its largest magnitude nearest to 4 .. 6: magnitudes of more than 7 such units take the next one."""
    b = x.float().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)
    e = torch.where(top > 0, e - 3 + (m > 0.875).int(), torch.full_like(e, -125)).clamp(-125, 125)
    y = torch.ldexp(b.abs(), -e)
    code = ((y > 0.25).int() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5)).to(torch.uint8)
    code = code + 8 * torch.signbit(b).to(torch.uint8)
    return code.flatten(-2), (e + 127).squeeze(-1).to(torch.uint8)


def _packed(code):
    return code[..., 0::2] | (code[..., 1::2] << 4)


_GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _values(packed, scale, dtype):
    """What packed codes [..., D / 2] with scale bytes [..., D / 32] stand for."""
    grid = torch.tensor(_GRID + [-g for g in _GRID], dtype=dtype, device=packed.device)
    v = torch.stack([grid[(packed & 15).int()], grid[(packed >> 4).int()]], -1).flatten(-2)
    return torch.ldexp(v.unflatten(-1, (-1, 32)), scale.int().unsqueeze(-1) - 127).flatten(-2)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _normal(gen, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device="cuda:0").to(dtype)


def _prepare_arena(case, gen):
    """Caches as they are in the middle of a generation: rows of 4-bit codes of N(0, 1) values, scores of earlier steps."""
    L, batch, Hkv, D, steps = case["L"], case["batch"], case["Hkv"], case["D"], case["steps"]
    lens = _arena_lens(case)
    cap = lens + (steps if case["kind"] == "generate" else 1)
    off = np.concatenate([[0], np.cumsum(cap)])
    total = int(off[-1])
    dev = torch.device("cuda:0")
    k, v = (torch.empty((total, D // 2), dtype=torch.uint8, device=dev) for _ in range(2))
    scale = torch.empty((total, D // 16), dtype=torch.uint8, device=dev)
    for r in range(0, total, 1 << 18):
        n = min(1 << 18, total - r)
        for plane, at in ((k, 0), (v, D // 32)):
            code, s = _quantized(_normal(gen, n, D))
            plane[r:r + n] = _packed(code)
            scale[r:r + n, at:at + D // 32] = s
    at = torch.arange(total, device=dev)
    pos = (at - torch.repeat_interleave(torch.from_numpy(off[:-1]).to(dev), torch.from_numpy(cap).to(dev))).int()
    st = dict(case=case, lens=lens, off=off, score=torch.rand((total,), generator=gen, device=dev), pos=pos)
    G = case["Hq"] // Hkv
    if own:
        from paper_2502_13176_amd import binding as B
        a = B.Arena(L, case["Hq"], Hkv, D, batch, "mxfp4", _budgets(case), int(cap[0] - lens[0]), SINK, RECENT, B.POLICY_SCORE,
                    case["kind"] == "generate")
        a.k.copy_(k), a.v.copy_(v), a.kv_scale.copy_(scale), a.score.copy_(st["score"]), a.pos.copy_(pos)
        a.set_lengths(lens)
        st["arena"] = a
    else:
        st |= dict(k=k, v=v, scale=scale, len=torch.from_numpy(lens).to(dev).int())
    st["q"] = _normal(gen, steps, L, batch, case["Hq"], D)
    if case["kind"] == "generate":
        st["kn"], st["vn"] = (_normal(gen, steps, L, batch, Hkv, D) for _ in range(2))
    st["out"] = torch.zeros((steps, L, batch, Hkv * G, D), dtype=torch.float32, device=dev)
    return st


def prepare(case, seed):
    kind, D = case["kind"], case["D"]
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    if kind in ("attend", "generate"):
        return _prepare_arena(case, gen)
    Hq, Hkv = case["Hq"], case["Hkv"]
    if kind == "rotate":
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        n = case["n"]
        qkv = _normal(gen, n, Hq + 2 * Hkv, D, dtype=dtype)  # the fused projection's output
        first = torch.randint(0, max(1, case["far"] - n), (1,), generator=gen, device=dev)
        pos = (first + torch.arange(n, device=dev)).int().expand(case["axes"], n).contiguous()
        if case["axes"] == 3:  # the second and third axis count rows and columns of images of 32 x 32 pieces
            pos[1] = pos[1] - pos[0] % 1024 + pos[0] % 1024 // 32
            pos[2] = pos[2] - pos[0] % 1024 + pos[0] % 32
        w = [(1 + 0.2 * torch.randn((D,), generator=gen, device=dev)).to(dtype) if case["norm"] else None for _ in range(2)]
        return dict(case=case, q=qkv[:, :Hq], k=qkv[:, Hq:Hq + Hkv], wq=w[0], wk=w[1], pos=pos, f=_inv_freq(case["rot"]))
    if kind == "prompt":
        lens = _lengths(case, case["T"])
        kv = [t + case["prefix"] for t in lens]
        st = dict(case=case, lens=lens, kv=kv)
        if case["padded"]:
            st["q"] = _normal(gen, len(lens), Hq, max(lens), D)
            st["k"], st["v"] = (_normal(gen, len(lens), Hkv, max(kv), D) for _ in range(2))
        else:
            st["q"] = _normal(gen, sum(lens), Hq, D)
            kv_rows = _normal(gen, sum(kv), 2 * Hkv, D)
            st["k"], st["v"] = kv_rows[:, :Hkv], kv_rows[:, Hkv:]
        return st
    dtype = torch.float32 if case["store"] == "f32" else torch.bfloat16
    lens, L, batch = _lengths(case, case["T"]), case["L"], case["batch"]
    n = sum(lens)
    st = dict(case=case, lens=lens, pos0=[5 * b for b in range(batch)])
    kv = _normal(gen, L, n, 2 * Hkv, D, dtype=dtype)
    st["k"], st["v"] = kv[:, :, :Hkv], kv[:, :, Hkv:]
    st["scores"] = torch.rand((L, Hkv, n), generator=gen, device=dev) if case["scores"] else None
    T = max(1, case["T"])
    total = L * batch * Hkv * T
    if own:
        from paper_2502_13176_amd import binding as B
        a = B.Arena(L, Hq, Hkv, D, batch, case["store"], [min(T, SINK + RECENT)] * (L * Hkv), T - min(T, SINK + RECENT), 0, 0)
        st["arena"] = a
    else:
        st["score"] = torch.zeros((total,), device=dev)
        st["pos"] = torch.zeros((total,), dtype=torch.int32, device=dev)
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _rotated(x, w, st):
    case = st["case"]
    rot = case["rot"]
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6) * w.float()
    f = torch.tensor(st["f"], dtype=torch.float64, device=x.device)
    axis = torch.repeat_interleave(torch.arange(case["axes"], device=x.device), torch.tensor(_sections(case), device=x.device))
    angle = st["pos"][axis].t().double() * f
    c, s = angle.cos().float().unsqueeze(1), angle.sin().float().unsqueeze(1)
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if case["pairs"] else (y[..., :rot // 2], y[..., rot // 2:rot])
    a, b = a * c - b * s, a * s + b * c
    turned = torch.stack([a, b], -1).flatten(-2) if case["pairs"] else torch.cat([a, b], -1)
    return torch.cat([turned, y[..., rot:]], -1).to(x.dtype)


def _sequences(st):
    """Views of every sequence: queries [Hq, t, D], keys and values [Hkv, keys, D], and where its outputs begin."""
    i = j = 0
    for b, (t, n) in enumerate(zip(st["lens"], st["kv"])):
        if st["case"]["padded"]:
            yield b, 0, t, n, st["q"][b, :, :t], st["k"][b, :, :n], st["v"][b, :, :n]
        else:
            yield b, i, t, n, st["q"][i:i + t].transpose(0, 1), st["k"][j:j + n].transpose(0, 1), st["v"][j:j + n].transpose(0, 1)
        i, j = i + t, j + n


def _prompt(st):
    case, q = st["case"], st["q"]
    G = case["Hq"] // case["Hkv"]
    out = torch.zeros_like(q)
    lse = torch.zeros(q.shape[:-1] if case["padded"] else (case["Hq"], q.shape[0]), device=q.device)
    for b, i, t, n, qs, ks, vs in _sequences(st):
        o = out[b, :, :t] if case["padded"] else out[i:i + t].transpose(0, 1)
        ls = lse[b, :, :t] if case["padded"] else lse[:, i:i + t]
        step = max(1, (1 << 28) // (case["Hq"] * n))
        for r in range(0, t, step):
            e = min(t, r + step)
            m = n - t + e  # keys that the last of these tokens sees
            k, v = (x[:, :m].float().repeat_interleave(G, 0) for x in (ks, vs))
            s = qs[:, r:e].float() @ k.transpose(1, 2) * (1 / math.sqrt(case["D"]))
            hidden = torch.arange(m, device=q.device) > torch.arange(n - t + r, m, device=q.device).unsqueeze(1)
            s = s.masked_fill(hidden, -math.inf)
            top = s.amax(-1, keepdim=True)
            p = torch.exp(s - top)
            total = p.sum(-1, keepdim=True)
            o[:, r:e] = (p @ v / total).to(q.dtype)
            ls[:, r:e] = ((top + total.log()) * LOG2E).squeeze(-1)
    return {"out": out, "lse": lse}


def _write(st):
    case = st["case"]
    L, batch, Hkv, D, T = case["L"], case["batch"], case["Hkv"], case["D"], max(1, case["T"])
    rows = []
    for x in (st["k"], st["v"]):
        y = x.transpose(1, 2)  # [L, Hkv, tokens, D]
        if case["store"] == "mxfp4":
            code, s = _quantized(y)
            y = _values(_packed(code), s, torch.float32).to(x.dtype)
        got = torch.zeros((L, batch, Hkv, T, D), dtype=x.dtype, device=x.device)
        i = 0
        for b, t in enumerate(st["lens"]):
            got[:, b, :, T - t:] = y[:, :, i:i + t]
            i += t
        rows.append(got.flatten(0, 2))
    score, pos = st["score"].view(L, batch, Hkv, T), st["pos"].view(L, batch, Hkv, T)
    i = 0
    for b, t in enumerate(st["lens"]):
        score[:, b, :, :t] = st["scores"][:, :, i:i + t] if case["scores"] else 0.0
        pos[:, b, :, :t] = st["pos0"][b] + torch.arange(t, device=pos.device)
        i += t
    live = torch.tensor(st["lens"], dtype=torch.int32, device=pos.device).view(1, batch, 1).expand(L, batch, Hkv).flatten()
    return {"k": rows[0], "v": rows[1], "score": st["score"], "pos": st["pos"], "len": live}


def _attend(st):
    """All steps of a pass, cache by cache: the steps' queries together, each over the rows that it sees."""
    case = st["case"]
    batch, Hkv, D, steps = case["batch"], case["Hkv"], case["D"], case["steps"]
    G, grows, dev = case["Hq"] // Hkv, case["kind"] == "generate", st["q"].device
    new = []
    if grows:  # the rows of all steps, at the end of every cache
        at = torch.from_numpy(st["off"][:-1] + st["lens"]).to(dev).view(-1, 1) + torch.arange(steps, device=dev)
        for plane, x, s0 in ((st["k"], st["kn"], 0), (st["v"], st["vn"], D // 32)):
            code, s = _quantized(x.permute(1, 2, 3, 0, 4).reshape(-1, steps, D))
            plane[at] = _packed(code)
            st["scale"][at.unsqueeze(-1), s0 + torch.arange(D // 32, device=dev)] = s
            new.append(_values(_packed(code), s, torch.float32).to(x.dtype))
        st["pos"][at] = case["ctx"] + torch.arange(steps, dtype=torch.int32, device=dev)
        st["score"][at] = 0.0
    for c, n in enumerate(int(x) for x in st["lens"]):
        layer, b, h = c // (batch * Hkv), c // Hkv % batch, c % Hkv
        o, m = int(st["off"][c]), n + (steps if grows else 0)
        K = _values(st["k"][o:o + m], st["scale"][o:o + m, :D // 32], torch.float32)
        V = _values(st["v"][o:o + m], st["scale"][o:o + m, D // 32:], torch.float32)
        q = st["q"][:, layer, b, h * G:(h + 1) * G].float().reshape(steps * G, D)
        s = q @ K.t() * (1 / math.sqrt(D))
        if grows:
            sees = n + 1 + torch.arange(steps, device=dev).repeat_interleave(G)
            s = s.masked_fill(torch.arange(m, device=dev) >= sees.unsqueeze(1), -math.inf)
        p = torch.exp(s - s.amax(-1, keepdim=True))
        p = p / p.sum(-1, keepdim=True)
        st["out"][:, layer, b, h * G:(h + 1) * G] = (p @ V).view(steps, G, D)
        if grows:
            st["score"][o:o + m] += p.sum(0)
    if not grows:
        return {"out": st["out"]}
    return {"out": st["out"], "score": st["score"], "pos": st["pos"], "len": st["len"] + steps, "k": new[0], "v": new[1]}


def _run_own(st):
    from paper_2502_13176_amd import binding as B
    case = st["case"]
    kind = case["kind"]
    if kind == "rotate":
        q, k = B.qk_norm_rope(st["q"], st["k"], st["pos"], st["f"], q_weight=st["wq"], k_weight=st["wk"], eps=1e-6,
                              sections=_sections(case), interleaved=case["pairs"])
        return {"q": q, "k": k}
    if kind == "prompt":
        if not case["padded"]:
            out, lse = B.prompt_attn(st["q"], st["k"], st["v"], st["lens"], kv_lens=st["kv"], want_lse=True)
            return {"out": out, "lse": lse}
        # outputs of padded places are not written
        out, lse = torch.zeros_like(st["q"]), torch.zeros(st["q"].shape[:-1], device=st["q"].device)
        B.prompt_attn(st["q"], st["k"], st["v"], st["lens"], kv_lens=st["kv"], out=out, lse=lse)
        return {"out": out, "lse": lse}
    a = st["arena"]
    if kind == "write":
        a.reset()
        for layer in range(case["L"]):
            a.append_prompt(layer, st["k"][layer], st["v"][layer], st["lens"], st["pos0"],
                            scores=st["scores"][layer] if case["scores"] else None)
        k, v = a.read_rows(0, case["L"], max(1, case["T"]))
        return {"k": k, "v": v, "score": a.score, "pos": a.pos, "len": a.len}
    ranges = [(0, case["L"])] if case["whole"] else [(layer, 1) for layer in range(case["L"])]
    if kind == "attend":
        for first, n in ranges:
            a.decode_attn(first, n, st["q"][0, first:first + n], st["out"][0, first:first + n])
        return {"out": st["out"]}
    a.set_lengths(st["lens"])  # another continuation of the same prefix
    for t in range(case["steps"]):
        for first, n in ranges:
            at = slice(first, first + n)
            a.append_decode_attn(first, n, st["kn"][t, at], st["vn"][t, at], case["ctx"] + t, st["q"][t, at], st["out"][t, at])
    a.flush_scores(0, case["L"])
    k, v = a.read_rows(0, case["L"], case["steps"])
    return {"out": st["out"], "score": a.score, "pos": a.pos, "len": a.len, "k": k, "v": v}


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "rotate":
        return {"q": _rotated(state["q"], state["wq"], state), "k": _rotated(state["k"], state["wk"], state)}
    if kind == "prompt":
        return _prompt(state)
    if kind == "write":
        return _write(state)
    return _attend(state)


# ---------------------------------------------------------------------------
# the same results in 64 bits
# ---------------------------------------------------------------------------

def _exact_rotate(st):
    case = st["case"]
    half, res = case["rot"] // 2, {}
    first = [2 * i if case["pairs"] else i for i in range(half)]
    second = [2 * i + 1 if case["pairs"] else i + half for i in range(half)]
    axis = [a for a, n in enumerate(_sections(case)) for _ in range(n)]
    turn = torch.polar(torch.ones((case["n"], half), dtype=torch.float64, device=st["q"].device),
                       torch.stack([st["pos"][axis[i]].double() * st["f"][i] for i in range(half)], 1))
    for name, x, w in (("q", st["q"], st["wq"]), ("k", st["k"], st["wk"])):
        y = x.double()
        if w is not None:
            y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / case["D"] + 1e-6) * w.double()
        z = torch.complex(y[..., first], y[..., second]) * turn[:, None]
        y[..., first], y[..., second] = z.real, z.imag
        res[name] = y
    return res


def _exact_prompt(st):
    case, q = st["case"], st["q"]
    G = case["Hq"] // case["Hkv"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.zeros(q.shape[:-1] if case["padded"] else (case["Hq"], q.shape[0]), dtype=torch.float64, device=q.device)
    for b, i, t, n, qs, ks, vs in _sequences(st):
        for h in range(case["Hq"]):
            kd, vd = ks[h // G].double().t().contiguous(), vs[h // G].double()
            for r in range(0, t, 2048):
                e = min(t, r + 2048)
                s = qs[h, r:e].double() @ kd / math.sqrt(case["D"])
                s += torch.full((e - r, n), -math.inf, dtype=torch.float64, device=q.device).triu_(n - t + r + 1)
                z = torch.logsumexp(s, 1)
                o = torch.exp(s - z[:, None]) @ vd
                if case["padded"]:
                    out[b, h, r:e], lse[b, h, r:e] = o, z * LOG2E
                else:
                    out[i + r:i + e, h], lse[h, i + r:i + e] = o, z * LOG2E
    return {"out": out, "lse": lse}


def _exact_attend(st):
    case = st["case"]
    G, Hkv, D, steps = case["Hq"] // case["Hkv"], case["Hkv"], case["D"], case["steps"]
    grows = case["kind"] == "generate"
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device=st["q"].device)
    score = st["score"].double()

    def stored(x):
        code, s = _quantized(x)
        return _values(_packed(code), s, torch.float64)

    for c in range(len(st["lens"])):
        layer, rest = divmod(c, case["batch"] * Hkv)
        b, h = divmod(rest, Hkv)
        o, n = int(st["off"][c]), int(st["lens"][c])
        K, V = st["rows"](o, n)
        if grows:
            K = torch.cat([K, stored(st["kn"][:, layer, b, h])])
            V = torch.cat([V, stored(st["vn"][:, layer, b, h])])
            score[o + n:o + n + steps] = 0
        for t in range(steps):
            m = n + t + 1 if grows else n
            p = torch.softmax(st["q"][t, layer, b, h * G:(h + 1) * G].double() @ K[:m].t() / math.sqrt(D), 1)
            out[t, layer, b, h * G:(h + 1) * G] = p @ V[:m]
            score[o:o + m] += p.sum(0)
    return {"out": out, "score": score, "pos": None, "len": None, "k": None, "v": None} if grows else {"out": out}


def exact(case, seed):
    kind = case["kind"]
    if kind == "write":
        return None  # whole numbers, and values that are stored exactly
    st = prepare(case, seed)
    if kind == "rotate":
        return _exact_rotate(st)
    if kind == "prompt":
        return _exact_prompt(st)
    D = case["D"]
    a = st.get("arena")
    k, v, scale = (a.k, a.v, a.kv_scale) if a is not None else (st["k"], st["v"], st["scale"])
    st["rows"] = lambda o, n: (_values(k[o:o + n], scale[o:o + n, :D // 32], torch.float64),
                               _values(v[o:o + n], scale[o:o + n, D // 32:], torch.float64))
    return _exact_attend(st)
