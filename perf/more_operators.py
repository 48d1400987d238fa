"""The operators of steps over several drafted tokens whose speed is measured: attention of a tree of drafted tokens over
the ragged caches, verification of the drafted tokens from given random numbers, and the accepted path's rows and scores
into the caches.

Shapes are those of this repository's workloads (`paper_2502_13176_amd/synth.py`), with fewer layers where a full stack would
only repeat the same launches; vocabularies are generic.  Where `own` is false everything is computed with elementary torch
operations, in 32 bits (verification, whose results are whole numbers next to borders, in 64); where it is true by the
library's calls.

Trees: node 0 of a sequence is a token that is decided already, parent[b, i] < i.  A node sees the live rows of a cache, its
ancestors and itself.  The accepted path goes from node 0 to the node behind which the next token is drawn.
"""
import math

import numpy as np
import torch

own = False

LOG2E = 1.4426950408889634
SINK, RECENT = 4, 16


def listed():
    return [
        # one user, four tokens in a row, one layer (latency)
        dict(name="tree_chain_llama_b1", kind="tree", store="bf16", L=1, Hq=32, Hkv=8, D=128, batch=1, N=4, shape="chain", ragged=False, ctx=8192, keep=50, sigma=1.0),
        # a serving batch, trees of up to 32 nodes, one layer
        dict(name="tree_llama_b8", kind="tree", store="bf16", L=1, Hq=32, Hkv=8, D=128, batch=8, N=32, shape="tree", ragged=True, ctx=32768, keep=30, sigma=1.5),
        # the same caches in 4 bits, odd tree, both layers in one call
        dict(name="tree_q4_llama_b8", kind="tree", store="mxfp4", L=2, Hq=32, Hkv=8, D=128, batch=8, N=13, shape="tree", ragged=False, ctx=32768, keep=30, sigma=1.5),
        # a small fp32 model, heads of 64
        dict(name="tree_f32_d64", kind="tree", store="f32", L=1, Hq=16, Hkv=8, D=64, batch=4, N=9, shape="tree", ragged=True, ctx=8192, keep=50, sigma=1.0),
        # the largest: contexts of 131072, trees of 64 nodes, seven query heads to a cache
        dict(name="tree_long_n64", kind="tree", store="bf16", L=1, Hq=28, Hkv=4, D=128, batch=4, N=64, shape="tree", ragged=False, ctx=131072, keep=30, sigma=1.0),
        # one user, a greedy chain (latency)
        dict(name="verify_greedy_b1", kind="verify", dtype="bf16", batch=1, N=5, V=32000, shape="chain", ragged=False, drafts=False, temp="greedy", path=2),
        # a serving batch, chains drawn from a draft model, fp32 logits, odd vocabulary
        dict(name="verify_drafts_b16", kind="verify", dtype="f32", batch=16, N=6, V=100003, shape="chain", ragged=False, drafts=True, temp="one", path=4),
        # a serving batch, trees, every sequence with a temperature of its own
        dict(name="verify_tree_b8", kind="verify", dtype="bf16", batch=8, N=32, V=131072, shape="tree", ragged=True, drafts=False, temp="mixed", path=2),
        # one user's accepted rows into all caches of a model of which nothing ranks rows (latency)
        dict(name="accept_stream_b1", kind="accept", store="bf16", L=32, Hq=32, Hkv=8, D=128, batch=1, N=8, path=4, ctx=2048, keep=30, sigma=1.0, track=False),
        # accepted rows and their scores, four layers of a serving batch
        dict(name="accept_llama_b8", kind="accept", store="bf16", L=4, Hq=32, Hkv=8, D=128, batch=8, N=32, path=5, ctx=32768, keep=30, sigma=1.5, track=True),
        # the same over caches in 4 bits
        dict(name="accept_q4_llama_b8", kind="accept", store="mxfp4", L=4, Hq=32, Hkv=8, D=128, batch=8, N=16, path=5, ctx=32768, keep=30, sigma=1.5, track=True),
        # a whole step: attention of four layers, verification, the accepted rows of all layers
        dict(name="step_llama_b4", kind="step", store="bf16", L=4, Hq=32, Hkv=8, D=128, batch=4, N=16, shape="tree", ctx=32768, keep=30, sigma=1.0, track=True,
             V=32000, path=2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "verify", "verify", "accept", "accept", "step"])
    N = _log(rng, 1, 64)
    shape = rng.choice(["chain", "tree", "tree"])
    if kind == "verify":
        batch = _log(rng, 1, 16)
        drafts = rng.random() < 0.4
        V = _log(rng, 1000, min(160000, (1 << 25) // (batch * N * (2 if drafts else 1))))
        return dict(kind=kind, dtype=rng.choice(["bf16", "f32"]), batch=batch, N=N, V=V, shape="chain" if drafts and rng.random() < 0.7 else shape,
                    ragged=rng.random() < 0.5, drafts=drafts, temp=rng.choice(["greedy", "one", "mixed", "mixed"]), path=min(N, 2))
    Hkv = rng.choice([1, 2, 4, 8])
    D = rng.choice([128, 128, 64])
    store = rng.choice(["bf16", "bf16", "mxfp4", "f32"])
    G = rng.choice([1, 2, 4, 7, 8] + ([16] if D == 128 and store != "f32" else []))
    batch, L = _log(rng, 1, 16), rng.randint(1, 3)
    rows = (1 << 21) // (batch * L * Hkv)  # live rows of a cache, most
    if kind == "tree":
        rows = min(rows, (1 << 27) // (batch * L * Hkv * G * N))
    case = dict(kind=kind, store=store, L=L, Hq=G * Hkv, Hkv=Hkv, D=D, batch=batch, N=N, ctx=_log(rng, 512, max(1024, min(131072, rows))),
                keep=rng.choice([20, 30, 50]), sigma=rng.choice([0.5, 1.0, 1.5]))
    if kind == "tree":
        return dict(case, shape=shape, ragged=rng.random() < 0.5)
    if kind == "accept":
        return dict(case, path=rng.randint(1, min(N, 8)), track=rng.random() < 0.7)
    return dict(case, shape=shape, track=rng.random() < 0.7, V=_log(rng, 1000, 50000), path=min(N, 2))


# ---------------------------------------------------------------------------
# sizes that follow from a case alone
# ---------------------------------------------------------------------------

def _budgets(case):
    """Rows of the cache of every layer and KV head, heavy-tailed, about keep percent of the context on average."""
    m = case["L"] * case["Hkv"]
    rng = np.random.Generator(np.random.PCG64(7))
    w = rng.lognormal(0.0, case["sigma"], m)
    b = case["ctx"] * case["keep"] / 100 * m * w / w.sum()
    return [int(x) for x in np.clip(b, 96, case["ctx"])]


def _cache_lens(case):
    """Live rows of every cache, layer-major, then sequence, then KV head."""
    b = np.asarray(_budgets(case)).reshape(case["L"], 1, case["Hkv"])
    return np.broadcast_to(b, (case["L"], case["batch"], case["Hkv"])).reshape(-1).copy()


def _nodes(case):
    """Nodes of every sequence's tree: the first has the most."""
    if not case.get("ragged"):
        return np.full(case["batch"], case["N"])
    n = np.random.Generator(np.random.PCG64(case["batch"] * 7919 + case["N"])).integers(1, case["N"] + 1, case["batch"])
    n[0] = case["N"]
    return n


def work(case):
    kind, batch, N = case["kind"], case["batch"], case["N"]
    res = {"bytes": 0, "flops": 0}
    if kind in ("verify", "step"):
        # the rows of the nodes that the walk visits, some `path` of a sequence, and of the draft rows tried there
        es = 4 if case.get("dtype") == "f32" else 2
        rows = batch * (case["path"] + (case["path"] if case.get("drafts") else 0))
        res["bytes"] += rows * case["V"] * es
        res["flops"] += 4 * rows * case["V"]
        if kind == "verify":
            return res
    D, G = case["D"], case["Hq"] // case["Hkv"]
    es = 4 if case["store"] == "f32" else 2
    stored = D // 2 + D // 32 if case["store"] == "mxfp4" else D * es  # bytes of a cached row of K or V
    lens = _cache_lens(case).reshape(case["L"], batch, case["Hkv"])
    heads = case["L"] * case["Hkv"]
    if kind in ("tree", "step"):
        nodes = _nodes(case)
        res["bytes"] += int(lens.sum()) * 2 * stored + heads * int(nodes.sum()) * (2 * D * es + G * (2 * D * es + 4))
        res["flops"] += 4 * D * G * int((lens * nodes.reshape(1, -1, 1)).sum())
    if kind in ("accept", "step"):
        rows = heads * batch * case["path"]
        res["bytes"] += rows * (2 * D * es + 2 * stored + 8)
        if case["track"]:
            res["bytes"] += int(lens.sum()) * (stored + 8) + rows * G * (D * es + 4)
            res["flops"] += 2 * D * G * case["path"] * int(lens.sum())
    return res


# ---------------------------------------------------------------------------
# 4-bit rows: D / 2 bytes of E2M1 codes (element 2 i in the low half of byte i), one E8M0 scale for every 32 elements
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


def _as_stored(x, store):
    """Rows as a cache holds them, in their own type."""
    if store != "mxfp4":
        return x
    code, s = _quantized(x)
    return _values(_packed(code), s, torch.float32).to(x.dtype)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _normal(gen, *shape, dtype=torch.bfloat16):
    return torch.randn(shape, generator=gen, device="cuda:0").to(dtype)


def _trees(case, gen):
    """Parents [batch, N]: a chain, or branches of which the earlier nodes have more, as drafted by likelihood."""
    batch, N = case["batch"], case["N"]
    at = torch.arange(N, device="cuda:0")
    if case["shape"] == "chain":
        parent = (at - 1).expand(batch, N)
    else:
        u = torch.rand((batch, N), generator=gen, device="cuda:0")
        parent = (u * u * at).long().clamp(max=N).minimum(at - 1)
    return parent.int().contiguous()


def _prepare_caches(case, gen):
    """Caches in the middle of a generation: rows of N(0, 1) values, scores of earlier steps, room for a tree's longest path."""
    L, batch, Hkv, D, N, store = case["L"], case["batch"], case["Hkv"], case["D"], case["N"], case["store"]
    lens = _cache_lens(case)
    cap = lens + N
    off = np.concatenate([[0], np.cumsum(cap)])
    total = int(off[-1])
    dev = torch.device("cuda:0")
    dtype = torch.float32 if store == "f32" else torch.bfloat16
    st = dict(case=case, lens=lens, off=off)
    k, v = (torch.empty((total, D // 2 if store == "mxfp4" else D), dtype=torch.uint8 if store == "mxfp4" else dtype, device=dev) for _ in range(2))
    scale = torch.empty((total, D // 16), dtype=torch.uint8, device=dev) if store == "mxfp4" else None
    for r in range(0, total, 1 << 18):
        n = min(1 << 18, total - r)
        for plane, at in ((k, 0), (v, D // 32)):
            x = _normal(gen, n, D, dtype=dtype)
            if store == "mxfp4":
                code, s = _quantized(x)
                plane[r:r + n] = _packed(code)
                scale[r:r + n, at:at + D // 32] = s
            else:
                plane[r:r + n] = x
    at = torch.arange(total, device=dev)
    pos = (at - torch.repeat_interleave(torch.from_numpy(off[:-1]).to(dev), torch.from_numpy(cap).to(dev))).int()
    score = torch.rand((total,), generator=gen, device=dev)
    if own:
        from paper_2502_13176_amd import binding as B
        a = B.Arena(L, case["Hq"], Hkv, D, batch, store, _budgets(case), N, SINK, RECENT,
                    B.POLICY_SCORE if case.get("track") else B.POLICY_STREAMING, bool(case.get("track")))
        a.k.copy_(k), a.v.copy_(v), a.score.copy_(score), a.pos.copy_(pos)
        if scale is not None:
            a.kv_scale.copy_(scale)
        a.set_lengths(lens)
        st["arena"] = a
        k, v, scale, score, pos = a.k, a.v, a.kv_scale, a.score, a.pos
    st |= dict(k=k, v=v, scale=scale, score=score, pos=pos, len=torch.from_numpy(lens).to(dev).int())
    # what the projections of all layers gave: queries, keys and values of a node side by side
    G = case["Hq"] // Hkv
    qkv = _normal(gen, L * batch * N, Hkv * (G + 2), D, dtype=dtype)
    st |= dict(q=qkv[:, :Hkv * G], kn=qkv[:, Hkv * G:Hkv * (G + 1)], vn=qkv[:, Hkv * (G + 1):])
    st["pos0"] = torch.full((batch,), case["ctx"], dtype=torch.int32, device=dev)
    return st


def _prepare_logits(case, gen, parent):
    """Logits of a model whose likely next tokens are in part the drafted ones (`path` nodes are accepted on average, node 0
    among them)."""
    batch, N, V = case["batch"], case["N"], case["V"]
    dev = parent.device
    dtype = torch.float32 if case.get("dtype") == "f32" else torch.bfloat16
    x = 2 * torch.randn((batch, N, V), generator=gen, device=dev)
    likely = torch.randint(0, V, (batch, N), generator=gen, device=dev)
    lift = math.log(V) + 2 + 3 * torch.rand((batch, N, 1), generator=gen, device=dev)
    x.scatter_add_(2, likely.unsqueeze(2), lift)
    st = dict(parent=parent, draft=None)
    above = parent.clamp(min=0).long()
    if case.get("drafts"):  # node i's token is drawn from a model that is like the target behind i's parent
        near = torch.gather(x, 1, above.unsqueeze(2).expand(-1, -1, V)) + 0.7 * torch.randn((batch, N, V), generator=gen, device=dev)
        st["draft"] = near.to(dtype)
        race = torch.empty((batch, N, V), device=dev).exponential_(generator=gen)
        token = (st["draft"].float() - race.log()).argmax(2)
    else:  # the first child of a node is its likely token most of the time, the others are anything
        first = torch.ones((batch, N), dtype=torch.bool, device=dev)
        for i in range(1, N):
            first[:, i] = (above[:, 1:i] != above[:, i:i + 1]).all(1)
        hit = first & (torch.rand((batch, N), generator=gen, device=dev) < 0.9)
        token = torch.where(hit, torch.gather(likely, 1, above), torch.randint(0, V, (batch, N), generator=gen, device=dev))
    st["token"] = token.int()
    st["logits"] = x.to(dtype)
    st["u"] = torch.rand((batch, N), generator=gen, device=dev)
    temp = {"greedy": [0.0], "one": [1.0], "mixed": [1.0, 0.7, 0.0, 1.3]}[case.get("temp", "one")]
    st["temp"] = torch.tensor([temp[b % len(temp)] for b in range(batch)], device=dev)
    return st


def prepare(case, seed):
    kind = case["kind"]
    gen = torch.Generator(device=torch.device("cuda:0"))
    gen.manual_seed(seed)
    if kind == "verify":
        st = dict(case=case) | _prepare_logits(case, gen, _trees(case, gen))
        st["nodes"] = torch.from_numpy(_nodes(case)).to("cuda:0").int() if case["ragged"] else None
        return st
    st = _prepare_caches(case, gen)
    batch, N = case["batch"], case["N"]
    if kind == "accept":
        path = torch.arange(N, device="cuda:0").expand(batch, N)
        skip = torch.rand((batch, N), generator=gen, device="cuda:0") * (N - case["path"] + 1)
        # ascending nodes, as a path through a tree is: the first is node 0, the next ones leave some out
        node = (path + skip.sort(1).values.long() * (path > 0)).clamp(max=N - 1)
        st["path"] = torch.where(path < case["path"], node, -1).int().contiguous()
        st["n_path"] = torch.full((batch,), case["path"], dtype=torch.int32, device="cuda:0")
        st["lse"] = _path_lse(st) if case["track"] else None
        return st
    parent = _trees(case, gen)
    if kind == "step":
        st |= _prepare_logits(case, gen, parent)
    st["parent"] = parent
    st["nodes"] = torch.from_numpy(_nodes(case)).to("cuda:0").int() if case.get("ragged") else None
    return st


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _caches(st):
    """Every cache: its number, layer * batch + sequence, KV head, first row, live rows."""
    case = st["case"]
    for c, n in enumerate(int(x) for x in st["lens"]):
        yield c, c // case["Hkv"], c % case["Hkv"], int(st["off"][c]), n


def _rows(st, plane, o, n):
    """n rows of a plane from row o on, in 32 bits."""
    if st["scale"] is None:
        return st[plane][o:o + n].float()
    w = st["scale"].shape[1] // 2
    return _values(st[plane][o:o + n], st["scale"][o:o + n, :w] if plane == "k" else st["scale"][o:o + n, w:], torch.float32)


def _by_head(st, x, s, h, heads):
    """Rows of sequence s (of all layers' sequences) and KV head h: [N, heads, D]."""
    N = st["case"]["N"]
    return x[s * N:(s + 1) * N, h * heads:(h + 1) * heads]


def _seen(parent):
    """[batch, N, N]: whether node i sees node j."""
    batch, N = parent.shape
    seen = torch.eye(N, dtype=torch.bool, device=parent.device).repeat(batch, 1, 1)
    for i in range(1, N):
        p = parent[:, i].long()
        above = torch.gather(seen, 1, p.clamp(0, N - 1).view(-1, 1, 1).expand(-1, 1, N))[:, 0]
        seen[:, i] |= above & ((p >= 0) & (p < i)).unsqueeze(1)
    return seen


def _tree(st):
    case = st["case"]
    L, batch, Hq, Hkv, D, N = (case[x] for x in ("L", "batch", "Hq", "Hkv", "D", "N"))
    G = Hq // Hkv
    out = torch.zeros((L * batch * N, Hq, D), dtype=st["q"].dtype, device=st["q"].device)
    lse = torch.zeros((Hq, L * batch * N), device=out.device)
    hidden = ~_seen(st["parent"])
    kn, vn = _as_stored(st["kn"], case["store"]).float(), _as_stored(st["vn"], case["store"]).float()
    live = (torch.arange(N, device=out.device) < st["nodes"].view(-1, 1)) if st["nodes"] is not None else None
    for c, s, h, o, n in _caches(st):
        q = _by_head(st, st["q"], s, h, G).float().reshape(N * G, D) * (1 / math.sqrt(D))
        own_rows = (q @ _by_head(st, kn, s, h, 1)[:, 0].t()).view(N, G, N).masked_fill(hidden[s % batch].unsqueeze(1), -math.inf)
        x = torch.cat([q @ _rows(st, "k", o, n).t(), own_rows.view(N * G, N)], 1)
        top = x.amax(1, keepdim=True)
        p = torch.exp(x - top)
        total = p.sum(1, keepdim=True)
        res = (p[:, :n] @ _rows(st, "v", o, n) + p[:, n:] @ _by_head(st, vn, s, h, 1)[:, 0]) / total
        at = slice(s * N, (s + 1) * N)
        res, ls = res.view(N, G, D), ((top + total.log()) * LOG2E).view(N, G)
        if live is not None:
            res, ls = res * live[s % batch].view(N, 1, 1), ls * live[s % batch].view(N, 1)
        out[at, h * G:(h + 1) * G] = res.to(out.dtype)
        lse[h * G:(h + 1) * G, at] = ls.t()
    return {"out": out, "lse": lse}


def _distribution(x, temp):
    """softmax(x / temp) of rows [batch, V]; temp 0: all of it on the first of the largest logits."""
    x = torch.nan_to_num(x.double(), nan=-math.inf, posinf=3.4028234663852886e38, neginf=-math.inf)
    top = x.amax(1, keepdim=True)
    e = torch.exp((x - top) / torch.where(temp > 0, temp, torch.ones_like(temp)).double().unsqueeze(1))
    e = torch.where(top > -math.inf, e, torch.zeros_like(e))
    p = e / e.sum(1, keepdim=True).clamp(min=1e-300)
    one = torch.zeros_like(p).scatter_(1, x.argmax(1, keepdim=True), 1.0) * (top > -math.inf)
    return torch.where((temp > 0).unsqueeze(1), p, one)


def _verify(st):
    x, token, parent, u, temp = st["logits"], st["token"].long(), st["parent"], st["u"].double(), st["temp"]
    batch, N, V = x.shape
    at = torch.arange(batch, device=x.device)
    nodes = st.get("nodes")
    cur = torch.zeros_like(at)
    path = torch.full((batch, N), -1, dtype=torch.int32, device=x.device)
    path[:, 0] = 0
    n_path = torch.ones((batch,), dtype=torch.int32, device=x.device)
    r = _distribution(x[:, 0], temp)
    for i in range(1, N):
        tried = parent[:, i] == cur
        if nodes is not None:
            tried = tried & (i < nodes)
        t = token[:, i:i + 1]
        q = torch.zeros_like(r).scatter_(1, t, 1.0)
        if st["draft"] is not None:
            q = torch.where((temp > 0).unsqueeze(1), _distribution(st["draft"][:, i], temp), q)
        good = tried & (u[:, i] * q.gather(1, t)[:, 0] < r.gather(1, t)[:, 0])
        rest = (r - q).clamp(min=0)
        left = rest.sum(1, keepdim=True)
        rest = torch.where(left > 0, rest / left, r)
        r = torch.where(good.unsqueeze(1), _distribution(x[:, i], temp), torch.where(tried.unsqueeze(1), rest, r))
        cur = torch.where(good, i, cur)
        path[at, n_path.long().clamp(max=N - 1)] = torch.where(good, i, path[at, n_path.long().clamp(max=N - 1)].long()).int()
        n_path = n_path + good.int()
    c = r.cumsum(1)
    last = (r > 0).long().mul(torch.arange(1, V + 1, device=x.device)).amax(1) - 1  # (-1: nothing can follow)
    token = (c <= u[:, :1] * c[:, -1:]).sum(1).minimum(last)
    return {"path": path, "n_path": n_path, "next": token.int()}


def _path_rows(st, x, s, h, heads):
    """Rows of the accepted path of sequence s: [path, heads, D], the path padded to N with node 0."""
    return _by_head(st, x, s, h, heads)[st["path"][s % st["case"]["batch"]].clamp(min=0).long()]


def _path_lse(st):
    """log2 of the normalisers of the path's nodes, in the place of every node's [Hq, tokens]."""
    case = st["case"]
    G, N, D, batch = case["Hq"] // case["Hkv"], case["N"], case["D"], case["batch"]
    P = case["path"]
    lse = torch.zeros((case["Hq"], case["L"] * batch * N), device=st["q"].device)
    kn = _as_stored(st["kn"], case["store"]).float()
    for c, s, h, o, n in _caches(st):
        q = _path_rows(st, st["q"], s, h, G)[:P].float().reshape(P * G, D) / math.sqrt(D)
        mine = (q @ _path_rows(st, kn, s, h, 1)[:P, 0].t()).view(P, G, P)
        mine = mine.masked_fill(torch.ones((P, P), dtype=torch.bool, device=q.device).triu(1).unsqueeze(1), -math.inf)
        x = torch.cat([q @ _rows(st, "k", o, n).t(), mine.view(P * G, P)], 1)
        at = s * N + st["path"][s % batch][:P].long()
        lse[h * G:(h + 1) * G, at] = (torch.logsumexp(x, 1) * LOG2E).view(P, G).t()
    return lse


def _accept(st, path, n_path, lse):
    """The path's rows behind the live ones; st keeps its lengths, so that a pass can follow."""
    case = st["case"]
    batch, D, N, store = case["batch"], case["D"], case["N"], case["store"]
    G, dev = case["Hq"] // case["Hkv"], st["q"].device
    st = dict(st, path=path)
    at = torch.arange(N, device=dev)
    got_k, got_v, lens = [], [], []
    for c, s, h, o, n in _caches(st):
        b = s % batch
        on = at < n_path[b]
        rows = o + n + at
        for plane, x, w in (("k", st["kn"], 0), ("v", st["vn"], D // 32)):
            y = _path_rows(st, x, s, h, 1)[:, 0]
            if store == "mxfp4":
                code, sc = _quantized(y)
                st[plane][rows] = torch.where(on.unsqueeze(1), _packed(code), st[plane][rows])
                st["scale"][rows, w:w + D // 32] = torch.where(on.unsqueeze(1), sc, st["scale"][rows, w:w + D // 32])
            else:
                st[plane][rows] = torch.where(on.unsqueeze(1), y, st[plane][rows])
        st["pos"][rows] = torch.where(on, st["pos0"][b] + at.int(), st["pos"][rows])
        new = torch.zeros((N,), device=dev)
        if case["track"]:
            q = _path_rows(st, st["q"], s, h, G).float().reshape(N * G, D) * (1 / math.sqrt(D))
            z = lse[h * G:(h + 1) * G, s * N + path[b].clamp(min=0).long()].t().reshape(N * G, 1) / LOG2E
            p = torch.exp(q @ _rows(st, "k", o, n + N).t() - z).view(N, G, n + N)
            p = p * (on.view(N, 1, 1) & (torch.arange(n + N, device=dev) <= n + at.view(N, 1, 1)))
            p = torch.where(p > 0, p, torch.zeros_like(p)).sum((0, 1))
            st["score"][o:o + n] += p[:n]
            new = p[n:]
        st["score"][rows] = torch.where(on, new, st["score"][rows])
        last = o + n + n_path[b] - N + at  # the cache's last N rows
        for plane, got in (("k", got_k), ("v", got_v)):
            if store == "mxfp4":
                got.append(_values(st[plane][last], st["scale"][last][:, :D // 32] if plane == "k" else st["scale"][last][:, D // 32:], torch.float32).to(st["kn"].dtype))
            else:
                got.append(st[plane][last])
        lens.append(n + n_path[b])
    return {"k": torch.stack(got_k), "v": torch.stack(got_v), "score": st["score"], "pos": st["pos"], "len": torch.stack(lens).int()}


def _run_own(st):
    from paper_2502_13176_amd import binding as B
    case = st["case"]
    kind = case["kind"]
    if kind == "verify":
        path, n_path, token = B.verify_draft(st["logits"], st["token"], st["parent"], st["u"], draft_logits=st["draft"], temperature=st["temp"], n_nodes=st["nodes"])
        return {"path": path, "n_path": n_path, "next": token}
    a, L, batch, N = st["arena"], case["L"], case["batch"], case["N"]
    if kind == "tree":
        if st["nodes"] is None:
            out, lse = a.tree_attn(0, L, st["kn"], st["vn"], st["parent"], st["q"], want_lse=True)
        else:  # places of absent nodes are not written
            out = torch.zeros(st["q"].shape, dtype=st["q"].dtype, device=st["q"].device)
            lse = torch.zeros((case["Hq"], L * batch * N), device=out.device)
            a.tree_attn(0, L, st["kn"], st["vn"], st["parent"], st["q"], n_nodes=st["nodes"], out=out, lse=lse)
        return {"out": out, "lse": lse}
    a.set_lengths(st["lens"])  # another continuation of the same prefix
    res, path, n_path, lse = {}, st.get("path"), st.get("n_path"), st.get("lse")
    if kind == "step":
        out = torch.empty(st["q"].shape, dtype=st["q"].dtype, device=st["q"].device)
        lse = torch.empty((case["Hq"], L * batch * N), device=out.device)
        for layer in range(L):
            at = slice(layer * batch * N, (layer + 1) * batch * N)
            a.tree_attn(layer, 1, st["kn"][at], st["vn"][at], st["parent"], st["q"][at], out=out[at], lse=lse[:, at])
        path, n_path, token = B.verify_draft(st["logits"], st["token"], st["parent"], st["u"], temperature=st["temp"])
        res = {"out": out, "lse": lse, "path": path, "n_path": n_path, "next": token}
    if case["track"]:
        a.append_accepted(0, L, st["kn"], st["vn"], path, n_path, st["pos0"], q=st["q"], lse=lse)
    else:
        a.append_accepted(0, L, st["kn"], st["vn"], path, n_path, st["pos0"])
    k, v = a.read_rows(0, L, N)
    return res | {"k": k, "v": v, "score": a.score, "pos": a.pos, "len": a.len}


def run(state):
    if own:
        return _run_own(state)
    kind = state["case"]["kind"]
    if kind == "tree":
        return _tree(state)
    if kind == "verify":
        return _verify(state)
    if kind == "accept":
        return _accept(state, state["path"], state["n_path"], state["lse"])
    res = _tree(state) | _verify(state)
    return res | _accept(state, res["path"], res["n_path"], res["lse"])


# ---------------------------------------------------------------------------
# the same results in 64 bits
# ---------------------------------------------------------------------------

def _wide(plane, scale, first):
    """Rows of a plane in 64 bits."""
    if scale is None:
        return plane.double()
    w = scale.shape[1] // 2
    return _values(plane, scale[:, first * w:(first + 1) * w], torch.float64)


def _exact_tree(st):
    case, nodes = st["case"], st["nodes"]
    batch, N, D = case["batch"], case["N"], case["D"]
    G, dev = case["Hq"] // case["Hkv"], st["q"].device
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device=dev)
    lse = torch.zeros((case["Hq"], st["q"].shape[0]), dtype=torch.float64, device=dev)
    parent = st["parent"].cpu().tolist()
    kn, vn = (_as_stored(x, case["store"]).double() for x in (st["kn"], st["vn"]))
    for c, n in enumerate(int(x) for x in st["lens"]):
        s, h = divmod(c, case["Hkv"])
        b = s % batch
        o = int(st["off"][c])
        scale = None if st["scale"] is None else st["scale"][o:o + n]
        K, V = _wide(st["k"][o:o + n], scale, 0).t().contiguous(), _wide(st["v"][o:o + n], scale, 1)
        m = N if nodes is None else int(nodes[b])
        mask = torch.full((m, N), -math.inf, dtype=torch.float64)
        for i in range(m):
            j = i
            while j >= 0:
                mask[i, j] = 0.0
                j = parent[b][j]
        mask = mask.to(dev)
        for g in range(h * G, (h + 1) * G):
            q = st["q"][s * N:s * N + m, g].double()
            x = torch.cat([q @ K, q @ kn[s * N:(s + 1) * N, h].t().contiguous() + mask * math.sqrt(D)], 1) / math.sqrt(D)
            z = torch.logsumexp(x, 1)
            p = torch.exp(x - z[:, None])
            out[s * N:s * N + m, g] = p[:, :n] @ V + p[:, n:] @ vn[s * N:(s + 1) * N, h].contiguous()
            lse[g, s * N:s * N + m] = z * LOG2E
    return {"out": out, "lse": lse}


def _exact_scores(st, path, n_path, lse):
    """Scores after the path's rows have come in: weights by the path's own normalisers, one node at a time."""
    case = st["case"]
    batch, N, D = case["batch"], case["N"], case["D"]
    G = case["Hq"] // case["Hkv"]
    score = st["score"].double()
    kn = _as_stored(st["kn"], case["store"]).double()
    for c, n in enumerate(int(x) for x in st["lens"]):
        s, h = divmod(c, case["Hkv"])
        b = s % batch
        o = int(st["off"][c])
        nodes = path[b][:int(n_path[b])].long()
        score[o + n:o + n + len(nodes)] = 0
        if not case["track"]:
            continue
        K = torch.cat([_wide(st["k"][o:o + n], None if st["scale"] is None else st["scale"][o:o + n], 0), kn[s * N + nodes, h]]).t().contiguous()
        for t, i in enumerate(nodes.tolist()):
            q = st["q"][s * N + i, h * G:(h + 1) * G].double()
            seen = n + t + 1
            w = torch.exp2(q @ K[:, :seen].contiguous() * (LOG2E / math.sqrt(D)) - lse[h * G:(h + 1) * G, s * N + i].double()[:, None])
            score[o:o + seen] += w.sum(0)
    return score


def exact(case, seed):
    kind = case["kind"]
    if kind == "verify":
        return None  # whole numbers
    st = prepare(case, seed)
    if kind == "tree":
        return _exact_tree(st)
    none = dict.fromkeys(("k", "v", "score", "pos", "len"))  # (rows are copied, or rounded as a cache stores them)
    if kind == "accept":
        return none | {"score": _exact_scores(st, st["path"], st["n_path"], st["lse"])}
    seen = _exact_tree(st)
    at = _verify(st)
    return seen | dict.fromkeys(("path", "n_path", "next")) | none | {"score": _exact_scores(st, at["path"], at["n_path"], seen["lse"])}
