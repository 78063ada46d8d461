"""Cases for the operators of a paged cache held in 4 bits, and of the position rotation.

A model's keys are normalised per head and rotated by their position (`rotate`); the rows that are to be kept join the
cache, rotated and quantised on the way (`append`, which here also reads back what the cache then holds for them); the
nodes of the draft tree attend to the cache (`attention`).

The 4-bit form: a row's elements in groups of 16, each with a scale s, the smallest float of 5 exponent and 3 fraction
bits (no sign) with 7 s >= the group's largest magnitude; an element is a whole number of -7 .. 7 times s.  A block holds
one head's tokens of one page: the codes (whole number + 8) of all of them, then the scales.

Sizes are those of the benchmark workloads (sequences, nodes, depth) with ordinary head layouts.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
DEV = "cuda:0"
EPS = 1e-6


def listed():
    return [
        # one new token of one short conversation: all latency
        dict(name="attention one token", op="attention", dtype="bf16", B=1, N=1, depth=0, kids=1, hq=32, hkv=8, dim=128,
             page=16, lmin=700, lmax=700),
        # a server without drafts: 64 conversations, one new token each
        dict(name="attention single tokens", op="attention", dtype="bf16", B=64, N=1, depth=0, kids=1, hq=32, hkv=8, dim=128,
             page=16, lmin=500, lmax=8000),
        # a wide tree of one long conversation, seven query heads to a key head
        dict(name="attention long tree", op="attention", dtype="bf16", B=1, N=64, depth=8, kids=4, hq=28, hkv=4, dim=128,
             page=64, lmin=32001, lmax=32001),
        # the largest batch: 256 sequences x 24 nodes over texts of very different length
        dict(name="attention large batch", op="attention", dtype="bf16", B=256, N=24, depth=6, kids=3, hq=32, hkv=8, dim=128,
             page=64, lmin=130, lmax=4100),
        # one key head per query head, small heads, half precision
        dict(name="attention small heads", op="attention", dtype="f16", B=16, N=32, depth=6, kids=4, hq=16, hkv=16, dim=64,
             page=16, lmin=1, lmax=8190),
        # single precision throughout (a model checked against a reference)
        dict(name="attention single precision", op="attention", dtype="f32", B=8, N=16, depth=4, kids=3, hq=16, hkv=4, dim=64,
             page=32, lmin=50, lmax=1500),
        # the smallest: one token's keys and values of one layer into a 16-bit cache, keys rotated on the way
        dict(name="append one token", op="append", dtype="bf16", B=1, N=1, layers=1, heads=8, dim=128, rotary=128, page=16,
             packed=False, lmin=700, lmax=700, nmin=1, nmax=1, tree=False, norm=True, turn=True, pairs=False),
        # accepted paths of a batch, all layers at once, from keys that are rotated already
        dict(name="append accepted paths", op="append", dtype="bf16", B=64, N=24, layers=28, heads=4, dim=128, rotary=128, page=16,
             packed=True, lmin=100, lmax=900, nmin=1, nmax=7, tree=True, norm=False, turn=False, pairs=False),
        # whole prompts of odd lengths from the projection's own rows: norm, rotation and quantisation on the way, 32 layers
        dict(name="append prompts", op="append", dtype="bf16", B=3, N=509, layers=32, heads=8, dim=128, rotary=128, page=64,
             packed=True, lmin=0, lmax=300, nmin=200, nmax=509, tree=False, norm=True, turn=True, pairs=False),
        # the smallest: queries and keys of one token of one layer
        dict(name="rotate one token", op="rotate", dtype="bf16", B=1, N=1, depth=0, hq=32, hkv=8, dim=128, rotary=128,
             lmin=700, lmax=700, norm=True, pairs=False),
        # trees of a batch, half of an odd head size rotated, neighbours in pairs, half precision, far positions
        dict(name="rotate trees in part", op="rotate", dtype="f16", B=64, N=24, depth=6, hq=28, hkv=4, dim=80, rotary=40,
             lmin=130, lmax=900000, norm=False, pairs=True),
        # prompts: one layer's queries and keys of 16,384 tokens
        dict(name="rotate prompts", op="rotate", dtype="bf16", B=4, N=4096, depth=0, hq=32, hkv=8, dim=128, rotary=128,
             lmin=0, lmax=4096, norm=True, pairs=False),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "append", "append", "rotate", "rotate"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    page = rng.choice([16, 16, 32, 48, 64, 128])
    dim = rng.choice([64, 64, 80, 128, 128, 128, 256])
    if op == "attention":
        depth, kids = rng.randint(1, 8), rng.randint(1, 4)
        N = rng.choice([1, 1, rng.randint(2, 16), rng.randint(17, 64)])
        N = min(N, sum(kids**d for d in range(depth + 1)))
        hkv, group = rng.choice([1, 2, 4, 8, 16]), rng.choice([1, 2, 4, 7, 8])
        B, lmax = _log(rng, 1, 256), _log(rng, 1, 40000)
        if dtype == "f32":
            B, lmax, hkv, dim = min(B, 16), min(lmax, 2000), min(hkv, 4), min(dim, 128)
        # no more than the largest listed case: its cache, and its number of scores
        lmax = max(1, min(lmax, 1_000_000_000 // (B * hkv * dim), 400_000_000 // (B * hkv * group * N)))
        return dict(op=op, dtype=dtype, B=B, N=N, depth=min(depth, N - 1), kids=kids, hq=hkv * group, hkv=hkv, dim=dim, page=page,
                    lmin=rng.randint(max(0, lmax // 20), lmax), lmax=lmax)
    turn, pairs = rng.random() < 0.7, rng.random() < 0.3
    rotary = rng.choice([dim, dim, dim, dim // 2])
    if op == "append":
        tree = rng.random() < 0.5
        B = _log(rng, 1, 96) if tree else rng.randint(1, 4)
        N = rng.randint(2, 64) if tree else _log(rng, 1, 509)
        most = rng.randint(1, min(9, N)) if tree else N
        return dict(op=op, dtype=dtype, B=B, N=N, layers=rng.choice([1, 1, 12, 24, 28]), heads=rng.choice([1, 2, 4, 8]), dim=min(dim, 128),
                    rotary=min(rotary, 128), page=page, packed=rng.random() < 0.7, lmin=rng.randint(0, 100), lmax=rng.randint(100, 600),
                    nmin=1, nmax=most, tree=tree, norm=turn and rng.random() < 0.5, turn=turn, pairs=pairs)
    B, N = _log(rng, 1, 256), _log(rng, 1, 4096)
    hkv = rng.choice([1, 2, 4, 8])
    hq = hkv * rng.choice([1, 2, 4, 7])
    N = max(1, min(N, 80_000_000 // (B * (hq + hkv) * dim)))
    lmax = _log(rng, 1, 1000000)
    return dict(op=op, dtype=dtype, B=B, N=N, depth=rng.choice([0, 6]), hq=hq, hkv=hkv, dim=dim, rotary=rotary, lmin=lmax // 2, lmax=lmax,
                norm=rng.random() < 0.6, pairs=pairs)


# ---- the tree of a case and its lengths -------------------------------------------------------------------------


def _parents(N, depth, kids):
    """Breadth-first parent array: the chain down to `depth`, then as many other children as fit, level by level."""
    nodes = {tuple([0] * d) for d in range(depth + 1)}
    level = [()]
    for _ in range(depth):
        level = [p + (r,) for p in level[:N] for r in range(kids)]
        for p in level:
            if len(nodes) < N:
                nodes.add(p)
    order = sorted(nodes, key=lambda p: (len(p), p))
    index = {p: i for i, p in enumerate(order)}
    return np.array([-1] + [index[p[:-1]] for p in order[1:]], np.int32)


def _ancestors(parent):
    """[N, N] truth values: node v is node u or lies above it."""
    N = len(parent)
    a = np.zeros((N, N), bool)
    for u in range(N):
        if u:
            a[u] = a[parent[u]]
        a[u, u] = True
    return a


def _spread(lo, hi, B):
    """B whole numbers from lo to hi, evenly apart (their sum does not go by the seed)."""
    return np.linspace(lo, hi, B).round().astype(np.int64) if B > 1 else np.array([hi], np.int64)


def _pages(c):
    lens = _spread(c["lmin"], c["lmax"], c["B"])
    return int(((lens + c["page"] - 1) // c["page"]).sum())


def _offsets(c, rng):
    """What each node adds to its sequence's position: its depth in a tree, else its place (None)."""
    if c["op"] == "rotate" and not c["depth"] or c["op"] == "append" and not c["tree"]:
        return None
    depth = c.get("depth", 6)
    return np.minimum(np.sort(rng.integers(0, depth + 1, c["N"])), np.arange(c["N"])).astype(np.int32)


# ---- the 4-bit form ---------------------------------------------------------------------------------------------


def _scale_of(byte):
    """The float of 5 exponent and 3 fraction bits: a half without its sign and its last seven bits."""
    s = (byte.to(torch.int16) << 7).view(torch.float16).float()
    return torch.where(byte >= 0xF8, math.nan, s)


def _pack(x):
    """Rows [.., dim] in 32 bits -> codes [.., dim / 2], scales [.., dim / 16], both bytes."""
    g = x.unflatten(-1, (-1, 16))
    least = g.abs().amax(-1).double() / 7
    exponent = torch.where(least > 0, torch.frexp(least)[1] - 1, -14).clamp(min=-14)
    steps = torch.ceil(torch.ldexp(least, 3 - exponent))  # of an eighth of that power of two
    byte = (((exponent + 14) << 3) + steps.to(torch.int32)).clamp(max=0xF7)
    byte = torch.where(torch.isfinite(least), byte, 0xFF).to(torch.uint8)
    s = _scale_of(byte)[..., None]
    code = torch.where(s > 0, torch.round(g / s).clamp(-7, 7), 0.0).to(torch.int32) + 8
    w = code.flatten(-2).unflatten(-1, (-1, 8))
    low, high = w[..., [0, 4, 1, 5]], w[..., [2, 6, 3, 7]]
    return (low | high << 4).to(torch.uint8).flatten(-2), byte


def _unpack(codes, byte):
    """Their values in 32 bits."""
    low, high = (codes & 15).unflatten(-1, (-1, 4)), (codes >> 4).unflatten(-1, (-1, 4))
    w = torch.stack([low[..., 0], low[..., 2], high[..., 0], high[..., 2], low[..., 1], low[..., 3], high[..., 1], high[..., 3]], -1)
    return ((w.flatten(-2).unflatten(-1, (-1, 16)).float() - 8) * _scale_of(byte)[..., None]).flatten(-2)


def _parts(cache, page, dim):
    """Views of a packed cache's codes [.., page, dim / 2] and scales [.., page, dim / 16]."""
    cut = page * dim // 2
    return cache[..., :cut].unflatten(-1, (page, dim // 2)), cache[..., cut:].unflatten(-1, (page, dim // 16))


def _packed_cache(shape, page, dim, g, gain):
    """A cache [.., page * dim * 9 / 16] bytes of normally distributed rows whose elements differ in size."""
    cache = torch.empty(shape + (page * dim * 9 // 16,), dtype=torch.uint8, device=DEV)
    codes, scales = _parts(cache, page, dim)
    step = max(1, 50_000_000 // (int(np.prod(shape[1:])) * page * dim))
    for i in range(0, shape[0], step):
        part = codes[i : i + step]
        x = torch.randn(part.shape[:-1] + (dim,), generator=g, device=DEV) * gain
        codes[i : i + step], scales[i : i + step] = _pack(x.bfloat16().float())
    return cache


# ---- inputs -----------------------------------------------------------------------------------------------------


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    B, N, dim, dt = c["B"], c["N"], c["dim"], DTYPES[c["dtype"]]
    lens = rng.permutation(_spread(c["lmin"], c["lmax"], B))
    s = {"case": c, "len": dev(lens)}
    # keys have a few channels that are much larger than the others
    gain = dev(np.exp(0.5 * rng.normal(size=dim)).astype(np.float32))
    if c["op"] == "attention":
        hq, hkv, page = c["hq"], c["hkv"], c["page"]
        cols = max(1, -(-c["lmax"] // page))
        need = -(-lens // page)
        pool = int(need.sum()) + 3
        ids, at = rng.permutation(pool), 0
        table = np.full((B, cols), -1, np.int32)
        for b in range(B):
            table[b, : need[b]] = ids[at : at + need[b]]
            at += need[b]
        s["table"] = dev(table)
        s["cache_k"] = _packed_cache((pool, hkv), page, dim, g, gain)
        s["cache_v"] = _packed_cache((pool, hkv), page, dim, g, 1.0)
        # one projection's output: queries, keys and values of the nodes side by side
        qkv = torch.randn((B, N, hq + 2 * hkv, dim), generator=g, device=DEV, dtype=dt)
        s["q"], s["k"], s["v"] = qkv[:, :, :hq], qkv[:, :, hq : hq + hkv], qkv[:, :, hq + hkv :]
        s["parent"] = _parents(N, c["depth"], c["kids"])
        s["sees"] = dev(_ancestors(s["parent"]))
        if own:
            from paper_2506_04708_b200 import serving

            s["plan"] = serving.PackedTreeAttention(B, N, hq, hkv, dim, dt, page, pool, cols, parent=s["parent"])
        return s
    offset = _offsets(c, rng)
    s["offset"] = None if offset is None else dev(offset)
    half = c["rotary"] // 2
    s["freq"] = dev((10000.0 ** (-np.arange(half) / half)).astype(np.float32))
    weight = lambda *n: (1 + 0.2 * torch.randn(n, generator=g, device=DEV)).to(dt)  # noqa: E731
    if c["op"] == "rotate":
        hq, hkv = c["hq"], c["hkv"]
        qkv = torch.randn((B, N, hq + 2 * hkv, dim), generator=g, device=DEV, dtype=dt)
        s["q"], s["k"] = qkv[:, :, :hq], qkv[:, :, hq : hq + hkv]
        s["weight_q"], s["weight_k"] = (weight(dim), weight(dim)) if c["norm"] else (None, None)
        if own:
            from paper_2506_04708_b200 import serving

            s["plan"] = serving.HeadRotation(B, N, hq, hkv, dim, dt, freq=s["freq"], offset=s["offset"], interleaved=c["pairs"],
                                             norm=c["norm"], weight_q=s["weight_q"], weight_k=s["weight_k"], eps=EPS)
        return s
    L, H, page, width = c["layers"], c["heads"], c["page"], c["nmax"]
    n = rng.permutation(_spread(c["nmin"], c["nmax"], B))
    need = -(-(lens + width) // page)
    pool = int(need.sum()) + 2
    ids, at = rng.permutation(pool), 0
    slots, path = np.full((B, width), -1, np.int64), np.full((B, width), -1, np.int32)
    for b in range(B):
        mine = ids[at : at + need[b]]
        at += need[b]
        pos = lens[b] + np.arange(n[b])
        slots[b, : n[b]] = mine[pos // page] * page + pos % page
        path[b, : n[b]] = np.sort(rng.permutation(N)[: n[b]])
    s["slots"], s["n"], s["path"] = dev(slots), dev(n), dev(path) if c["tree"] else None
    kv = torch.randn((L, B, N, 2 * H, dim), generator=g, device=DEV, dtype=dt)
    s["k"], s["v"] = kv[:, :, :, :H], kv[:, :, :, H:]
    s["weight_k"] = weight(L, dim) if c["norm"] else None
    for name in ("cache_k", "cache_v"):
        if c["packed"]:
            s[name] = torch.randint(0, 256, (L, pool, H, page * dim * 9 // 16), generator=g, device=DEV, dtype=torch.uint8)
        else:
            s[name] = torch.randn((L, pool, H, page, dim), generator=g, device=DEV, dtype=dt)
    if own:
        from paper_2506_04708_b200 import serving

        s["plan"] = serving.KvAppend(L, B, N, H, dim, dt, page, pool, width, packed=c["packed"], freq=s["freq"] if c["turn"] else None,
                                     offset=s["offset"] if c["turn"] else None, interleaved=c["pairs"], norm=c["norm"], weight_k=s["weight_k"], eps=EPS)
        s["back"] = serving.KvRead(L, B, H, dim, torch.bfloat16, page, pool, width, packed=True) if c["packed"] else None
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------


def run(state):
    s, c = state, state["case"]
    if own:
        if c["op"] == "attention":
            return s["plan"](s["q"], s["k"], s["v"], s["cache_k"], s["cache_v"], s["table"], s["len"])
        if c["op"] == "rotate":
            return s["plan"](s["q"], s["k"], s["len"])
        s["plan"](s["k"], s["v"], s["slots"], s["cache_k"], s["cache_v"], base=s["len"] if c["turn"] else None, path=s["path"])
        return s["back"](s["slots"], s["cache_k"], s["cache_v"]) if c["packed"] else (s["cache_k"], s["cache_v"])
    return {"attention": _attention, "append": _append, "rotate": _rotate}[c["op"]](s)


def _attention(s):
    """softmax(q k^T / sqrt(dim)) v over the pages of the sequence, as far as it is long, and the node's ancestors."""
    c = s["case"]
    B, N, hq, hkv, dim, page = c["B"], c["N"], c["hq"], c["hkv"], c["dim"], c["page"]
    span = s["table"].shape[1] * page
    table = s["table"].clamp(min=0).long()

    def keys(cache, tree):
        past = _unpack(*_parts(cache[table], page, dim)).transpose(1, 2).reshape(B, hkv, span, dim)
        return torch.cat([past, tree.float().transpose(1, 2)], 2)

    k, v = keys(s["cache_k"], s["k"]), keys(s["cache_v"], s["v"])
    q = s["q"].float().view(B, N, hkv, hq // hkv, dim).permute(0, 2, 3, 1, 4).reshape(B, hkv, hq // hkv * N, dim)
    score = torch.matmul(q, k.transpose(2, 3)).view(B, hkv, hq // hkv, N, span + N) * (1.0 / math.sqrt(dim))
    past = torch.arange(span, device=DEV)[None, :] < s["len"][:, None]
    seen = torch.cat([past[:, None, :].expand(B, N, span), s["sees"][None].expand(B, N, N)], 2)
    score = score.masked_fill(~seen[:, None, None], float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, hkv, -1, span + N), v).view(B, hkv, hq // hkv, N, dim) / total
    lse = (top + torch.log(total)).squeeze(-1)
    return out.permute(0, 3, 1, 2, 4).reshape(B, N, hq, dim).to(DTYPES[c["dtype"]]), lse.permute(0, 3, 1, 2).reshape(B, N, hq)


def _normal(x, weight):
    y = x.float()
    return y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * weight.float()


def _turned(y, pos, freq, pairs):
    """Rows [.., heads, dim] turned by pos [..]: angles in 64 bits, they may be far beyond a turn."""
    half = freq.shape[0]
    angle = (pos.double()[..., None] * freq.double())[..., None, :]
    cos, sin = angle.cos().float(), angle.sin().float()
    if pairs:
        a, b = y[..., : 2 * half].unflatten(-1, (half, 2)).unbind(-1)
        turned = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = y[..., :half], y[..., half : 2 * half]
        turned = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([turned, y[..., 2 * half :]], -1)


def _rotate(s):
    """Norm of each head's row, then the turn of its pairs by the token's position."""
    c = s["case"]
    offset = torch.arange(c["N"], device=DEV) if s["offset"] is None else s["offset"]
    pos = s["len"][:, None] + offset[None]
    heads = lambda x, w: _turned(_normal(x, w) if c["norm"] else x.float(), pos, s["freq"], c["pairs"]).to(x.dtype)  # noqa: E731
    return heads(s["q"], s["weight_q"]), heads(s["k"], s["weight_k"])


def _append(s):
    """Rows of the accepted nodes to their slots.  A place past a sequence's tokens repeats its last one; it reads back as zeros."""
    c = s["case"]
    page, dim, dt = c["page"], c["dim"], DTYPES[c["dtype"]]
    width = s["slots"].shape[1]
    j = torch.minimum(torch.arange(width, device=DEV)[None], s["n"][:, None] - 1)
    slot = torch.gather(s["slots"], 1, j)
    node = j if s["path"] is None else torch.gather(s["path"], 1, j).long()
    b = torch.arange(c["B"], device=DEV)[:, None]
    k, v = s["k"][:, b, node], s["v"][:, b, node]  # [layers, B, width, heads, dim]
    if c["norm"]:
        k = _normal(k, s["weight_k"][:, None, None, None])
    if c["turn"]:
        offset = node if s["offset"] is None else s["offset"].long()[node]
        k = _turned(k.float(), s["len"][:, None] + offset, s["freq"], c["pairs"])
    k = k.to(dt)
    for_all = (slice(None), slot // page, slice(None), slot % page)
    got = []
    for cache, x in ((s["cache_k"], k), (s["cache_v"], v)):
        x = x.permute(1, 2, 0, 3, 4)
        if not c["packed"]:
            cache[for_all] = x
            got.append(cache)
            continue
        codes, scales = _parts(cache, page, dim)
        codes[for_all], scales[for_all] = _pack(x.float())
        there = (torch.arange(width, device=DEV)[None] < s["n"][:, None])[..., None, None, None]
        got.append(torch.where(there, _unpack(codes[for_all], scales[for_all]), 0.0).bfloat16().permute(2, 0, 1, 3, 4))
    return tuple(got)


# ---- what a pass cannot do without ------------------------------------------------------------------------------


def work(case):
    c = case
    B, es = c["B"], BYTES[c["dtype"]]
    if c["op"] == "attention":
        past = int(_spread(c["lmin"], c["lmax"], B).sum())
        sees = int(_ancestors(_parents(c["N"], c["depth"], c["kids"])).sum())
        nodes = B * c["N"] * c["dim"] * es
        read = past * c["hkv"] * c["dim"] * 9 // 8 + nodes * (c["hq"] + 2 * c["hkv"]) + _pages(c) * 4 + B * 8
        return {"bytes": read + nodes * c["hq"] + B * c["N"] * c["hq"] * 4, "flops": 4 * c["dim"] * c["hq"] * (past * c["N"] + B * sees)}
    if c["op"] == "rotate":
        rows = B * c["N"] * (c["hq"] + c["hkv"])
        return {"bytes": rows * c["dim"] * es * 2 + B * 8 + c["rotary"] * 2, "flops": rows * (3 * c["rotary"] + (4 * c["dim"] if c["norm"] else 0))}
    rows = int(_spread(c["nmin"], c["nmax"], B).sum())
    values = rows * c["layers"] * c["heads"] * c["dim"] * 2
    padded = B * c["nmax"] * c["layers"] * c["heads"] * c["dim"] * 2
    # packed: read, store, read back, write (padded places too)
    moved = values * es + (values * 9 // 8 + padded * 2 if c["packed"] else values * es)
    return {"bytes": moved + B * c["nmax"] * 8, "flops": values * 4}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------


def _values(block, page, dim):
    """Values in 64 bits of blocks [.., bytes]: element by element from the definition of the form."""
    i = torch.arange(dim, device=DEV)
    place, inside = i // 8 * 4 + (i % 2) * 2 + i % 8 // 4, i % 8 // 2 % 2  # the byte of element i in its row, and which half of it
    token = torch.arange(page, device=DEV)[:, None]
    codes = block[..., (token * (dim // 2) + place).flatten()].long()
    codes = (codes >> (4 * inside).repeat(page)) % 16 - 8
    byte = block[..., (page * dim // 2 + token * (dim // 16) + i // 16).flatten()].long()
    e, f = byte // 8, (byte % 8).double()
    scale = torch.where(e == 0, f / 8 * 2.0**-14, (1 + f / 8) * torch.pow(2.0, (e - 15).double()))
    scale[e == 31] = math.nan
    return (codes * scale).unflatten(-1, (page, dim))


def _nearest(x):
    """What rows [.., dim] are in 4 bits: the best whole number of the smallest sufficient scale."""
    scales = torch.tensor([f / 8 * 2.0**-14 for f in range(8)] + [(1 + f / 8) * 2.0 ** (e - 15) for e in range(1, 31) for f in range(8)],
                          dtype=torch.float64, device=DEV)
    g = x.unflatten(-1, (-1, 16))
    s = scales[torch.searchsorted(scales * 7, g.abs().amax(-1).contiguous()).clamp(max=len(scales) - 1)][..., None]
    whole = torch.round(g / torch.where(s == 0, 1.0, s)).clamp(-7, 7)
    return (whole * s).flatten(-2)


def _exact_rows(x, weight, pos, freq, pairs):
    """x [.., heads, dim], pos [..] or None, in 64 bits, pair by pair as complex numbers."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / y.shape[-1] + EPS) * weight.double()
    if pos is None:
        return y
    n = 2 * freq.shape[0]
    order = torch.arange(n, device=DEV).view(-1, 2) if pairs else torch.arange(n, device=DEV).view(2, -1).T
    z = torch.complex(y[..., order[:, 0]], y[..., order[:, 1]])
    t = pos.double()[..., None, None] * freq.double()
    z = z * torch.polar(torch.ones_like(t), t)
    y = y.clone()
    y[..., order[:, 0]], y[..., order[:, 1]] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    dim, dt = c["dim"], DTYPES[c["dtype"]]
    if c["op"] == "attention":
        outs, lses = [], []
        group, page = c["hq"] // c["hkv"], c["page"]
        for b in range(c["B"]):
            n = int(s["len"][b])
            ids = s["table"][b, : -(-n // page)].long()
            # [heads, tokens, dim] of the text, then of the tree
            past = [_values(cache[ids], page, dim).permute(1, 0, 2, 3).flatten(1, 2)[:, :n] for cache in (s["cache_k"], s["cache_v"])]
            k, v = (torch.cat([p, s[name][b].transpose(0, 1).double()], 1).repeat_interleave(group, 0) for p, name in zip(past, "kv"))
            z = torch.einsum("uhd,hkd->huk", s["q"][b].double(), k) / math.sqrt(dim)
            z[:, :, n:] += torch.where(s["sees"], 0.0, -math.inf).double()[None]
            lses.append(torch.logsumexp(z, -1).transpose(0, 1))
            outs.append(torch.einsum("huk,hkd->uhd", torch.softmax(z, -1), v))
        return torch.stack(outs), torch.stack(lses)
    if c["op"] == "rotate":
        place = torch.arange(c["N"], device=DEV) if s["offset"] is None else s["offset"].long()
        pos = s["len"][:, None] + place
        if s["q"].numel() > 200_000_000:
            return None
        return tuple(_exact_rows(s[n], s["weight_" + n], pos, s["freq"], c["pairs"]) for n in "qk")
    page, width = c["page"], c["nmax"]
    if s["cache_k"].numel() > 400_000_000:
        return None
    got = {}
    for name in "kv":
        cache = None if c["packed"] else s["cache_" + name].double()
        back = torch.zeros((c["layers"], c["B"], width, c["heads"], dim), dtype=torch.float64, device=DEV) if c["packed"] else None
        for b in range(c["B"]):
            n = int(s["n"][b])
            node = torch.arange(n, device=DEV) if s["path"] is None else s["path"][b, :n].long()
            rows = s[name][:, b, node].double()
            if name == "k":
                pos = s["len"][b] + (node if s["offset"] is None else s["offset"].long()[node]) if c["turn"] else None
                w = s["weight_k"][:, None, None] if c["norm"] else None
                rows = _exact_rows(rows, w, pos, s["freq"], c["pairs"])
            if c["packed"]:
                back[:, b, :n] = _nearest(rows.to(dt).double())
            else:
                slot = s["slots"][b, :n]
                cache[:, slot // page, :, slot % page] = rows.transpose(0, 1)
        got[name] = back if c["packed"] else cache
    return got["k"], got["v"]
