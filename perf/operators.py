"""Cases for the operators that a decoding loop runs around the draft-tree step.

A model that verifies draft trees keeps the keys and values of each sequence's text in pages of a cache.  Per step it
attends from all nodes of the tree to that cache and to the nodes' own ancestors (`attention`), changes the logits of
every node by what the sequence and the node's path already said, by biases and by a grammar (`logits`), and, once the
step has said which path was accepted, finds room for it (`map`) and stores its keys and values for all layers
(`commit`).

Sizes are those of the benchmark workloads (sequences, nodes, depth, vocabulary) with ordinary head layouts.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}
DEV = "cuda:0"


def listed():
    return [
        # one new token of one short conversation: the smallest call, all latency
        dict(name="attention one token", op="attention", dtype="bf16", B=1, N=1, depth=0, kids=1, hq=32, hkv=8, dim=128,
             page=16, lmin=700, lmax=700),
        # a wide tree of one long conversation (64 nodes, depth 8), seven query heads to a key head
        dict(name="attention long tree", op="attention", dtype="bf16", B=1, N=64, depth=8, kids=4, hq=28, hkv=4, dim=128,
             page=64, lmin=32001, lmax=32001),
        # the largest batch: 256 sequences x 24 nodes over texts of very different length
        dict(name="attention large batch", op="attention", dtype="bf16", B=256, N=24, depth=6, kids=3, hq=32, hkv=8, dim=128,
             page=64, lmin=130, lmax=4100),
        # one key head per query head, small heads, half precision, 16 sequences x 32 nodes
        dict(name="attention small heads", op="attention", dtype="f16", B=16, N=32, depth=6, kids=4, hq=16, hkv=16, dim=64,
             page=16, lmin=1, lmax=8190),
        # single precision throughout (a model checked against a reference), 16 nodes
        dict(name="attention single precision", op="attention", dtype="f32", B=8, N=16, depth=4, kids=3, hq=16, hkv=4, dim=64,
             page=32, lmin=50, lmax=1500),
        # slots for the accepted paths of a large batch, after each step
        dict(name="map after a step", op="map", B=256, width=7, page=16, lmin=100, lmax=8000, nmin=1, nmax=7),
        # pages and slots for a batch of whole prompts
        dict(name="map for prompts", op="map", B=96, width=8192, page=16, lmin=0, lmax=0, nmin=33, nmax=8192),
        # accepted paths of a small batch: 16 sequences, 28 layers
        dict(name="commit small batch", op="commit", dtype="bf16", B=16, N=32, depth=6, kids=4, layers=28, heads=4, dim=128,
             page=16, lmin=100, lmax=900, nmin=1, nmax=4, identity=False),
        # a prompt's keys and values, written whole (every node in order), 32 layers
        dict(name="commit prompts", op="commit", dtype="bf16", B=3, N=509, depth=0, kids=1, layers=32, heads=8, dim=128,
             page=64, lmin=0, lmax=300, nmin=200, nmax=509, identity=True),
        # one sequence, 8 nodes: penalties for repeated tokens only
        dict(name="logits one sequence", op="logits", dtype="f32", B=1, N=8, depth=4, kids=2, V=32000, hist=600, prompt=200,
             bias=0, masks=0),
        # the largest: 256 sequences x 24 nodes, biases, and a grammar for half of the rows
        dict(name="logits large batch", op="logits", dtype="bf16", B=256, N=24, depth=6, kids=3, V=151936, hist=2500, prompt=900,
             bias=16, masks=64),
        # an odd vocabulary (rows that start anywhere), one node per sequence, long texts
        dict(name="logits odd vocabulary", op="logits", dtype="bf16", B=64, N=1, depth=0, kids=1, V=50257, hist=12000, prompt=5000,
             bias=300, masks=7),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "map", "commit", "logits", "logits"])
    depth, kids = rng.randint(1, 8), rng.randint(1, 4)
    N = rng.choice([1, rng.randint(2, 16), rng.randint(17, 64)])
    N = min(N, _tree_size(depth, kids))
    depth = min(depth, N - 1)
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"] if op == "attention" else ["bf16", "bf16", "f32"])
    if op == "attention":
        hkv = rng.choice([1, 2, 4, 8, 16])
        group = rng.choice([1, 2, 4, 7, 8])
        dim = rng.choice([64, 64, 80, 128, 128, 128, 256])
        B, lmax = _log(rng, 1, 256), _log(rng, 1, 40000)
        if dtype == "f32":
            B, lmax, hkv, dim = min(B, 16), min(lmax, 2000), min(hkv, 4), min(dim, 128)
        # no more than the largest listed case: its cache, and its number of scores
        lmax = max(1, min(lmax, 2_000_000_000 // (B * hkv * dim * 2 * BYTES[dtype]), 400_000_000 // (B * hkv * group * N)))
        lmin = rng.randint(max(0, lmax // 20), lmax)
        return dict(op=op, dtype=dtype, B=B, N=N, depth=depth, kids=kids, hq=hkv * group, hkv=hkv, dim=dim,
                    page=rng.choice([16, 16, 32, 48, 64, 128]), lmin=lmin, lmax=lmax)
    if op == "map":
        if rng.random() < 0.6:
            width, lmax = rng.randint(1, 33), _log(rng, 16, 30000)
        else:
            width, lmax = _log(rng, 64, 8192), rng.choice([0, 500])
        B = _log(rng, 1, 1000 if width < 64 else 96)
        return dict(op=op, B=B, width=width, page=rng.choice([16, 16, 32, 48, 64]), lmin=lmax // 10, lmax=lmax,
                    nmin=max(1, width // 9), nmax=width)
    if op == "commit":
        identity = rng.random() < 0.3
        B = rng.randint(1, 4) if identity else _log(rng, 1, 96)
        if identity:
            N, depth, kids = _log(rng, 20, 509), 0, 1
        most = N if identity else depth + 1
        return dict(op=op, dtype=dtype, B=B, N=N, depth=depth, kids=kids, layers=rng.choice([1, 12, 24, 28]),
                    heads=rng.choice([1, 2, 4, 8]), dim=rng.choice([64, 80, 128]), page=rng.choice([16, 32, 64]), lmin=rng.randint(0, 100),
                    lmax=rng.randint(100, 600), nmin=1, nmax=most, identity=identity)
    V = rng.choice([32000, 50257, 128256, 151936, rng.randint(1000, 150000)])
    B = max(1, min(_log(rng, 1, 256), 900_000_000 // (2 * V * N)))
    hist = _log(rng, 1, 16000)
    return dict(op=op, dtype=dtype, B=B, N=N, depth=depth, kids=kids, V=V, hist=hist, prompt=rng.randint(0, hist),
                bias=rng.choice([0, 0, rng.randint(1, 300)]), masks=rng.choice([0, 0, rng.randint(1, 60)]))


# ---- the tree of a case and its lengths -------------------------------------------------------------------------


def _tree_size(depth, kids):
    return sum(kids**d for d in range(depth + 1))


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


# ---- inputs -----------------------------------------------------------------------------------------------------


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rng = np.random.default_rng(seed)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    B = c["B"]
    s = {"case": c}
    if c["op"] in ("attention", "map", "commit"):
        s["len"] = dev(rng.permutation(_spread(c["lmin"], c["lmax"], B)))
    if c["op"] != "map":
        s["parent"] = _parents(c["N"], c["depth"], c["kids"]) if not c.get("identity") else None
    if c["op"] == "attention":
        dt = DTYPES[c["dtype"]]
        hq, hkv, dim, page = c["hq"], c["hkv"], c["dim"], c["page"]
        cols = max(1, -(-c["lmax"] // page))
        need = ((s["len"] + page - 1) // page).cpu().numpy()
        pool = int(need.sum()) + 3
        ids, at = rng.permutation(pool), 0
        table = np.full((B, cols), -1, np.int32)
        for b in range(B):
            table[b, : need[b]] = ids[at : at + need[b]]
            at += need[b]
        s["table"] = dev(table)
        shape = (pool, hkv, page, dim)
        s["cache_k"] = torch.randn(shape, generator=g, device=DEV, dtype=dt)
        s["cache_v"] = torch.randn(shape, generator=g, device=DEV, dtype=dt)
        # one projection's output: queries, keys and values of the nodes side by side
        qkv = torch.randn((B, c["N"], hq + 2 * hkv, dim), generator=g, device=DEV, dtype=dt)
        qkv[:, :, :hq] *= 1.5
        s["q"], s["k"], s["v"] = qkv[:, :, :hq], qkv[:, :, hq : hq + hkv], qkv[:, :, hq + hkv :]
        s["sees"] = dev(_ancestors(s["parent"]))
        if own:
            from paper_2506_04708_b200 import serving

            s["plan"] = serving.TreeAttention(B, c["N"], hq, hkv, dim, dt, page, pool, cols, parent=s["parent"])
    elif c["op"] == "map":
        page = c["page"]
        n = rng.permutation(_spread(c["nmin"], c["nmax"], B)).astype(np.int32)
        lens = s["len"].cpu().numpy()
        have, want = -(-lens // page), -(-(lens + n) // page)
        cols = int(-(-(c["lmax"] + c["nmax"]) // page))
        pool = int((want + 1).sum())
        ids, at = rng.permutation(pool).astype(np.int32), 0
        table = np.full((B, cols), -1, np.int32)
        for b in range(B):
            table[b, : have[b]] = ids[at : at + have[b]]
            at += have[b]
        free = np.full(pool, -1, np.int32)
        free[: pool - at] = ids[at:]
        s["new"], s["table"], s["free"] = dev(n), dev(table), dev(free)
        s["n_free"] = dev(np.array([pool - at], np.int32))
        if own:
            from paper_2506_04708_b200 import serving

            s["plan"] = serving.PageMap(B, c["width"], page, cols, pool)
    elif c["op"] == "commit":
        dt = DTYPES[c["dtype"]]
        L, N, H, dim, page = c["layers"], c["N"], c["heads"], c["dim"], c["page"]
        width = N if c["identity"] else c["depth"] + 1
        lens = s["len"].cpu().numpy()
        n = np.minimum(rng.permutation(_spread(c["nmin"], c["nmax"], B)), width)
        need = -(-(lens + width) // page)
        pool = int(need.sum()) + 2
        ids, at = rng.permutation(pool), 0
        slots, path = np.full((B, width), -1, np.int64), np.full((B, width), -1, np.int32)
        for b in range(B):
            mine = ids[at : at + need[b]]
            at += need[b]
            pos = lens[b] + np.arange(n[b])
            slots[b, : n[b]] = mine[pos // page] * page + pos % page
            path[b, : n[b]] = np.sort(rng.permutation(np.arange(1, N))[: n[b]]) if n[b] < N else np.arange(n[b])
            path[b, 0] = 0
        s["slots"], s["path"], s["n"] = dev(slots), None if c["identity"] else dev(path), dev(n)
        s["k"] = torch.randn((L, B, N, H, dim), generator=g, device=DEV, dtype=dt)
        s["v"] = torch.randn((L, B, N, H, dim), generator=g, device=DEV, dtype=dt)
        s["cache_k"] = torch.randn((L, pool, H, page, dim), generator=g, device=DEV, dtype=dt)
        s["cache_v"] = torch.randn((L, pool, H, page, dim), generator=g, device=DEV, dtype=dt)
        if own:
            from paper_2506_04708_b200 import serving

            s["plan"] = serving.KvCommit(L, B, N, H, dim, dt, page, pool, width)
    else:
        dt = DTYPES[c["dtype"]]
        N, V = c["N"], c["V"]
        s["logits"] = torch.empty((B, N, V), device=DEV, dtype=dt)
        s["logits"].normal_(0.0, 2.5, generator=g)
        lens = rng.permutation(_spread(max(1, c["hist"] // 2), c["hist"], B))
        prompts = np.minimum(lens, c["prompt"])
        # text repeats itself: half of the tokens come from the few that the sequence says often
        text = rng.integers(0, V, (B, c["hist"]))
        often = rng.integers(0, V, (B, 40))
        again = rng.random((B, c["hist"])) < 0.5
        text = np.where(again, np.take_along_axis(often, rng.integers(0, 40, (B, c["hist"])), 1), text).astype(np.int32)
        tree = np.take_along_axis(often, rng.integers(0, 40, (B, N)), 1).astype(np.int32)
        tree[:, 0] = text[np.arange(B), lens - 1]
        s["text"], s["n_text"], s["n_prompt"], s["tree"] = dev(text), dev(lens), dev(prompts), dev(tree)
        s["repetition"] = dev((1.0 + 0.3 * rng.random(B)).astype(np.float32))
        s["frequency"] = dev((0.5 * rng.random(B)).astype(np.float32))
        s["presence"] = dev((0.5 * rng.random(B)).astype(np.float32))
        s["path"] = dev(_ancestors(s["parent"]))
        if c["bias"]:
            k = c["bias"]
            # distinct tokens: one from each k-th of the vocabulary
            ids = (np.arange(k) * (V // k) + rng.integers(0, V // k, (B, k))).astype(np.int32)
            s["bias_start"] = dev((np.arange(B + 1) * k).astype(np.int32))
            s["bias_id"], s["bias_value"] = dev(ids.reshape(-1)), dev(rng.normal(0, 3, B * k).astype(np.float32))
        if c["masks"]:
            # a grammar's state allows between a few and most of the tokens; half of the rows have one
            words = (V + 31) // 32
            m = torch.randint(-(2**31), 2**31, (c["masks"], words), generator=g, device=DEV, dtype=torch.int64)
            m2 = torch.randint(-(2**31), 2**31, (c["masks"], words), generator=g, device=DEV, dtype=torch.int64)
            few = (torch.arange(c["masks"], device=DEV) % 2 == 0)[:, None]
            s["mask"] = torch.where(few, m & m2, m | m2).to(torch.int32)
            pick = rng.integers(0, c["masks"], B * N)
            s["mask_row"] = dev(np.where(rng.random(B * N) < 0.5, pick, -1).astype(np.int32))
        if own:
            from paper_2506_04708_b200 import serving

            s["plan"] = serving.LogitsProcessor(B, N, V, dt, parent=s["parent"])
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------


def run(state):
    s, op = state, state["case"]["op"]
    if own:
        plan = s["plan"]
        if op == "attention":
            return plan(s["q"], s["k"], s["v"], s["cache_k"], s["cache_v"], s["table"], s["len"])
        if op == "map":
            slots, granted, length, n_free = plan(s["len"], s["new"], s["table"], s["free"], s["n_free"])
            return slots, granted, length, n_free, s["table"]
        if op == "commit":
            plan(s["k"], s["v"], s["slots"], s["cache_k"], s["cache_v"], path=s["path"])
            return s["cache_k"], s["cache_v"]
        return plan(s["logits"], s["text"], s["n_text"], n_prompt=s["n_prompt"], tree_tokens=s["tree"], repetition=s["repetition"],
                    frequency=s["frequency"], presence=s["presence"], bias_start=s.get("bias_start"), bias_id=s.get("bias_id"),
                    bias_value=s.get("bias_value"), mask=s.get("mask"), mask_row=s.get("mask_row"))
    return {"attention": _attention, "map": _map, "commit": _commit, "logits": _logits}[op](s)


def _attention(s):
    """softmax(q k^T / sqrt(dim)) v over the pages of the sequence, as far as it is long, and the node's ancestors."""
    c = s["case"]
    B, N, hq, hkv, dim = c["B"], c["N"], c["hq"], c["hkv"], c["dim"]
    span = s["table"].shape[1] * c["page"]
    table = s["table"].clamp(min=0).long()

    def keys(cache, tree):
        past = cache[table].float().transpose(1, 2).reshape(B, hkv, span, dim)
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


def _map(s):
    """Pages for len + new tokens of each sequence, handed out in order, and the slot of each new token."""
    page, width = s["case"]["page"], s["case"]["width"]
    n, new, table = s["len"], s["new"].long(), s["table"]
    cols = table.shape[1]
    have, want = (n + page - 1) // page, (n + new + page - 1) // page
    fits = (new >= 0) & (new <= width) & (want <= cols)
    need = torch.where(fits, want - have, 0)
    upto = torch.cumsum(need, 0)
    served = fits & ((need == 0) | (upto <= s["n_free"]))
    col = torch.arange(cols, device=DEV)[None]
    at = s["n_free"] - 1 - (upto - need)[:, None] - (col - have[:, None])
    fresh = (col >= have[:, None]) & (col < want[:, None]) & served[:, None]
    table = torch.where(fresh, s["free"][at.clamp(0, s["free"].numel() - 1)], table)
    granted = torch.where(served, new, 0)
    j = torch.arange(width, device=DEV)[None]
    pos = n[:, None] + j
    slot = torch.gather(table, 1, (pos // page).clamp(max=cols - 1)).long() * page + pos % page
    slots = torch.where(j < granted[:, None], slot, -1)
    taken = torch.where(served, need, 0).sum()
    return slots, torch.where(served, new, -1).int(), n + granted, (s["n_free"] - taken).int(), table


def _commit(s):
    """Copies the rows of the accepted nodes to their slots.  A place past a path repeats the path's last row."""
    c = s["case"]
    width = s["slots"].shape[1]
    j = torch.minimum(torch.arange(width, device=DEV)[None], s["n"][:, None] - 1)
    slot = torch.gather(s["slots"], 1, j)
    node = j if s["path"] is None else torch.gather(s["path"], 1, j).long()
    b = torch.arange(c["B"], device=DEV)[:, None]
    for_all = (slice(None), slot // c["page"], slice(None), slot % c["page"])
    s["cache_k"][for_all] = s["k"][:, b, node].permute(1, 2, 0, 3, 4)
    s["cache_v"][for_all] = s["v"][:, b, node].permute(1, 2, 0, 3, 4)
    return s["cache_k"], s["cache_v"]


def _logits(s):
    """Repetition, frequency and presence penalties by the text and the node's path, biases, then the grammar."""
    c = s["case"]
    B, N, V = c["B"], c["N"], c["V"]
    x = s["logits"].float()
    place = torch.arange(s["text"].shape[1], device=DEV)[None]
    text = s["text"].long()
    said = torch.zeros((B, V), device=DEV).scatter_add_(1, text, (place < s["n_text"][:, None]).float())
    out = torch.zeros((B, V), device=DEV).scatter_add_(1, text, ((place < s["n_text"][:, None]) & (place >= s["n_prompt"][:, None])).float())
    above = s["path"].clone()
    above[:, 0] = False  # the root is the text's last token: it has been counted
    ids = s["tree"].long()[:, None, :].expand(B, N, N)
    drafted = torch.zeros((B, N, V), device=DEV).scatter_add_(2, ids, above[None].expand(B, N, N).float())
    count = out[:, None] + drafted
    r = s["repetition"][:, None, None]
    x = torch.where(said[:, None] + drafted > 0, torch.where(x > 0, x / r, x * r), x)
    x = x - s["frequency"][:, None, None] * count - s["presence"][:, None, None] * (count > 0)
    if c["bias"]:
        bias = torch.zeros((B, V), device=DEV).scatter_(1, s["bias_id"].view(B, -1).long(), s["bias_value"].view(B, -1))
        x = x + bias[:, None]
    if c["masks"]:
        bits = (s["mask"][:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
        allowed = bits.reshape(c["masks"], -1)[:, :V].bool()
        row = s["mask_row"].view(B, N).long()
        x = torch.where((row >= 0)[..., None] & ~allowed[row.clamp(min=0)], float("-inf"), x)
    return x.to(DTYPES[c["dtype"]])


# ---- what a pass cannot do without ------------------------------------------------------------------------------


def work(case):
    c = case
    B, es = c["B"], BYTES.get(c.get("dtype"), 4)
    if c["op"] == "attention":
        past = int(_spread(c["lmin"], c["lmax"], B).sum())
        sees = int(_ancestors(_parents(c["N"], c["depth"], c["kids"])).sum())
        nodes = B * c["N"] * c["dim"] * es
        read = past * c["hkv"] * c["dim"] * 2 * es + nodes * (c["hq"] + 2 * c["hkv"]) + _pages(c) * 4 + B * 8
        return {"bytes": read + nodes * c["hq"] + B * c["N"] * c["hq"] * 4, "flops": 4 * c["dim"] * c["hq"] * (past * c["N"] + B * sees)}
    if c["op"] == "map":
        lens, new = _spread(c["lmin"], c["lmax"], B), int(_spread(c["nmin"], c["nmax"], B).sum())
        fresh = new // c["page"]
        return {"bytes": B * (8 + 4 + 4) + fresh * 8 + 8 + B * c["width"] * 8 + B * 12, "flops": 0}
    if c["op"] == "commit":
        rows = int(_spread(c["nmin"], c["nmax"], B).sum())
        return {"bytes": rows * c["layers"] * c["heads"] * c["dim"] * es * 2 * 2 + rows * 12, "flops": 0}
    rows = B * c["N"] * c["V"]
    text = int(_spread(max(1, c["hist"] // 2), c["hist"], B).sum())
    masks = min(c["masks"], max(1, B * c["N"] // 2)) * ((c["V"] + 31) // 32) * 4
    return {"bytes": rows * es * 2 + text * 4 + B * c["bias"] * 8 + masks, "flops": rows * 4}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "attention":
        outs, lses = [], []
        group = c["hq"] // c["hkv"]
        for b in range(c["B"]):
            n = int(s["len"][b])
            ids = s["table"][b, : -(-n // c["page"])].long()
            # [heads, tokens, dim] of the text, then of the tree
            ks = [s["cache_k"][ids].permute(1, 0, 2, 3).flatten(1, 2)[:, :n].double(), s["k"][b].transpose(0, 1).double()]
            vs = [s["cache_v"][ids].permute(1, 0, 2, 3).flatten(1, 2)[:, :n].double(), s["v"][b].transpose(0, 1).double()]
            k, v = (torch.cat(t, 1).repeat_interleave(group, 0) for t in (ks, vs))
            z = torch.einsum("uhd,hkd->huk", s["q"][b].double(), k) / math.sqrt(c["dim"])
            z[:, :, n:] += torch.where(s["sees"], 0.0, -math.inf).double()[None]
            lses.append(torch.logsumexp(z, -1).transpose(0, 1))
            outs.append(torch.einsum("huk,hkd->uhd", torch.softmax(z, -1), v))
        return torch.stack(outs), torch.stack(lses)
    if c["op"] == "map":
        return None  # whole numbers: they have to be equal
    if c["op"] == "commit":
        if s["cache_k"].numel() > 200_000_000:
            return None
        got = []
        for cache, rows in ((s["cache_k"], s["k"]), (s["cache_v"], s["v"])):
            cache = cache.double()
            for b in range(c["B"]):
                for j in range(int(s["n"][b])):
                    at, node = int(s["slots"][b, j]), j if s["path"] is None else int(s["path"][b, j])
                    cache[:, at // c["page"], :, at % c["page"]] = rows[:, b, node].double()
            got.append(cache)
        return tuple(got)
    B, N, V = c["B"], c["N"], c["V"]
    if B * N * V > 3_000_000_000:
        return None
    out = torch.empty((B, N, V), dtype=torch.float64, device=DEV)
    text, tree = s["text"].cpu().numpy(), s["tree"].cpu().numpy()
    words = None
    if c["masks"]:
        raw = s["mask"].cpu().numpy().view(np.uint32)
        words = np.unpackbits(raw.view(np.uint8), axis=1, bitorder="little")[:, :V].astype(bool)
        words = torch.from_numpy(words).to(DEV)
    pick = s["mask_row"].cpu().numpy().reshape(B, N) if c["masks"] else None
    for b in range(B):
        n, first = int(s["n_text"][b]), int(s["n_prompt"][b])
        r, f, p = (float(s[k][b]) for k in ("repetition", "frequency", "presence"))
        for u in range(N):
            way, at = [], u
            while at > 0:
                way.append(int(tree[b, at]))
                at = int(s["parent"][at])
            ids, times = np.unique(np.concatenate([text[b, first:n], np.array(way, np.int32)]), return_counts=True)
            ids, times = torch.from_numpy(ids.astype(np.int64)).to(DEV), torch.from_numpy(times).to(DEV).double()
            met = torch.from_numpy(np.unique(np.concatenate([text[b, :n], np.array(way, np.int32)])).astype(np.int64)).to(DEV)
            x = s["logits"][b, u].double()
            x[met] = torch.where(x[met] > 0, x[met] / r, x[met] * r)
            x[ids] -= f * times + p
            if c["bias"]:
                k = c["bias"]
                x[s["bias_id"][b * k : (b + 1) * k].long()] += s["bias_value"][b * k : (b + 1) * k].double()
            if pick is not None and pick[b, u] >= 0:
                x[~words[pick[b, u]]] = -math.inf
            out[b, u] = x
    return out
