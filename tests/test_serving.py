"""The operators around the decoding step: tree attention over a paged cache, page maps, cache commit, logits
processing.  GPU results against plain statements in 64 bits (oracle/serving_ref.py); host-side checks on the CPU.

Tolerances.  u: unit roundoff of the output type (2^-8 bf16, 2^-11 f16, 2^-24 f32).  Attention: the output is rounded
once (u |o|); weights may be rounded to the input type before they multiply the values (u sum p|v|; f16 weights below
2^-14 also lose up to 2^-25 of the largest weight each: 2^-25 sum |v|); scores are fp32 sums of dim products, off by at
most e = (dim + 8) 2^-24 scale max sum |q||k|, which moves every weight by a factor 1 +- 2e; exponentials, sums and the
division are fp32 with fewer than 2^5 roundings that count: 2^-19 sum p|v|.  lse: e plus 2^-19 (1 + |lse|).
Logits: three or four fp32 roundings of values no larger than `size`, then one to the output type.
"""
import ctypes as C
import os

import numpy as np
import pytest

from oracle import serving_ref as ref
from paper_2506_04708_b200 import binding, build as lib_build, inputs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
U = {"bf16": 2.0**-8, "f16": 2.0**-11, "f32": 2.0**-24}


def _dtype(name):
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[name]


# ---------------------------------------------------------------- host side, no GPU
@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return binding.lib()


def test_structures_match_the_header(tmp_path):
    import subprocess
    pairs = [("stand_attention", binding.StandAttention), ("stand_kv_shape", binding.StandKvShape),
             ("stand_logits", binding.StandLogits), ("stand_logits_inputs", binding.StandLogitsInputs)]
    prog = ['#include <stdio.h>', '#include <stddef.h>', '#include "stand.h"', 'int main(void) {']
    for name, st in pairs:
        prog.append(f'printf("%zu\\n", sizeof({name}));')
        prog += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in st._fields_]
    prog += ['return 0; }']
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(prog))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(t) for t in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for _, st in pairs:
        want += [C.sizeof(st)] + [getattr(st, f).offset for f, _ in st._fields_]
    assert got == want


@pytest.mark.parametrize("N,D,kb", [(1, 0, 1), (8, 4, 2), (24, 6, 3), (64, 8, 4), (200, 9, 4)])
def test_tree_mask_names_the_ancestors(lib, N, D, kb):
    parent = inputs.topology(N, D, kb)
    words = (N + 31) // 32
    got = np.zeros((N, words), np.uint32)
    assert lib.stand_tree_mask(parent.ctypes.data, N, got.ctypes.data) == 0
    bits = np.unpackbits(got.view(np.uint8), axis=1, bitorder="little")[:, :N].astype(bool)
    assert np.array_equal(bits, ref.ancestors(parent))
    assert not np.unpackbits(got.view(np.uint8), axis=1, bitorder="little")[:, N:].any()


def test_tree_mask_refuses_what_is_no_tree(lib):
    out = np.zeros((4, 1), np.uint32)
    for bad in ([0, 0, 0, 0], [-1, 1, 0, 0], [-1, 0, 3, 0], [-1, -1, 0, 0]):
        par = np.array(bad, np.int32)
        assert lib.stand_tree_mask(par.ctypes.data, 4, out.ctypes.data) == -1
    par = np.array([-1, 0, 0, 1], np.int32)
    assert lib.stand_tree_mask(None, 4, out.ctypes.data) == -1
    assert lib.stand_tree_mask(par.ctypes.data, 4, None) == -1
    assert lib.stand_tree_mask(par.ctypes.data, 0, out.ctypes.data) == -1
    assert lib.stand_tree_mask(par.ctypes.data, 641, out.ctypes.data) == -1


def _shape(**kw):
    d = dict(B=2, N=8, heads_q=8, heads_kv=2, dim=64, dtype=1, page_size=16, pages=10, max_pages=4, scale=0.125)
    d.update(kw)
    return binding.StandAttention(*[d[n] for n, _ in binding.StandAttention._fields_[:10]])


def test_attention_refuses_invalid_calls(lib):
    size = lib.stand_tree_attention_scratch_bytes
    good = size(C.byref(_shape()))
    assert good > 0
    for bad in (dict(B=0), dict(N=0), dict(N=65537), dict(heads_q=7), dict(heads_kv=0), dict(dim=0), dict(dim=257),
                dict(dtype=3), dict(dtype=-1), dict(page_size=8), dict(page_size=24), dict(page_size=8192), dict(pages=-1),
                dict(max_pages=-1), dict(scale=float("nan"))):
        assert size(C.byref(_shape(**bad))) == 0, bad
    assert size(None) == 0
    a = C.c_void_p(0x100000)  # never touched: every call here is refused before a launch

    def call(shape=_shape(), q=a, k=a, v=a, ck=a, cv=a, table=a, length=a, mask=None, stride=0, scratch=a, n=good, out=a):
        return lib.stand_tree_attention(C.byref(shape), q, k, v, ck, cv, table, length, mask, stride, None, scratch, n, out, None, None)

    for name in ("q", "k", "v", "ck", "cv", "table", "length", "out"):
        assert call(**{name: None}) == -1, name
    assert call(shape=_shape(dim=300)) == -1
    assert call(mask=a, stride=-1) == -1
    assert call(shape=_shape(N=700), mask=a, n=1 << 40) == -1
    assert call(scratch=None) == -2
    assert call(scratch=C.c_void_p(0x100010)) == -2
    assert call(n=good - 1) == -2
    neg = _shape()
    neg.q_stride[1] = -5
    assert call(shape=neg) == -1


def test_paging_and_logits_refuse_invalid_calls(lib):
    a, b = C.c_void_p(0x100000), C.c_void_p(0x200000)

    def page_map(ln=a, new=a, B=2, width=3, page=16, cols=4, free=a, cap=5, nf=a, table=a, slots=a, lo=b, nfo=b):
        return lib.stand_page_map(ln, new, B, width, page, cols, free, cap, nf, table, slots, None, lo, nfo, None)

    for bad in (dict(ln=None), dict(new=None), dict(B=0), dict(width=0), dict(page=0), dict(cols=-1), dict(free=None), dict(cap=-1),
                dict(nf=None), dict(table=None), dict(slots=None), dict(nfo=None), dict(lo=a), dict(nfo=a)):
        assert page_map(**bad) == -1, bad

    def release(ln=a, done=a, B=2, page=16, cols=4, table=a, cap=5, free=a, nf=a, lo=b, nfo=b):
        return lib.stand_page_release(ln, done, B, page, cols, table, cap, free, nf, lo, nfo, None)

    for bad in (dict(ln=None), dict(done=None), dict(B=0), dict(page=0), dict(cols=-1), dict(table=None), dict(cap=-1), dict(free=None),
                dict(nf=None), dict(lo=None), dict(nfo=None), dict(lo=a), dict(nfo=a)):
        assert release(**bad) == -1, bad

    def commit(k=a, v=a, slots=a, ck=b, cv=b, shape=None, **kw):
        d = dict(layers=1, B=1, N=4, heads=2, dim=64, dtype=1, page_size=16, pages=3, width=2, reserved=0)
        d.update(kw)
        s = binding.StandKvShape(*[d[n] for n, _ in binding.StandKvShape._fields_[:10]])
        return lib.stand_kv_commit(C.byref(s), k, v, None, slots, ck, cv, None)

    for bad in (dict(k=None), dict(v=None), dict(slots=None), dict(ck=None), dict(cv=None), dict(layers=0), dict(layers=70000), dict(B=0),
                dict(N=0), dict(heads=0), dict(dim=0), dict(dtype=3), dict(page_size=0), dict(pages=-1), dict(width=0), dict(reserved=1)):
        assert commit(**bad) == -1, bad
    assert lib.stand_kv_commit(None, a, a, None, a, b, b, None) == -1

    parent = np.array([-1, 0, 0, 1], np.int32)
    deep = np.arange(-1, 39, dtype=np.int32)

    def logits(x_in=a, x_out=b, fields=(), par=parent, **kw):
        d = dict(B=2, N=4, V=100, dtype=1, parent=None if par is None else par.ctypes.data, in_stride=100, out_stride=100,
                 text_stride=5, masks=0, biases=0, reserved=0)
        d.update(kw)
        s = binding.StandLogits(*[d[n] for n, _ in binding.StandLogits._fields_])
        x = binding.StandLogitsInputs()
        for f in fields:
            setattr(x, f, 0x100000)
        return lib.stand_process_logits(C.byref(s), C.byref(x), x_in, x_out, None)

    for bad in (dict(x_in=None), dict(x_out=None), dict(B=0), dict(N=0), dict(N=641), dict(V=1), dict(V=(1 << 20) + 1), dict(dtype=2),
                dict(in_stride=99), dict(out_stride=99), dict(text_stride=-1), dict(masks=-1), dict(biases=-1), dict(reserved=1),
                dict(par=None), dict(par=deep, N=40), dict(par=np.array([0, 0, 0, 1], np.int32)),
                dict(par=np.array([-1, 2, 0, 1], np.int32)), dict(x_out=a, out_stride=104), dict(x_in=C.c_void_p(0x100001)),
                dict(fields=["text"]), dict(fields=["n_text"]), dict(fields=["n_prompt"]), dict(fields=["bias_start"], biases=4),
                dict(fields=["mask"]), dict(fields=["mask_row"])):
        assert logits(**bad) == -1, bad


# ---------------------------------------------------------------- attention
def _attention_case(seed, dtype, lens, N, hq, hkv, dim, page, parent=None, mask=None, undrafted=0.0, spare=2, cols=None, nan=True):
    """Device tensors of one call and the same as numpy arrays.  What no row may see holds NaN or inf."""
    import torch
    rng = np.random.default_rng(seed)
    B = len(lens)
    dt = _dtype(dtype)
    need = [-(-max(n, 0) // page) for n in lens]
    cols = max(need + [1]) if cols is None else cols
    pool = sum(need) + spare
    ids = rng.permutation(pool)
    table = rng.choice([-7, 0, pool, 10**9], (B, cols)).astype(np.int32)  # past a sequence's length: anything
    at = 0
    round_ = lambda a: torch.from_numpy(a.astype(np.float32)).to(dt)  # noqa: E731
    ck, cv = (round_(rng.standard_normal((pool, hkv, page, dim))) for _ in range(2))
    for b, n in enumerate(lens):
        table[b, : need[b]] = ids[at: at + need[b]]
        at += need[b]
        if nan and n % page:
            ck[int(table[b, need[b] - 1]), :, n % page:] = float("nan")
            cv[int(table[b, need[b] - 1]), :, n % page:] = float("inf")
    if nan:
        for i in ids[at:]:
            ck[int(i)], cv[int(i)] = float("nan"), float("nan")
    qkv = round_(rng.standard_normal((B, N, hq + 2 * hkv, dim)))
    qkv[:, :, :hq] *= 2
    tree = rng.integers(0, 1000, (B, N)).astype(np.int32)
    if undrafted:
        for b in range(B):
            for u in range(1, N):
                up = parent[u] if parent is not None else u - 1
                if rng.random() < undrafted or tree[b, up] < 0:
                    tree[b, u] = -1
                    if nan:
                        qkv[b, u, hq:hq + hkv], qkv[b, u, hq + hkv:] = float("nan"), float("-inf")
    return dict(qkv=qkv, ck=ck, cv=cv, table=table, len=np.array(lens, np.int64), tree=tree if undrafted else None, parent=parent,
                mask=mask, hq=hq, hkv=hkv, dim=dim, page=page, N=N, dtype=dtype)


def _seen(c):
    N = c["N"]
    if c["parent"] is not None:
        return ref.ancestors(c["parent"])
    if c["mask"] is not None:
        return c["mask"]
    return np.tril(np.ones((N, N), bool))


def _bits(seen):
    N = seen.shape[-1]
    words = (N + 31) // 32
    pad = np.zeros(seen.shape[:-1] + (words * 32,), np.uint8)
    pad[..., :N] = seen
    return np.packbits(pad, axis=-1, bitorder="little").view(np.int32)


def _run_attention(c, stream=None, scale=None, move=None):
    import torch
    from paper_2506_04708_b200 import serving
    dev = "cuda:0"
    B, N, hq, hkv = len(c["len"]), c["N"], c["hq"], c["hkv"]
    qkv, ck, cv = c["qkv"].to(dev), c["ck"].to(dev), c["cv"].to(dev)
    q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
    if move is not None:
        q, k, v, ck, cv = move(q, k, v, ck, cv)
    mask = None if c["mask"] is None else torch.from_numpy(_bits(c["mask"])).to(dev)
    plan = serving.TreeAttention(B, N, hq, hkv, c["dim"], _dtype(c["dtype"]), c["page"], ck.shape[0], c["table"].shape[1], scale=scale,
                                 parent=c["parent"], mask=mask)
    plan.out.fill_(float("nan"))
    plan.lse.fill_(float("nan"))
    tree = None if c["tree"] is None else torch.from_numpy(c["tree"]).to(dev)
    args = (q, k, v, ck, cv, torch.from_numpy(c["table"]).to(dev), torch.from_numpy(c["len"]).to(dev))
    torch.cuda.synchronize()
    out, lse = plan(*args, tree_tokens=tree, stream=stream)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def _reference(c, scale=None):
    x = c["qkv"].double().numpy()
    hq, hkv = c["hq"], c["hkv"]
    s = 1.0 / np.sqrt(c["dim"]) if scale is None else scale
    return ref.attention(x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:], c["ck"].double().numpy(), c["cv"].double().numpy(),
                         c["table"], c["len"], _seen(c), s, c["tree"])


def _check_attention(c, got, want=None, scale=None):
    out, lse = got
    r_out, r_lse, weight, spread, reach = _reference(c, scale) if want is None else want
    u = U[c["dtype"]]
    e = (c["dim"] + 8) * 2.0**-24 * reach
    tol = u * np.abs(r_out) + (u + 2 * e[..., None] + 2.0**-19) * weight + (2.0**-25 * spread if c["dtype"] == "f16" else 0) + 1e-30
    empty = np.isneginf(r_lse)
    assert np.array_equal(np.isneginf(lse), empty)
    assert (out[empty] == 0).all()
    assert np.isfinite(out).all()
    worst = np.max(np.abs(out - r_out) / tol)
    assert worst <= 1.0, worst
    d = np.abs(lse[~empty] - r_lse[~empty])
    assert (d <= (e + 2.0**-19 * (1 + np.abs(r_lse)))[~empty]).all(), d.max()


ALL_TYPES = ["bf16", "f16", "f32"]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
@pytest.mark.parametrize("N,D,kb,hq,hkv,dim,page", [
    (1, 0, 1, 8, 2, 128, 16), (1, 0, 1, 3, 3, 64, 32), (8, 4, 2, 8, 2, 64, 16), (24, 6, 3, 12, 3, 128, 64), (64, 8, 4, 7, 1, 128, 48),
    (13, 4, 3, 6, 2, 80, 16), (33, 6, 4, 5, 1, 96, 128), (9, 4, 2, 4, 2, 256, 16), (40, 6, 4, 4, 1, 192, 32), (5, 2, 2, 2, 1, 8, 16)])
def test_tree_attention_matches_the_definition(dtype, N, D, kb, hq, hkv, dim, page):
    """Lengths around page and tile boundaries, a sequence without text, one with a single token."""
    lens = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 517]
    if N > 30:
        lens = [0, 1, 64, 130, 517]
    c = _attention_case(N * dim, dtype, lens, N, hq, hkv, dim, page, parent=inputs.topology(N, D, kb))
    _check_attention(c, _run_attention(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
@pytest.mark.parametrize("B,length,N,hq,hkv", [(1, 5000, 8, 8, 2), (2, 4097, 64, 7, 1), (1, 9000, 1, 16, 2), (3, 2500, 24, 8, 1)])
def test_long_texts_are_split_and_joined(dtype, B, length, N, hq, hkv):
    """Few rows over long texts: the keys are shared out over the GPU and the pieces joined."""
    parent = inputs.topology(N, min(8, N - 1), 4)
    c = _attention_case(length, dtype, [length - 37 * b for b in range(B)], N, hq, hkv, 128, 16, parent=parent)
    _check_attention(c, _run_attention(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
@pytest.mark.parametrize("N,hq,hkv,dim", [(70, 4, 1, 64), (200, 4, 2, 64), (640, 1, 1, 64), (700, 2, 1, 128), (129, 16, 1, 128)])
def test_chains_and_prompts_without_a_mask(dtype, N, hq, hkv, dim):
    """No mask: node u sees nodes 0..u.  More nodes than a mask may name."""
    c = _attention_case(N, dtype, [0, 33, 150], N, hq, hkv, dim, 16)
    _check_attention(c, _run_attention(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
def test_a_tree_of_the_largest_size(dtype):
    parent = inputs.topology(640, 12, 4)
    c = _attention_case(5, dtype, [70], 640, 1, 1, 64, 16, parent=parent)
    _check_attention(c, _run_attention(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
def test_undrafted_nodes_get_empty_rows(dtype):
    parent = inputs.topology(24, 6, 3)
    c = _attention_case(11, dtype, [0, 100, 64, 700], 24, 8, 2, 128, 16, parent=parent, undrafted=0.4)
    assert (c["tree"] < 0).any()
    _check_attention(c, _run_attention(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
@pytest.mark.parametrize("shared", [True, False])
def test_any_mask_and_rows_that_see_nothing(dtype, shared):
    """Random visibility, some rows empty of nodes: with no text those are empty rows.  Bits above a row's own node
    do not count."""
    rng = np.random.default_rng(3)
    N, lens = 45, [0, 0, 17, 200]
    seen = rng.random((len(lens), N, N)) < 0.3
    seen[:, ::5] = False
    if shared:
        seen = seen[0]
    c = _attention_case(12, dtype, lens, N, 6, 2, 64, 16, mask=seen)
    out, lse = _run_attention(c)
    assert np.isneginf(lse[0, 0]).all()
    _check_attention(c, (out, lse))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
def test_a_value_that_is_not_finite_reaches_only_the_rows_that_see_it(dtype):
    parent = inputs.topology(24, 6, 3)
    c = _attention_case(21, dtype, [0, 90], 24, 4, 2, 64, 16, parent=parent)
    hq, hkv, bad = 4, 2, 5
    clean = _reference(c)
    c["qkv"][:, bad, hq + hkv + 1, 7] = float("inf")   # value head 1, element 7
    c["qkv"][0, bad, hq + hkv, 3] = float("nan")       # value head 0, element 3, first sequence
    out, lse = _run_attention(c)
    below = ref.ancestors(parent)[:, bad]
    assert np.isposinf(out[:, below, 2:, 7]).all() and np.isnan(out[0, below, :2, 3]).all()
    hit = np.zeros_like(out, bool)
    hit[:, below, 2:, 7] = True
    hit[0, below, :2, 3] = True
    assert np.isfinite(out[~hit]).all()
    _check_attention(c, (np.where(hit, clean[0], out), lse), want=clean)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
@pytest.mark.parametrize("how", ["token-major cache", "contiguous nodes", "odd offsets", "padded rows"])
def test_strides_and_alignment(dtype, how):
    """Other layouts of the cache and the nodes; storage that starts off a 16-byte boundary."""
    import torch
    c = _attention_case(31, dtype, [0, 1, 77, 300], 8, 8, 2, 64, 32, parent=inputs.topology(8, 4, 2))

    def move(q, k, v, ck, cv):
        if how == "token-major cache":  # [pages, page, heads, dim]
            return (q, k, v) + tuple(x.transpose(1, 2).contiguous().transpose(1, 2) for x in (ck, cv))
        if how == "contiguous nodes":
            return q.contiguous(), k.contiguous(), v.contiguous(), ck, cv
        if how == "odd offsets":
            def shift(x):
                y = torch.empty(x.numel() + 1, dtype=x.dtype, device=x.device)[1:].view(x.shape)
                return y.copy_(x)
            return tuple(shift(x) for x in (q, k, v, ck, cv))

        def pad(x):  # rows of 3 more elements
            y = torch.empty(x.shape[:-1] + (x.shape[-1] + 3,), dtype=x.dtype, device=x.device)[..., :-3]
            return y.copy_(x)
        return tuple(pad(x) for x in (q, k, v, ck, cv))

    _check_attention(c, _run_attention(c, move=move))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
def test_steep_and_flat_scores(dtype):
    """Scores that grow along the text (the running maximum rises all the time), large ones, and all equal ones."""
    import torch
    c = _attention_case(41, dtype, [400, 700], 8, 4, 1, 64, 16, parent=inputs.topology(8, 4, 2), nan=False)
    for b, n in enumerate(c["len"]):
        for pos in range(n):
            c["ck"][int(c["table"][b, pos // 16]), :, pos % 16] *= 8.0 * pos / n
    _check_attention(c, _run_attention(c))
    want = _reference(c, 1.0)
    _check_attention(c, _run_attention(c, scale=1.0), want=want)
    c["qkv"][:, :, :4] = 0
    _check_attention(c, _run_attention(c))
    c["ck"] = -torch.abs(c["ck"]) - 4  # all scores far below zero
    c["qkv"][:, :, 4] = -6
    c["qkv"][:, :, :4] = 3
    _check_attention(c, _run_attention(c))


@pytest.mark.gpu
def test_lengths_and_tables_out_of_range_do_not_fault():
    """A length below 0 counts as 0, one beyond the table as the table; entries outside the pool read as zeros."""
    for dtype in ALL_TYPES:
        c = _attention_case(51, dtype, [40, 64, 64], 8, 4, 2, 64, 16, parent=inputs.topology(8, 4, 2), nan=False)
        c["len"][:] = [-5, 10**12, 60]
        c["table"][2, 1] = 10**9
        c["table"][2, 2] = -3
        _check_attention(c, _run_attention(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_cache_whose_offsets_pass_32_bits(dtype):
    """Pages at the far end of a pool of more than 2^32 bytes (bf16: more than 2^31 elements)."""
    import torch
    from paper_2506_04708_b200 import serving
    dev, hkv, page, dim = "cuda:0", 8, 16, 128
    per_page = hkv * page * dim
    pool = 2**31 // per_page + 40
    dt = _dtype(dtype)
    small = _attention_case(61, dtype, [130, 257], 8, 16, 8, dim, page, parent=inputs.topology(8, 4, 2), spare=0, nan=False)
    n = small["ck"].shape[0]
    ck, cv = (torch.empty((pool, hkv, page, dim), dtype=dt, device=dev) for _ in range(2))
    ck[-n:], cv[-n:] = small["ck"].to(dev), small["cv"].to(dev)
    table = np.where((small["table"] >= 0) & (small["table"] < n), small["table"] + (pool - n), 0).astype(np.int32)
    qkv = small["qkv"].to(dev)
    plan = serving.TreeAttention(2, 8, 16, 8, dim, dt, page, pool, table.shape[1], parent=small["parent"])
    out, lse = plan(qkv[:, :, :16], qkv[:, :, 16:24], qkv[:, :, 24:], ck, cv, torch.from_numpy(table).to(dev),
                    torch.from_numpy(small["len"]).to(dev))
    _check_attention(small, (out.double().cpu().numpy(), lse.double().cpu().numpy()))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
def test_attention_gives_the_same_bits_every_time_and_on_another_stream(dtype):
    import torch
    c = _attention_case(71, dtype, [3000, 5, 900], 24, 8, 2, 128, 16, parent=inputs.topology(24, 6, 3))
    first = _run_attention(c)
    for stream in (None, torch.cuda.Stream()):
        again = _run_attention(c, stream=stream)
        assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])


@pytest.mark.gpu
def test_attention_binding_refuses_wrong_tensors():
    import torch
    from paper_2506_04708_b200 import serving
    dev = "cuda:0"
    with pytest.raises(binding.StandError):
        serving.TreeAttention(1, 4, 3, 2, 64, torch.bfloat16, 16, 4, 4)
    with pytest.raises(binding.StandError):
        serving.TreeAttention(1, 4, 2, 2, 64, torch.float64, 16, 4, 4)
    plan = serving.TreeAttention(1, 4, 2, 2, 64, torch.bfloat16, 16, 4, 4)
    bf = dict(dtype=torch.bfloat16, device=dev)
    q, cache = torch.zeros((1, 4, 2, 64), **bf), torch.zeros((4, 2, 16, 64), **bf)
    table, length = torch.zeros((1, 4), dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int64, device=dev)
    good = [q, q, q, cache, cache, table, length]
    plan(*good)
    for i, bad in ((0, q.float()), (0, q[:, :2]), (1, q.cpu()), (2, q.transpose(2, 3).contiguous().transpose(2, 3)), (3, cache[:2]),
                   (4, cache.transpose(1, 2).contiguous().transpose(1, 2)), (5, table.long()), (6, length.int())):
        args = list(good)
        args[i] = bad
        with pytest.raises(binding.StandError):
            plan(*args)
    with pytest.raises(binding.StandError):
        plan(*good, tree_tokens=torch.zeros((1, 4), dtype=torch.int64, device=dev))


# ---------------------------------------------------------------- page map, release
def _run_map(length, new, width, page, table, free, n_free, stream=None):
    import torch
    from paper_2506_04708_b200 import serving
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")  # noqa: E731
    plan = serving.PageMap(len(length), width, page, table.shape[1], len(free))
    t = dev(table)
    plan.slots.fill_(-99)
    args = dev(length), dev(new), t, dev(free), dev(np.array([n_free], np.int32))
    torch.cuda.synchronize()
    slots, granted, ln, nf = plan(*args, stream=stream)
    torch.cuda.synchronize()
    return slots.cpu().numpy(), granted.cpu().numpy(), ln.cpu().numpy(), int(nf.item()), t.cpu().numpy()


def _map_case(rng, B, width, page, cols, lmax, spare):
    length = rng.integers(0, lmax + 1, B).astype(np.int64)
    new = rng.integers(0, width + 1, B).astype(np.int32)
    have = -(-length // page)
    pool = int(have.sum()) + spare
    ids, at = rng.permutation(pool).astype(np.int32), 0
    table = np.full((B, cols), -1, np.int32)
    for b in range(B):
        n = min(int(have[b]), cols)
        table[b, :n] = ids[at:at + n]
        at += int(have[b])
    free = np.full(pool, -1, np.int32)
    n_free = pool - at
    free[:n_free] = ids[at:]
    return length, new, table, free, n_free


@pytest.mark.gpu
@pytest.mark.parametrize("B,width,page,cols,lmax", [
    (1, 1, 16, 8, 100), (1, 7, 16, 8, 100), (7, 7, 16, 20, 250), (8, 1, 1, 40, 30), (9, 33, 16, 40, 500), (256, 7, 16, 300, 4000),
    (1000, 5, 32, 40, 1000), (3, 5000, 16, 400, 300), (5, 2049, 48, 60, 100), (2, 256, 16, 40, 300), (2, 257, 16, 40, 300), (300, 300, 7, 90, 200)])
@pytest.mark.parametrize("room", ["plenty", "short", "none"])
def test_page_map_matches_the_serial_statement(B, width, page, cols, lmax, room):
    rng = np.random.default_rng(B * width)
    length, new, table, free, n_free = _map_case(rng, B, width, page, cols, min(lmax, cols * page), 4 + B * (width // page + 2))
    if room == "short":  # the list ends somewhere in the batch
        n_free = max(1, int((-(-(length + new) // page) - -(-length // page)).sum()) // 2)
    elif room == "none":
        n_free = 0
    want = ref.page_map(length, new, width, page, table, free, n_free)
    got = _run_map(length, new, width, page, table, free, n_free)
    for g, w in zip(got, want):
        assert np.array_equal(g, w)


@pytest.mark.gpu
def test_page_map_refuses_single_sequences():
    """Counts outside [0, width], negative lengths and tables that are too small: those sequences alone are refused."""
    length = np.array([10, -3, 20, 60, 5, 2**62, 16, 0], np.int64)
    new = np.array([4, 2, 9, 8, -1, 3, 8, 0], np.int32)
    table = np.arange(8 * 4, dtype=np.int32).reshape(8, 4)
    free = np.arange(100, 120, dtype=np.int32)
    want = ref.page_map(length, new, 8, 16, table, free, 20)
    got = _run_map(length, new, 8, 16, table, free, 20)
    for g, w in zip(got, want):
        assert np.array_equal(g, w)
    assert list(got[1]) == [4, -1, -1, -1, -1, -1, 8, 0]


@pytest.mark.gpu
def test_pages_go_round():
    """Steps of growth and release over a small pool: no page belongs to two sequences, none is lost."""
    import torch
    from paper_2506_04708_b200 import serving
    rng = np.random.default_rng(9)
    B, width, page, cols, pool = 12, 6, 16, 10, 90
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")  # noqa: E731
    plan = serving.PageMap(B, width, page, cols, pool)
    length, table = dev(np.zeros(B, np.int64)), dev(np.full((B, cols), -1, np.int32))
    free, n_free = dev(rng.permutation(pool).astype(np.int32)), dev(np.array([pool], np.int32))
    h = dict(len=np.zeros(B, np.int64), table=table.cpu().numpy(), free=free.cpu().numpy(), n=pool)
    for step in range(150):
        new = rng.integers(0, width + 1, B).astype(np.int32)
        slots, granted, length, n_free = plan(length, dev(new), table, free, n_free)
        w = ref.page_map(h["len"], new, width, page, h["table"], h["free"], h["n"])
        assert np.array_equal(slots.cpu().numpy(), w[0]) and np.array_equal(granted.cpu().numpy(), w[1])
        h["len"], h["n"], h["table"] = w[2], w[3], w[4]
        if step % 7 == 6:
            done = ((rng.random(B) < 0.3) | (h["len"] > 120)).astype(np.int32)
            length, n_free = plan.release(length, dev(done), table, free, n_free)
            h["free"], h["len"], h["n"] = ref.page_release(h["len"], done, page, h["table"], h["free"], h["n"])
        assert np.array_equal(length.cpu().numpy(), h["len"]) and int(n_free.item()) == h["n"]
        assert np.array_equal(free.cpu().numpy()[: h["n"]], h["free"][: h["n"]])
        used = np.concatenate([h["table"][b, : -(-int(h["len"][b]) // page)] for b in range(B)])
        assert sorted(list(used) + list(h["free"][: h["n"]])) == list(range(pool))


# ---------------------------------------------------------------- commit
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
@pytest.mark.parametrize("L,B,N,H,D,page,width", [(1, 1, 1, 1, 64, 16, 1), (3, 4, 24, 2, 128, 16, 7), (28, 2, 8, 8, 128, 64, 5), (2, 3, 9, 3, 7, 5, 4),
                                                  (5, 2, 40, 1, 80, 16, 40), (1, 2, 300, 4, 64, 32, 300)])
@pytest.mark.parametrize("identity", [False, True])
@pytest.mark.parametrize("layout", ["plain", "token-major", "odd"])
def test_commit_copies_the_rows_and_nothing_else(dtype, L, B, N, H, D, page, width, identity, layout):
    import torch
    from paper_2506_04708_b200 import serving
    rng = np.random.default_rng(L * N)
    dt = _dtype(dtype)
    pool = -(-B * width // page) + 3
    make = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(dt).to("cuda:0")  # noqa: E731
    k, v = make(L, B, N, H, D), make(L, B, N, H, D)
    ck, cv = make(L, pool, H, page, D), make(L, pool, H, page, D)
    if layout == "token-major":
        ck, cv = (x.transpose(2, 3).contiguous().transpose(2, 3) for x in (ck, cv))
        k, v = (x.transpose(2, 3).contiguous().transpose(2, 3) for x in (k, v))
    elif layout == "odd":
        k, v, ck, cv = (torch.empty(x.numel() + 1, dtype=dt, device="cuda:0")[1:].view(x.shape).copy_(x) for x in (k, v, ck, cv))
    slots = rng.permutation(pool * page)[: B * width].reshape(B, width).astype(np.int64)
    path = np.sort(rng.integers(0, N, (B, width)), 1).astype(np.int32)
    slots[rng.random((B, width)) < 0.2] = -1
    slots[0, 0] = pool * page        # just outside the pool
    if not identity and width > 1:
        path[-1, -1] = N             # just outside the nodes
        path[-1, 0] = -1
    want = [ref.kv_commit(s.float().cpu().numpy(), None if identity else path, slots, c.float().cpu().numpy()) for s, c in ((k, ck), (v, cv))]
    op = serving.KvCommit(L, B, N, H, D, dt, page, pool, width)
    op(k, v, torch.from_numpy(slots).to("cuda:0"), ck, cv, path=None if identity else torch.from_numpy(path).to("cuda:0"))
    assert np.array_equal(ck.float().cpu().numpy(), want[0]) and np.array_equal(cv.float().cpu().numpy(), want[1])


@pytest.mark.gpu
def test_commit_to_slots_whose_offsets_pass_32_bits():
    import torch
    from paper_2506_04708_b200 import serving
    H, page, D = 8, 16, 128
    pool = 2**31 // (H * page * D) + 5
    ck, cv = (torch.zeros((1, pool, H, page, D), dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    k, v = (torch.randn((1, 1, 4, H, D), device="cuda:0").bfloat16() for _ in range(2))
    slots = torch.tensor([[pool * page - 1, pool * page - 40, 3, -1]], device="cuda:0")
    serving.KvCommit(1, 1, 4, H, D, torch.bfloat16, page, pool, 4)(k, v, slots, ck, cv)
    for cache, src in ((ck, k), (cv, v)):
        assert torch.equal(cache[0, pool - 1, :, 15], src[0, 0, 0]) and torch.equal(cache[0, pool - 3, :, 8], src[0, 0, 1])
        assert torch.equal(cache[0, 0, :, 3], src[0, 0, 2]) and int((cache != 0).any(-1).sum()) == 3 * H


# ---------------------------------------------------------------- logits
def _logits_case(seed, dtype, B, N, V, hist, parts, D=4, kb=3, stride=None):
    import torch
    rng = np.random.default_rng(seed)
    parent = inputs.topology(N, min(D, N - 1), kb)
    x = torch.from_numpy((rng.standard_normal((B, N, V)) * 3).astype(np.float32)).to(_dtype(dtype))
    x[0, 0, : min(V, 3)] = float("-inf")
    x[rng.random(x.shape) < 0.02] = 0.0
    a = {}
    pool = rng.integers(0, V, 12)
    if "text" in parts:
        a["text"] = np.where(rng.random((B, hist)) < 0.5, rng.choice(pool, (B, hist)), rng.integers(0, V, (B, hist))).astype(np.int32)
        a["text"][rng.random((B, hist)) < 0.03] = rng.choice([-1, V, V + 77, -(2**31), 2**31 - 1])
        a["n_text"] = rng.integers(0, hist + 1, B).astype(np.int64)
        a["n_text"][0] = hist
        if B > 1:
            a["n_text"][1] = 0
        if "prompt" in parts:
            a["n_prompt"] = rng.integers(0, hist + 1, B).astype(np.int64)
    if "tree" in parts:
        a["tree"] = rng.choice(np.concatenate([pool, [-1, V - 1]]), (B, N)).astype(np.int32)
    for name, lo, hi in (("repetition", 0.7, 1.6), ("frequency", -0.3, 0.9), ("presence", -0.5, 0.8)):
        if name in parts:
            a[name] = rng.uniform(lo, hi, B).astype(np.float32)
    if "bias" in parts:
        bias = [[(int(t), float(np.float32(w))) for t, w in zip(rng.choice(np.concatenate([pool, rng.integers(0, V, 9), [-4, V]]), n), rng.normal(0, 5, n))]
                for n in rng.integers(0, 20, B)]
        bias[0] += [(int(pool[0]), 2.5), (int(pool[1]), float("-inf")), (int(pool[0]), -1.25)]
        a["bias"] = bias
    if "mask" in parts:
        a["allowed"] = rng.random((4, V)) < np.array([0.0, 0.02, 0.6, 1.0])[:, None]
        a["mask_row"] = rng.choice([-1, 0, 1, 2, 3, 4], (B, N)).astype(np.int32)
    return x, parent, a


def _run_logits(x, parent, a, in_place=False, stride=None, offset=0, stream=None):
    import torch
    from paper_2506_04708_b200 import serving
    dev = lambda n: torch.from_numpy(np.ascontiguousarray(n)).to("cuda:0")  # noqa: E731
    B, N, V = x.shape
    row = stride or V
    store = torch.empty(B * N * row + offset, dtype=x.dtype, device="cuda:0")
    src = store[offset:].view(B, N, row)[..., :V]
    src.copy_(x)
    kw = {("tree_tokens" if k == "tree" else k): dev(v) for k, v in a.items() if k not in ("bias", "allowed")}
    if "bias" in a:
        kw["bias_start"] = dev(np.cumsum([0] + [len(e) for e in a["bias"]]).astype(np.int32))
        kw["bias_id"] = dev(np.array([t for e in a["bias"] for t, _ in e], np.int32))
        kw["bias_value"] = dev(np.array([w for e in a["bias"] for _, w in e], np.float32))
    if "allowed" in a:
        kw["mask"] = dev(_bits_of(a["allowed"]))
    op = serving.LogitsProcessor(B, N, V, x.dtype, parent=parent)
    torch.cuda.synchronize()
    out = op(src, out=src if in_place else None, stream=stream, **kw)
    torch.cuda.synchronize()
    if not in_place:
        assert torch.equal(src.cpu().view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32), x.view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32))
    return out.double().cpu().numpy()


def _bits_of(allowed):
    m, V = allowed.shape
    pad = np.zeros((m, (V + 31) // 32 * 32), np.uint8)
    pad[:, :V] = allowed
    return np.packbits(pad, axis=-1, bitorder="little").view(np.int32)


def _check_logits(x, parent, a, got):
    want, size = ref.process_logits(x.double().numpy(), parent, a.get("text"), a.get("n_text"), a.get("n_prompt"), a.get("tree"),
                                    a.get("repetition"), a.get("frequency"), a.get("presence"), a.get("bias"), a.get("allowed"), a.get("mask_row"))
    u = U["bf16"] if x.element_size() == 2 else U["f32"]
    assert np.array_equal(np.isneginf(got), np.isneginf(want))
    ok = np.isfinite(want)
    tol = u * np.abs(want[ok]) + 8 * 2.0**-24 * size[ok] + 1e-38
    assert (np.abs(got[ok] - want[ok]) <= tol).all(), np.max(np.abs(got[ok] - want[ok]) / tol)


PARTS = [("text", "repetition"), ("text", "prompt", "frequency", "presence"), ("tree", "repetition", "presence", "frequency"), ("bias",), ("mask",),
         ("text", "prompt", "tree", "repetition", "frequency", "presence", "bias", "mask"), ()]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("parts", PARTS, ids=lambda p: "+".join(p) or "nothing")
@pytest.mark.parametrize("in_place", [False, True])
def test_logits_match_the_definition(dtype, parts, in_place):
    for i, (B, N, V, hist) in enumerate([(1, 1, 2, 5), (2, 1, 1000, 30), (3, 8, 4096, 64), (2, 24, 4097, 200), (1, 3, 9001, 1000), (2, 5, 31, 17)]):
        x, parent, a = _logits_case(i, dtype, B, N, V, hist, parts)
        _check_logits(x, parent, a, _run_logits(x, parent, a, in_place))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,stride,offset", [(1003, 1003, 0), (5001, 5007, 0), (2000, 2001, 1), (4100, 4104, 3), (8191, 8192, 8)])
def test_logits_rows_that_start_anywhere(dtype, V, stride, offset):
    for in_place in (False, True):
        x, parent, a = _logits_case(V, dtype, 2, 7, V, 90, PARTS[5])
        _check_logits(x, parent, a, _run_logits(x, parent, a, in_place, stride, offset))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masked_logits_may_hold_anything(dtype):
    import torch
    x, parent, a = _logits_case(77, dtype, 2, 6, 3000, 50, PARTS[5])
    clean = x.clone()
    a["mask_row"][:] = 2
    x[:, :, ~torch.from_numpy(a["allowed"][2])] = float("nan")
    for in_place in (False, True):
        _check_logits(clean, parent, a, _run_logits(x, parent, a, in_place)) if not in_place else None
    got = _run_logits(x, parent, a, True)
    _check_logits(clean, parent, a, got)


@pytest.mark.gpu
def test_logits_a_deep_path_and_a_long_text():
    """A chain as deep as trees may be, its tokens repeated; a text that says one token very often."""
    import torch
    from paper_2506_04708_b200 import serving  # noqa: F401
    V, N = 6000, 33
    parent = np.arange(-1, 32, dtype=np.int32)
    x = torch.randn((2, N, V))
    text = np.full((2, 70001), 17, np.int32)
    text[1, ::2] = 4095
    a = dict(text=text, n_text=np.array([70001, 70000], np.int64), n_prompt=np.array([10, 0], np.int64),
             tree=np.tile(np.array([17, 5, 17, 4096, 5, 9] * 6, np.int32)[:N], (2, 1)), frequency=np.array([0.01, 0.02], np.float32),
             presence=np.array([0.5, 0.25], np.float32), repetition=np.array([1.1, 1.3], np.float32))
    _check_logits(x, parent, a, _run_logits(x, parent, a))


@pytest.mark.gpu
def test_logits_of_more_than_2_to_the_31_elements():
    import torch
    from paper_2506_04708_b200 import serving
    B, N, V = 900, 16, 151936
    parent = inputs.topology(N, 4, 3)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    x = torch.empty((B, N, V), dtype=torch.bfloat16, device="cuda:0").normal_(0, 2, generator=g)
    text = torch.randint(0, V, (B, 50), dtype=torch.int32, device="cuda:0", generator=g)
    n = torch.full((B,), 50, dtype=torch.int64, device="cuda:0")
    pres = torch.full((B,), 0.5, device="cuda:0")
    out = serving.LogitsProcessor(B, N, V, torch.bfloat16, parent=parent)(x, text, n, presence=pres)
    for b in (0, 449, 899):
        want = x[b].float()
        want[:, text[b].long().unique()] -= 0.5
        assert torch.equal(out[b], want.bfloat16())


@pytest.mark.gpu
def test_logits_binding_refuses_wrong_tensors():
    import torch
    from paper_2506_04708_b200 import serving
    with pytest.raises(binding.StandError):
        serving.LogitsProcessor(1, 4, 100, torch.float16, parent=[-1, 0, 0, 0])
    with pytest.raises(binding.StandError):
        serving.LogitsProcessor(1, 4, 100, torch.float32)
    op = serving.LogitsProcessor(2, 4, 100, torch.float32, parent=[-1, 0, 0, 1])
    x = torch.zeros((2, 4, 100), device="cuda:0")
    f = torch.zeros(2, device="cuda:0")
    op(x, presence=f)
    for bad in (x.bfloat16(), x[:1], x.cpu(), x.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(binding.StandError):
            op(bad)
    for kw in (dict(presence=f.double()), dict(text=torch.zeros((2, 3), dtype=torch.int32, device="cuda:0")), dict(n_text=torch.zeros(2, dtype=torch.int64, device="cuda:0")),
               dict(bias_start=torch.zeros(3, dtype=torch.int32, device="cuda:0")), dict(mask=torch.zeros((1, 4), dtype=torch.int32, device="cuda:0")),
               dict(tree_tokens=torch.zeros((2, 5), dtype=torch.int32, device="cuda:0"))):
        with pytest.raises(binding.StandError):
            op(x, **kw)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,dim", [("bf16", 128), ("f16", 64), ("bf16", 256)])
def test_a_wait_that_runs_out_gives_nan_and_leaves_the_gpu_usable(dtype, dim):
    """The safe form: every wait of the kernel gives up before anything was copied.  The next call is right again."""
    c = _attention_case(81, dtype, [0, 700, 64], 8, 8, 2, dim, 16, parent=inputs.topology(8, 4, 2))
    binding.set_wait_limit(0)
    try:
        out, lse = _run_attention(c)
    finally:
        binding.set_wait_limit(-1)
    assert np.isnan(out).all() and np.isnan(lse).all()
    _check_attention(c, _run_attention(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
@pytest.mark.parametrize("B", [193, 700])
def test_batches_of_more_sequences_than_threads(dtype, B):
    """Many short texts, among them empty ones: a range of tiles covers dozens of sequences."""
    rng = np.random.default_rng(B)
    lens = [int(n) for n in np.where(rng.random(B) < 0.2, 0, rng.integers(1, 90, B))]
    lens[B // 2] = 1200
    c = _attention_case(B, dtype, lens, 3, 4, 2, 64, 16, parent=inputs.topology(3, 2, 2), nan=False)
    _check_attention(c, _run_attention(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
@pytest.mark.parametrize("N,hq,hkv,dim,page", [(1, 130, 1, 64, 16), (2, 300, 2, 128, 32), (3, 4, 2, 20, 16), (9, 6, 3, 36, 16), (4, 2, 1, 7, 48), (5, 128, 1, 128, 64)])
def test_head_layouts_beside_the_common_ones(dtype, N, hq, hkv, dim, page):
    """More query heads to a key head than a tile has rows; head sizes that are no multiple of 8."""
    c = _attention_case(N * hq, dtype, [0, 5, 70, 200], N, hq, hkv, dim, page, parent=inputs.topology(N, min(2, N - 1), 3))
    _check_attention(c, _run_attention(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
def test_no_cache_at_all_and_pages_of_the_largest_size(dtype):
    import torch
    from paper_2506_04708_b200 import serving
    c = _attention_case(5, dtype, [0, 0], 70, 4, 2, 64, 16)
    qkv = c["qkv"].to("cuda:0")
    none = torch.empty((0, 2, 16, 64), dtype=_dtype(dtype), device="cuda:0")
    plan = serving.TreeAttention(2, 70, 4, 2, 64, _dtype(dtype), 16, 0, 0)
    out, lse = plan(qkv[:, :, :4], qkv[:, :, 4:6], qkv[:, :, 6:], none, none, torch.empty((2, 0), dtype=torch.int32, device="cuda:0"),
                    torch.zeros(2, dtype=torch.int64, device="cuda:0"))
    _check_attention(c, (out.double().cpu().numpy(), lse.double().cpu().numpy()))
    c = _attention_case(6, dtype, [3000, 4096, 4097], 5, 4, 2, 64, 4096, parent=inputs.topology(5, 2, 2))
    _check_attention(c, _run_attention(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ALL_TYPES)
def test_broadcast_keys_and_queries(dtype):
    """Strides of zero: one key head's rows for all heads, one query row for all heads."""
    import torch
    c = _attention_case(91, dtype, [0, 130], 8, 8, 4, 64, 16, parent=inputs.topology(8, 4, 2), nan=False)
    x = c["qkv"]
    x[:, :, :8] = x[:, :, :1]
    x[:, :, 8:12] = x[:, :, 8:9]
    x[:, :, 12:] = x[:, :, 12:13]

    def move(q, k, v, ck, cv):
        wide = lambda t, n: t[:, :, :1].contiguous().expand(-1, -1, n, -1)  # noqa: E731
        return wide(q, 8), wide(k, 4), wide(v, 4), ck, cv

    _check_attention(c, _run_attention(c, move=move))


@pytest.mark.gpu
def test_operators_in_a_graph_follow_the_lengths():
    """Captured once, replayed after lengths, counts and texts have changed in place."""
    import torch
    from paper_2506_04708_b200 import serving
    c = _attention_case(95, "bf16", [600, 40, 333], 24, 8, 2, 128, 16, parent=inputs.topology(24, 6, 3), nan=False)
    dev = "cuda:0"
    qkv, ck, cv = c["qkv"].to(dev), c["ck"].to(dev), c["cv"].to(dev)
    table, length = torch.from_numpy(np.clip(c["table"], 0, ck.shape[0] - 1)).to(dev), torch.from_numpy(c["len"]).to(dev)
    c["table"] = table.cpu().numpy()
    plan = serving.TreeAttention(3, 24, 8, 2, 128, torch.bfloat16, 16, ck.shape[0], table.shape[1], parent=c["parent"])
    args = (qkv[:, :, :8], qkv[:, :, 8:10], qkv[:, :, 10:], ck, cv, table, length)
    x = torch.randn((3, 1, 5000), device=dev)
    text = torch.randint(0, 5000, (3, 300), dtype=torch.int32, device=dev)
    n_text, presence = torch.full((3,), 300, dtype=torch.int64, device=dev), torch.full((3,), 0.5, device=dev)
    op = serving.LogitsProcessor(3, 1, 5000, torch.float32)
    plan(*args)
    op(x, text, n_text, presence=presence)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, lse = plan(*args)
        y = op(x, text, n_text, presence=presence)
    for lens, n in (([600, 40, 333], 300), ([1, 0, 700], 7), ([64, 640, 128], 0)):
        lens = np.minimum(lens, table.shape[1] * 16)
        length.copy_(torch.from_numpy(np.array(lens, np.int64)))
        n_text.fill_(n)
        g.replay()
        torch.cuda.synchronize()
        c["len"] = np.array(lens, np.int64)
        _check_attention(c, (out.double().cpu().numpy(), lse.double().cpu().numpy()))
        want = x.clone()
        for b in range(3):
            want[b, 0, text[b, :n].long().unique()] -= 0.5
        assert torch.equal(y, want)
