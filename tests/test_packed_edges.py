"""Head rotation, appends, reads and attention over the 4-bit cache at their edges: orders of access within a block, values that are
not finite beside turned elements, values beyond a half, empty pools, rows laid over others.

Oracles and tolerances are those of test_packed_cache.py and test_serving.py, where they are derived; what differs is said at the test.
"""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

from oracle import packed_ref as pref
from paper_2506_04708_b200 import binding, build as lib_build, inputs
from tests import test_packed_cache as tp
from tests import test_serving as ts

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2506_04708_b200", "csrc")
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return binding.lib()


# ---------------------------------------------------------------- order within a block
def _body(source, head):
    """The text between the braces that follow `head`, without comments."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, source)).read())
    at = text.index("{", text.index(head))
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[at + 1:i]
    raise AssertionError(head)


def test_what_a_block_shares_of_its_range_is_written_before_its_last_barrier():
    """Other warps read these members without a barrier of their own, so no write to them may follow the last one here."""
    body = _body("attention_split.cuh", "ta_begin(const TaSplit& p")
    last = body.rindex("__syncthreads()")
    written = {m.group(1): m.start() for m in re.finditer(r"\bsh\.(\w+)(?:\[[^\]]*\])?\s*=[^=]", body)}
    assert set(written) == {"sum", "b", "b_start", "total", "groups"}
    assert all(at < last for at in written.values()), written


# ---------------------------------------------------------------- elements past the turned ones
def _bits_of(t):
    """The bits of a tensor's elements, all NaN alike."""
    import torch
    return torch.where(torch.isnan(t), float("nan"), t).contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16)


def _rows_with_odd_values(dtype, dim, rotary, pairs, seed=0):
    """Rows [1, 1, 9, 1, dim]: ordinary ones, then with values that are not finite on both sides of where the turned elements end, and with a zero
    below zero; per row the elements that the turn makes of those."""
    import torch
    x = torch.from_numpy(np.random.default_rng(seed).standard_normal((1, 1, 9, 1, dim)).astype(np.float32)).to(ts._dtype(dtype))
    hit = np.zeros((9, dim), bool)
    inf, nan = float("inf"), float("nan")
    for row, (at, value) in enumerate([(rotary, inf), (rotary + 1, nan), (rotary + 2, -inf), (dim - 1, nan), (dim - 2, inf), (rotary - 1, inf), (0, nan),
                                       (rotary + 1, -0.0)], 1):
        if at >= dim:
            continue
        x[0, 0, row, 0, at] = value
        if value != 0:
            hit[row, at] = True
            if at < rotary:
                hit[row, at ^ 1 if pairs else (at + rotary // 2) % rotary] = True
    return x, hit


def _moved(x, shift):
    """The same rows, `shift` elements behind a boundary of 16 bytes."""
    import torch
    out = torch.empty(x.shape[:-1] + (x.shape[-1] + 16,), dtype=x.dtype, device=DEV)[..., shift:shift + x.shape[-1]]
    return out.copy_(x)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("pairs", [True, False])
@pytest.mark.parametrize("shift", [0, 4, 1])
@pytest.mark.parametrize("dim,rotary", [(80, 40), (100, 36), (64, 2), (128, 20), (48, 46), (128, 64), (31, 30), (16, 10)])
def test_elements_past_the_turned_ones_stay_as_they_are(dtype, pairs, shift, dim, rotary):
    """Bit by bit, whatever their neighbours hold; turned ones as defined, except what a value that is not finite is turned with.  The rows of a cache of
    their own type are the same."""
    import torch
    from paper_2506_04708_b200 import serving
    x, hit = _rows_with_odd_values(dtype, dim, rotary, pairs)
    n = x.shape[2]
    freq = (1000.0 ** (-np.arange(rotary // 2) / (rotary // 2))).astype(np.float32)
    offset = torch.arange(5, 5 + n, dtype=torch.int32, device=DEV)
    rows = _moved(x[0], shift)
    plan = serving.HeadRotation(1, n, 1, 1, dim, x.dtype, freq=tp._dev(freq), offset=offset, interleaved=pairs)
    q, k = plan(rows, rows, q_out=_moved(x[0], shift), k_out=_moved(x[0], shift))
    assert torch.equal(_bits_of(q), _bits_of(k))
    assert torch.equal(_bits_of(q[..., rotary:]), _bits_of(rows[..., rotary:]))
    got = q.double().cpu().numpy()[0, :, 0]
    assert np.array_equal(~np.isfinite(got), hit)
    fine = np.where(np.isfinite(x.double().numpy()[0, 0, :, 0]), x.double().numpy()[0, 0, :, 0], 0.0)
    want, size = pref.rotate(fine, np.arange(5, 5 + n), freq, pairs)
    tp._near(np.where(hit, 0.0, got), np.where(hit, 0.0, want), size, dtype, False)
    cache, other = (torch.zeros((1, 1, 1, 16, dim + 16), dtype=x.dtype, device=DEV)[..., shift:shift + dim] for _ in range(2))
    add = serving.KvAppend(1, 1, n, 1, dim, x.dtype, 16, 1, n, freq=tp._dev(freq), offset=offset, interleaved=pairs)
    add(rows[None], rows[None], torch.arange(n, device=DEV)[None], cache, other)
    assert torch.equal(_bits_of(cache[0, 0, 0, :n]), _bits_of(k[0, :, 0]))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("dim,rotary", [(80, 40), (128, 20)])
def test_in_4_bits_a_value_that_is_not_finite_spoils_its_group_alone(dtype, dim, rotary):
    import torch
    from paper_2506_04708_b200 import serving
    x, hit = _rows_with_odd_values(dtype, dim, rotary, True)
    n = x.shape[2]
    freq = torch.ones(rotary // 2, device=DEV)
    cache = [torch.zeros((1, 1, 1, serving.packed_block_bytes(16, dim)), dtype=torch.uint8, device=DEV) for _ in range(2)]
    slots = torch.arange(n, device=DEV)[None]
    add = serving.KvAppend(1, 1, n, 1, dim, x.dtype, 16, 1, n, packed=True, freq=freq, interleaved=True)
    add(x.to(DEV), x.to(DEV), slots, *cache)
    k, v = serving.KvRead(1, 1, 1, dim, torch.float32, 16, 1, n, packed=True)(slots, *cache)
    group = lambda h: np.repeat(h.reshape(n, dim // 16, 16).any(-1), 16, -1)  # noqa: E731
    assert np.array_equal(np.isnan(k.cpu().numpy()[0, 0, :, 0]), group(hit))
    assert np.array_equal(np.isnan(v.cpu().numpy()[0, 0, :, 0]), group(~np.isfinite(x.double().numpy()[0, 0, :, 0])))


# ---------------------------------------------------------------- values beyond a half
def _beyond_a_half(seed, dtype, lens, N, hq, hkv, dim):
    """A packed case whose keys and values reach 8 * 61,440 where texts are long enough to bring results back below 65,504."""
    c = tp._packed_case(seed, dtype, lens, N, hq, hkv, dim, 16, parent=inputs.topology(N, min(N - 1, 3), 4), nan=False, spare=0)
    rng = np.random.default_rng(seed)
    for name, rate in (("ck", 0.3), ("cv", 0.02)):
        blocks = c[name + "_packed"].numpy()
        codes, scales = blocks[..., : 16 * dim // 2], blocks[..., 16 * dim // 2:].reshape(blocks.shape[:2] + (16, dim // 16))
        codes[rng.random(codes.shape) < 0.02] &= 0xF0  # a code of -8, which nothing stores, reads as one
        large = rng.random(scales.shape) < rate
        if name == "cv":
            for b, n in enumerate(lens):
                if n < 300:
                    large[c["table"][b, : -(-n // 16)]] = False
        scales[large] = rng.integers(0xE8, 0xF8, large.sum())
        import torch
        c[name] = torch.from_numpy(pref.block_values(blocks, 16, dim))
    return c


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("lens", [[0, 5, 300, 700, 130], [6000]])
@pytest.mark.parametrize("N,hq,hkv,dim,odd", [(1, 8, 2, 128, False), (3, 4, 2, 64, False), (9, 4, 2, 64, False), (24, 4, 2, 64, False), (64, 4, 2, 64, False),
                                              (24, 8, 2, 128, False), (3, 2, 1, 256, False), (5, 4, 2, 80, False), (24, 8, 2, 128, True)])
def test_packed_attention_over_values_beyond_a_half(dtype, lens, N, hq, hkv, dim, odd):
    """A cache may hold 491,520 and a half ends at 65,504: every kernel takes what the codes stand for, whatever the call's type."""
    import torch
    if len(lens) == 1:
        lens = [lens[0] + N] if N > 30 else lens * 2
    c = _beyond_a_half(dim + 2 * N, dtype, lens, N, hq, hkv, dim)
    scale = 2.0**-21
    want = ts._reference(c, scale)
    assert np.abs(c["ck"].numpy()).max() > 400000 and np.abs(c["cv"].numpy()).max() > 400000 and np.abs(want[0]).max() < 60000

    def move(q, k, v, ck, cv):
        shift = lambda x: torch.empty(x.numel() + 1, dtype=x.dtype, device=DEV)[1:].view(x.shape).copy_(x)  # noqa: E731
        return (shift(q), shift(k), shift(v), ck, cv) if odd else (q, k, v, ck, cv)

    tp._check(c, tp._run_packed(c, scale=scale, move=move), want=want)


# ---------------------------------------------------------------- queries at the ends of their range
@pytest.mark.gpu
@pytest.mark.parametrize("size,scale", [(2.0**-120, 2.0**117), (2.0**-126, 2.0**122), (2.0**-118, 2.0**-40), (2.0**-100, 2.0**-60), (2.0**118, 2.0**-121), (0.0, 2.0**-100)])
@pytest.mark.parametrize("N,hq,dim", [(1, 4, 128), (1, 4, 64), (3, 8, 128), (24, 8, 64)])
def test_packed_queries_at_the_ends_of_the_range(size, scale, N, hq, dim):
    """bfloat16 rows as small and as large as the type has them, under scales that make ordinary scores of them or nothing at all."""
    c = tp._packed_case(93, "bf16", [300, 5, 0, 77], N, hq, 2, dim, 16, parent=inputs.topology(N, min(3, N - 1), 3), nan=False)
    c["qkv"][:, :, :hq] = (c["qkv"][:, :, :hq].double() * size).to(c["qkv"].dtype)
    tp._check(c, tp._run_packed(c, scale=scale), want=ts._reference(c, scale))


# ---------------------------------------------------------------- pools without pages
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("packed", [False, True])
def test_a_pool_without_pages(dtype, packed):
    """Appends skip every place, reads give zeros, attention takes every page as one of zeros."""
    import torch
    from paper_2506_04708_b200 import serving
    dt = ts._dtype(dtype)
    L, B, N, H, dim, page = 2, 3, 4, 2, 64, 16
    shape = (0, H, serving.packed_block_bytes(page, dim)) if packed else (0, H, page, dim)
    cache = torch.empty((L,) + shape, dtype=torch.uint8 if packed else dt, device=DEV)
    x = torch.randn((L, B, N, H, dim), device=DEV).to(dt)
    slots = torch.tensor([[0, 1, -1, 7]], device=DEV).expand(B, N).contiguous()
    serving.KvAppend(L, B, N, H, dim, dt, page, 0, N, packed=packed)(x, x, slots, cache, cache)
    for got in serving.KvRead(L, B, H, dim, dt, page, 0, N, packed=packed)(slots, cache, cache, k=x.clone(), v=x.clone()):
        assert not got.any()
    kind = serving.PackedTreeAttention if packed else serving.TreeAttention
    for nodes, hq in ((1, 2), (4, 2), (9, 8)):
        q = torch.randn((B, nodes, hq + 2 * H, dim), device=DEV).to(dt)
        args = q[:, :, :hq], q[:, :, hq:hq + H], q[:, :, hq + H:]
        table, length = torch.tensor([[0, -1, 5]] * B, dtype=torch.int32, device=DEV), torch.tensor([0, 20, 48], device=DEV)
        out, lse = kind(B, nodes, hq, H, dim, dt, page, 0, 3)(*args, cache[0], cache[0], table, length)
        zeros = torch.zeros((B * 3, H, page, dim), dtype=torch.float64)
        c = dict(qkv=q.cpu(), ck=zeros, cv=zeros, table=table.cpu().numpy(), len=length.cpu().numpy(), tree=None, parent=None, mask=None, hq=hq, hkv=H, dim=dim,
                 page=page, N=nodes, dtype=dtype)
        tp._check(c, (out.double().cpu().numpy(), lse.double().cpu().numpy()))


def test_caches_may_be_missing_only_where_there_are_no_pages(lib):
    A, B2 = C.c_void_p(0x100000), C.c_void_p(0x200000)  # never touched: every call here is refused before a launch
    for packed in (0, 1):
        for pages in (1, 5):
            assert lib.stand_kv_append(C.byref(tp._rows(packed=packed, pages=pages)), A, A, A, A, A, A, A, A, None, B2, None) == -1
            assert lib.stand_kv_read(C.byref(tp._rows(packed=packed, pages=pages, N=0, rotary_dim=0, norm=0, eps=0.0)), B2, None, A, A, A, None) == -1


# ---------------------------------------------------------------- rows laid over others
def _bytes_of(at, row, dims):
    """Every byte of rows, once for each time that it is one."""
    a = np.array([at], np.int64)
    for count, stride in dims:
        a = (a[:, None] + np.arange(count) * stride).ravel()
    return (a[:, None] + np.arange(row)).ravel()


def test_rows_that_meet_are_found(tmp_path):
    """Against the bytes themselves: dimensions inside one another, in any order, of equal and of other strides, rows between other rows."""
    exe = str(tmp_path / "rows_meet")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-o", exe, os.path.join(ROOT, "tests", "rows_meet.cpp")], check=True)
    rng = np.random.default_rng(0)
    lines, want, met = [], [], 0

    def layout(row):
        """A nested layout of 0 .. 4 dimensions, in any order."""
        size, out = row, []
        for _ in range(rng.integers(0, 5)):
            count = int(rng.integers(1, 5))
            stride = size + int(rng.choice([0, 0, 1, size, 2 * size, 7]))
            out.append((count, stride))
            size = stride * count
        return [out[i] for i in rng.permutation(len(out))]

    for i in range(6000):
        row = int(rng.integers(1, 9))
        x = layout(row)
        kind = rng.integers(0, 3)
        y = [(int(rng.integers(1, c + 1)), s) for c, s in x] if kind == 0 else (x if kind == 1 else layout(row))  # slices of one tensor, the same shape, another one
        other = row if kind else int(rng.integers(1, row + 1))
        far = 1 + sum((c - 1) * s for c, s in x) + row
        at = 10**6, 10**6 + int(rng.integers(-far, far + 1)) * int(rng.random() < 0.95)
        for a, r, dims in ((at[0], row, x), (at[1], other, y)):
            lines.append(f"{a} {r} {len(dims)} " + " ".join(f"{c} {s}" for c, s in dims))
        meet = bool(np.intersect1d(_bytes_of(at[0], row, x), _bytes_of(at[1], other, y)).size)
        met += meet
        alike = at[0] == at[1] and row == other and len(x) == len(y) and all(c == d and (c == 1 or s == t) for (c, s), (d, t) in zip(x, y))
        want.append((meet, alike))
    # far apart, long and with strides of 0; layouts that are not decided (three strides of no order among one another) are not said to meet
    for a, b, meet in (("4096 256 3 64 1048576 4096 2048 40 256", "14336 256 3 64 1048576 4096 2048 8 256", True), ("0 256 2 2147483647 10240 32 256", "8192 256 2 2147483647 10240 8 256", False),
                       ("0 256 2 2147483647 10240 33 256", "8192 256 2 2147483647 10240 8 256", True), ("0 8 1 5 0", "4 8 0", True), ("0 8 2 0 64 5 8", "0 8 0", False),
                       ("0 1 3 1000 1000003 1000 1000033 1000 1000037", "7 1 3 1000 1000081 1000 1000099 1000 1000117", None)):
        lines += [a, b]
        want.append((meet, False))
    got = subprocess.run([exe], input="\n".join(lines), check=True, capture_output=True, text=True).stdout.split()
    assert len(got) == len(want) and 1000 < met < 5000
    for i, (g, (meet, alike)) in enumerate(zip(got, want)):
        assert (meet is None or g[0] == str(int(meet))) and g[1] == str(int(alike)), (i, lines[2 * i:2 * i + 2], g, meet, alike)


def test_rows_laid_over_others_are_refused(lib):
    """At the C interface; no call here gets as far as a launch."""
    at = lambda n: C.c_void_p(0x1000000 + 2 * n)  # noqa: E731  (elements of 16 bits)
    far = C.c_void_p(0x9000000)
    one = dict(B=2, N=3, heads_q=4, heads_kv=2, dim=64, rotary_dim=64, norm=0, eps=0.0)
    side = (3 * 8 * 64, 8 * 64, 64)  # a projection of 4 + 2 + 2 heads
    own = {4: (768, 256, 64), 2: (384, 128, 64)}

    def rotate(q, k, qo, ko, qs=side, ks=side, qos=side, kos=side, **kw):
        s = tp._rotation(**dict(one, **kw), q_stride=qs, k_stride=ks, q_out_stride=qos, k_out_stride=kos)
        return lib.stand_rotate_heads(C.byref(s), q, k, None, None, far, None, None, qo, ko, None)

    q, k, v = at(0), at(256), at(384)
    apart = dict(qos=own[4], kos=own[2])
    for bad in (dict(qo=k, ko=far, kos=own[2]), dict(qo=far, qos=own[4], ko=q), dict(qo=at(64), ko=far, kos=own[2]), dict(qo=q, qos=own[4], ko=far, kos=own[2]),
                dict(qo=at(32), ko=far, kos=own[2]), dict(qo=v, ko=v), dict(qo=q, ko=at(320)), dict(qo=at(3 * 8 * 64), ko=far, kos=own[2]),
                dict(qo=far, qos=own[4], ko=C.c_void_p(0x9000000 + 128), kos=own[2]), dict(qo=far, qos=(0, 256, 64), ko=q, kos=side),
                dict(qo=far, qos=(768, 256, 0), ko=at(4096), kos=own[2]), dict(qo=at(4096), qos=own[4], ko=far, kos=(0, 128, 64))):
        assert rotate(**dict(dict(q=q, k=k), **bad)) == -1, bad
    assert rotate(q=q, k=q, qo=q, ko=far, kos=own[2]) == -1  # in place, but the keys are the same rows
    # keys written twice from rows that are not the same
    assert rotate(q=q, k=at(128), qo=far, ko=far, heads_q=2, qos=own[2], kos=own[2]) == -1

    rows = dict(layers=2, B=2, N=3, heads=2, dim=64, page_size=16, pages=5, norm=0, rotary_dim=0, eps=0.0)
    src = (2 * 3 * 2 * 64, 3 * 2 * 64, 2 * 64, 64)
    for packed, stride, size in ((0, (5 * 2 * 16 * 64, 2 * 16 * 64, 16 * 64, 64), 2 * 5 * 2 * 16 * 64), (1, (5 * 2 * 576, 2 * 576, 576, 0), 2 * 5 * 288)):

        def append(k, v, ck, cv, cache=stride):
            s = tp._rows(**dict(rows, packed=packed), k_stride=src, v_stride=src, cache_stride=cache)
            return lib.stand_kv_append(C.byref(s), k, v, None, None, None, None, None, A, ck, cv, None)

        A = C.c_void_p(0x8000000)
        for bad in (dict(k=at(0), v=far, ck=at(0), cv=A), dict(k=far, v=at(64), ck=A, cv=at(0)), dict(k=at(size - 64), v=far, ck=A, cv=at(0)), dict(k=far, v=at(0), ck=at(768), cv=A),
                    dict(k=far, v=far, ck=at(0), cv=at(0), cache=(0,) + stride[1:]), dict(k=far, v=far, ck=at(0), cv=at(0), cache=stride[:2] + (0,) + stride[3:])):
            assert append(**bad) == -1, bad

        def read(k, v, ck, cv):
            s = tp._rows(**dict(rows, packed=packed, N=0), cache_stride=stride)
            return lib.stand_kv_read(C.byref(s), ck, cv, A, k, v, None)

        for bad in (dict(k=at(0), v=far, ck=at(0), cv=A), dict(k=far, v=at(size - 8), ck=A, cv=at(0)), dict(k=far, v=C.c_void_p(0x9000000 + 128), ck=at(0), cv=at(0)),
                    dict(k=far, v=far, ck=at(0), cv=at(65536))):
            assert read(**bad) == -1, bad


@pytest.mark.gpu
def test_rows_between_others_are_written():
    """Results beside inputs in one tensor, row by row; in place; the same rows to the same place twice."""
    import torch
    from paper_2506_04708_b200 import serving
    B, N, hq, hkv, dim = 3, 5, 4, 2, 64
    buf = torch.randn((B, N, 2 * (hq + hkv), dim), device=DEV).bfloat16()
    q, k, qo, ko = buf.split([hq, hkv, hq, hkv], 2)
    op = serving.HeadRotation(B, N, hq, hkv, dim, torch.bfloat16, freq=torch.ones(32, device=DEV))
    want = [t.clone() for t in op(q.contiguous(), k.contiguous())]
    before = q.clone(), k.clone()
    op(q, k, q_out=qo, k_out=ko)
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1]) and torch.equal(q, before[0]) and torch.equal(k, before[1])
    op(q, k, q_out=qo, k_out=k)  # one in place
    assert torch.equal(qo, want[0]) and torch.equal(k, want[1])
    with pytest.raises(binding.StandError):
        op(q, k, q_out=buf[:, :, 1:1 + hq], k_out=ko)
    same = serving.HeadRotation(B, N, hkv, hkv, dim, torch.bfloat16, freq=torch.ones(32, device=DEV))
    one = same(before[1], before[1], q_out=ko, k_out=ko)[0]
    assert torch.equal(one, want[1])
    # a layer's rows between the pages of a cache that they go to
    arena = torch.zeros((1, 4, 2, 16 * dim + dim), dtype=torch.bfloat16, device=DEV)
    cache, rows = arena[..., :16 * dim].unflatten(-1, (16, dim)), arena[..., 16 * dim:][:, :, None]
    rows.copy_(torch.randn(rows.shape, device=DEV))
    other = torch.zeros((1, 4, 2, 17 * dim), dtype=torch.bfloat16, device=DEV)[..., :16 * dim].unflatten(-1, (16, dim))
    slots = torch.tensor([[3], [40], [17], [50]], device=DEV)
    serving.KvAppend(1, 4, 1, 2, dim, torch.bfloat16, 16, 4, 1)(rows, rows, slots, cache, other)
    for b, s in enumerate((3, 40, 17, 50)):
        assert torch.equal(cache[0, s // 16, :, s % 16], rows[0, b, 0]) and torch.equal(other[0, s // 16, :, s % 16], rows[0, b, 0])
    with pytest.raises(binding.StandError):
        serving.KvRead(1, 4, 2, dim, torch.bfloat16, 16, 4, 1)(slots, cache, cache, k=arena.flatten()[:512].view(1, 4, 1, 2, dim))


# ---------------------------------------------------------------- rows beyond the range of sums
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_whose_squares_pass_the_range_come_out_as_zeros(dtype):
    """As the contract says; the other rows are what they are without them, and rows just within it are normalised."""
    import torch
    from paper_2506_04708_b200 import serving
    x = torch.from_numpy(np.random.default_rng(2).standard_normal((1, 6, 2, 64)).astype(np.float32)).to(ts._dtype(dtype)).to(DEV)
    op = serving.HeadRotation(1, 6, 2, 2, 64, x.dtype, freq=torch.ones(32, device=DEV), norm=True)
    clean = op(x, x)[0].clone()
    x[0, 1, 0] *= 2.0**100
    x[0, 2, 1] *= 2.0**50  # squares of up to 2^104, 64 of them
    got = op(x, x)[0].clone()
    assert not got[0, 1, 0].any()
    want, size = pref.rotate(x[0, 2, 1].double().cpu().numpy()[None], np.array([2]), np.ones(32, np.float32), False, None, 1e-6)
    tp._near(got[0, 2, 1].double().cpu().numpy()[None], want, size, dtype, True)
    got[0, 1, 0], got[0, 2, 1] = clean[0, 1, 0], clean[0, 2, 1]
    assert torch.equal(got, clean)
