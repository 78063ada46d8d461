"""Head rotation, appends to the paged cache, its 4-bit form and attention over it, against plain statements in 64 bits
(oracle/packed_ref.py, oracle/serving_ref.py).

Tolerances.  u: unit roundoff of the output's type.  Rotation: the sum of squares has at most 16 + 4 roundings on the way
to an element's sum, its root half as many, the reciprocal root 2 units and three products: fewer than 2^5 roundings of
2^-24, 2^-19 of the normalised magnitudes; cosine and sine are off by at most 2^-23 + 2^-24 and the two products and the sum by 2^-24
each: 2^-21 of |a| + |b|; then one rounding to the type.  Stored codes are whole numbers: equal.  Attention: as
test_serving.py derives it; cached values are exact in all types.  Weights of cached tokens are halves in all 16-bit calls, 2^7 of
them at the running maximum, which is no further than 2^8 below the largest: a half is off by 2^-12 of itself or, below 2^-14, by 2^-25, so by less than
2^-32 of a row's largest weight: 2^-32 sum |v| is added for bfloat16 (half has 2^-25 there already), whose own tolerance is relative throughout.
"""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from oracle import packed_ref as pref
from paper_2506_04708_b200 import binding, build as lib_build, inputs
from tests import test_serving as ts

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return binding.lib()


# ---------------------------------------------------------------- host side, no GPU
def test_structures_match_the_header(tmp_path):
    pairs = [("stand_rotation", binding.StandRotation), ("stand_kv_rows", binding.StandKvRows)]
    prog = ['#include <stdio.h>', '#include <stddef.h>', '#include "stand.h"', 'int main(void) {']
    for name, st in pairs:
        prog.append(f'printf("%zu\\n", sizeof({name}));')
        prog += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in st._fields_]
    prog += ['printf("%zu\\n", STAND_PACKED_BLOCK_BYTES(48, 80));', 'return 0; }']
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(prog))
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)], check=True)
    got = [int(t) for t in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = []
    for _, st in pairs:
        want += [C.sizeof(st)] + [getattr(st, f).offset for f, _ in st._fields_]
    from paper_2506_04708_b200 import serving
    assert got == want + [serving.packed_block_bytes(48, 80)] and got[-1] == 48 * 80 // 2 + 48 * 80 // 16


def test_the_plain_statement_of_the_form():
    """Every scale and code once; ties go to the even code; a group's largest element never needs more than 7."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((400, 32)) * np.exp(4 * rng.standard_normal((400, 1)))
    codes, scales = pref.pack(x.astype(np.float32))
    back = pref.values(codes, scales)
    s = np.repeat(pref.SCALES[scales], 16, -1)
    top = np.abs(x.astype(np.float32)).reshape(400, 2, 16).max(-1)
    assert (np.abs(back - x) <= s * (0.5 + 1e-6)).all()
    assert (7 * pref.SCALES[scales] >= top).all() and (7 * pref.SCALES[scales - 1] < top).all()
    group = np.zeros((1, 16))
    group[0, :6] = 7, 0.5, 1.5, 2.5, -0.5, -1.5
    assert pref.values(*pref.pack(group))[0, :6].tolist() == [7, 0, 2, 2, 0, -2]
    assert np.isnan(pref.values(*pref.pack(np.array([[np.inf] + [1.0] * 15 + [2.0] * 16])))[0, :16]).all()


A, B2 = C.c_void_p(0x100000), C.c_void_p(0x200000)  # never touched: every call here is refused before a launch


def _rotation(**kw):
    d = dict(B=2, N=3, heads_q=4, heads_kv=2, dim=64, dtype=1, rotary_dim=64, interleaved=0, norm=1, eps=1e-6, reserved=0, reserved2=0)
    strides = {n: kw.pop(n) for n in list(kw) if n.endswith("stride")}
    d.update(kw)
    s = binding.StandRotation(*[d[n] for n, _ in binding.StandRotation._fields_[:12]])
    for n, v in strides.items():
        setattr(s, n, v) if isinstance(v, int) else getattr(s, n).__setitem__(slice(None), v)
    return s


def test_rotation_refuses_invalid_calls(lib):
    def call(q=A, k=A, wq=A, wk=A, freq=A, base=A, offset=A, qo=A, ko=A, **kw):
        return lib.stand_rotate_heads(C.byref(_rotation(**kw)), q, k, wq, wk, freq, base, offset, qo, ko, None)

    for bad in (dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(freq=None), dict(rotary_dim=0), dict(B=0), dict(N=0), dict(heads_q=0),
                dict(heads_kv=0), dict(heads_q=1 << 17), dict(heads_kv=1 << 17), dict(dim=0), dict(dim=257), dict(dtype=3), dict(dtype=-1),
                dict(rotary_dim=63), dict(rotary_dim=66), dict(rotary_dim=-2), dict(interleaved=2), dict(norm=2), dict(norm=0), dict(eps=0.0),
                dict(eps=float("nan")), dict(eps=float("inf")), dict(reserved=1), dict(reserved2=1), dict(offset_stride=-1),
                dict(q_stride=(-1, 0, 0)), dict(k_stride=(0, -1, 0)), dict(q_out_stride=(0, 0, -1)), dict(k_out_stride=(0, -1, 0)),
                dict(q=C.c_void_p(0x100001)), dict(ko=C.c_void_p(0x100001)), dict(wk=C.c_void_p(0x100001)), dict(freq=C.c_void_p(0x100002)),
                dict(base=C.c_void_p(0x100004)), dict(offset=C.c_void_p(0x100002))):
        assert call(**bad) == -1, bad
    assert lib.stand_rotate_heads(None, A, A, None, None, A, A, A, A, A, None) == -1


def _rows(**kw):
    d = dict(layers=2, B=2, N=3, heads=2, dim=64, dtype=1, page_size=16, pages=5, width=3, packed=1, rotary_dim=64, interleaved=0, norm=1,
             eps=1e-6, reserved=0, reserved2=0)
    strides = {n: kw.pop(n) for n in list(kw) if n.endswith("stride")}
    d.update(kw)
    s = binding.StandKvRows(*[d[n] for n, _ in binding.StandKvRows._fields_[:16]])
    for n, v in strides.items():
        setattr(s, n, v) if isinstance(v, int) else getattr(s, n).__setitem__(slice(None), v)
    return s


COMMON = (dict(layers=0), dict(layers=4097), dict(B=0), dict(heads=0), dict(heads=4097), dict(dim=0), dict(dim=257), dict(dim=72), dict(dtype=3),
          dict(page_size=0), dict(page_size=24), dict(page_size=8192), dict(pages=-1), dict(width=0), dict(width=1 << 31 - 1), dict(packed=2), dict(reserved=1),
          dict(reserved2=1), dict(cache_stride=(0, 0, 8, 0)), dict(cache_stride=(0, 24, 0, 0)), dict(cache_stride=(0, 0, 0, 64)),
          dict(cache_stride=(-16, 0, 0, 0)), dict(ck=None), dict(cv=None), dict(slots=None), dict(k=None), dict(v=None),
          dict(ck=C.c_void_p(0x100008)), dict(cv=C.c_void_p(0x100008)), dict(slots=C.c_void_p(0x100004)), dict(k=C.c_void_p(0x100001)),
          dict(v=C.c_void_p(0x100001)), dict(packed=0, ck=C.c_void_p(0x100001)), dict(packed=0, cache_stride=(0, 0, 0, -1)))


def test_append_refuses_invalid_calls(lib):
    def call(k=A, v=A, w=A, freq=A, base=A, offset=A, path=A, slots=A, ck=B2, cv=B2, **kw):
        return lib.stand_kv_append(C.byref(_rows(**kw)), k, v, w, freq, base, offset, path, slots, ck, cv, None)

    for bad in COMMON + (dict(N=0), dict(rotary_dim=0), dict(freq=None), dict(rotary_dim=66), dict(rotary_dim=31), dict(interleaved=-1), dict(norm=0),
                         dict(norm=-1), dict(eps=-1.0), dict(k_stride=(0, 0, 0, -1)), dict(v_stride=(-1, 0, 0, 0)), dict(offset_stride=-4),
                         dict(path=C.c_void_p(0x100002)), dict(w=C.c_void_p(0x100001)), dict(base=C.c_void_p(0x100004))):
        assert call(**dict(bad)) == -1, bad
    assert lib.stand_kv_append(None, A, A, None, None, None, None, None, A, B2, B2, None) == -1


def test_read_refuses_invalid_calls(lib):
    def call(k=A, v=A, slots=A, ck=B2, cv=B2, **kw):
        return lib.stand_kv_read(C.byref(_rows(**dict(dict(N=0, rotary_dim=0, norm=0, eps=0.0), **kw))), ck, cv, slots, k, v, None)

    for bad in COMMON + (dict(rotary_dim=2), dict(norm=1)):
        assert call(**dict(bad)) == -1, bad
    assert lib.stand_kv_read(None, B2, B2, A, A, A, None) == -1


def test_packed_attention_refuses_invalid_calls(lib):
    size = lib.stand_tree_attention_scratch_bytes(C.byref(ts._shape()))

    def call(q=A, k=A, v=A, ck=A, cv=A, table=A, length=A, mask=None, stride=0, scratch=A, n=size, out=A, cache=(0, 0, 0), **kw):
        s = ts._shape(**kw)
        s.cache_stride[:] = cache
        return lib.stand_packed_tree_attention(C.byref(s), q, k, v, ck, cv, table, length, mask, stride, None, scratch, n, out, None, None)

    for name in ("q", "k", "v", "ck", "cv", "table", "length", "out"):
        assert call(**{name: None}) == -1, name
    for bad in (dict(dim=72), dict(dim=8), dict(cache=(8, 0, 0)), dict(cache=(0, 40, 0)), dict(cache=(0, 0, 64)), dict(cache=(-16, 0, 0)),
                dict(ck=C.c_void_p(0x100008)), dict(cv=C.c_void_p(0x100004)), dict(heads_q=7), dict(dtype=4), dict(page_size=20), dict(mask=A, stride=-1)):
        assert call(**bad) == -1, bad
    assert call(scratch=None) == -2 and call(n=size - 1) == -2 and call(scratch=C.c_void_p(0x100080)) == -2


# ---------------------------------------------------------------- head rotation
def _heads(seed, dtype, B, N, hq, hkv, dim, rotary, norm, offsets, far):
    """Numpy inputs of one call."""
    import torch
    rng = np.random.default_rng(seed)
    dt = ts._dtype(dtype)
    x = torch.from_numpy(rng.standard_normal((B, N, hq + 2 * hkv, dim)).astype(np.float32) * 3).to(dt)
    freq = (10000.0 ** (-np.arange(rotary // 2) / max(1, rotary // 2))).astype(np.float32) if rotary else None
    weight = [torch.from_numpy((1 + 0.3 * rng.standard_normal(dim)).astype(np.float32)).to(dt) if norm == "weights" else None for _ in range(2)]
    offset = {"none": None, "shared": rng.integers(0, 9, N).astype(np.int32), "own": rng.integers(-3, 9, (B, N)).astype(np.int32)}[offsets]
    base = rng.integers(0, far, B)
    return x, freq, weight, offset, base


def _where(base, offset, B, N):
    off = np.arange(N) if offset is None else offset
    return (0 if base is None else base[:, None]) + np.broadcast_to(off, (B, N))


def _dev(a):
    import torch
    return None if a is None else (a if isinstance(a, torch.Tensor) else torch.from_numpy(np.ascontiguousarray(a))).to(DEV)


def _near(got, want, size, dtype, norm):
    u = ts.U[dtype]
    tol = u * np.abs(want) * 0.5 * 2 + (2.0**-21 + (2.0**-19 if norm else 0)) * size * (1 + u) + (2.0**-25 if dtype == "f16" else 1e-38)
    worst = np.max(np.abs(got - want) / tol)
    assert worst <= 1.0, worst


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("B,N,hq,hkv,dim,rotary,norm,offsets,far", [
    (1, 1, 32, 8, 128, 128, "weights", "none", 700), (3, 5, 4, 1, 64, 64, "ones", "shared", 10**6), (2, 7, 3, 3, 80, 40, "", "own", 2**31 - 20),
    (2, 33, 6, 2, 256, 256, "weights", "shared", 5000), (4, 100, 2, 1, 16, 16, "", "none", 1), (2, 3, 5, 2, 100, 36, "weights", "own", 40000),
    (1, 2, 2, 1, 1, 0, "weights", "none", 9), (2, 300, 28, 4, 128, 64, "weights", "shared", 900000), (3, 3, 2, 2, 31, 30, "ones", "none", 90),
    (600, 2, 1, 1, 96, 96, "weights", "own", 100000), (2, 3, 40, 40, 48, 0, "weights", "none", 2)])
def test_rotation_matches_the_definition(dtype, pairs, B, N, hq, hkv, dim, rotary, norm, offsets, far):
    from paper_2506_04708_b200 import serving
    offsets = offsets if rotary else "none"
    x, freq, weight, offset, base = _heads(dim + N, dtype, B, N, hq, hkv, dim, rotary, norm, offsets, far)
    kw = dict(freq=_dev(freq), offset=_dev(offset), interleaved=pairs, norm=bool(norm), weight_q=_dev(weight[0]), weight_k=_dev(weight[1]), eps=1e-5)
    plan = serving.HeadRotation(B, N, hq, hkv, dim, x.dtype, **kw)
    d = x.to(DEV)
    plan.q_out.fill_(float("nan"))
    plan.k_out.fill_(float("nan"))
    got = plan(d[:, :, :hq], d[:, :, hq:hq + hkv], _dev(base))
    pos = _where(base, offset, B, N)[..., None]
    for out, lo, hi, w in ((got[0], 0, hq, weight[0]), (got[1], hq, hq + hkv, weight[1])):
        want, size = pref.rotate(x[:, :, lo:hi].double().numpy(), pos, freq, pairs, None if w is None else w.double().numpy(), 1e-5 if norm else None)
        _near(out.double().cpu().numpy(), want, size, dtype, norm)
    # in place: the same bits, and nothing else of the projection is touched
    e = d.clone()
    plan(e[:, :, :hq], e[:, :, hq:hq + hkv], _dev(base), q_out=e[:, :, :hq], k_out=e[:, :, hq:hq + hkv])
    import torch
    assert torch.equal(e[:, :, :hq], got[0]) and torch.equal(e[:, :, hq:hq + hkv], got[1]) and torch.equal(e[:, :, hq + hkv:], d[:, :, hq + hkv:])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
def test_rotation_of_rows_laid_out_in_other_ways(dtype):
    """Head-major rows, rows off 16-byte boundaries, one row for all heads; results into slices."""
    import torch
    from paper_2506_04708_b200 import serving
    B, N, hq, hkv, dim = 2, 5, 4, 2, 64
    x, freq, weight, offset, base = _heads(3, dtype, B, N, hq, hkv, dim, 64, "weights", "shared", 1000)
    plan = serving.HeadRotation(B, N, hq, hkv, dim, x.dtype, freq=_dev(freq), offset=_dev(offset), norm=True, weight_q=_dev(weight[0]), weight_k=_dev(weight[1]))
    q, k = x.to(DEV)[:, :, :hq], x.to(DEV)[:, :, hq:hq + hkv]
    want = [t.clone() for t in plan(q.contiguous(), k.contiguous(), _dev(base))]
    pos = _where(base, offset, B, N)[..., None]
    for out, t, w in ((want[0], q, weight[0]), (want[1], k, weight[1])):
        _near(out.double().cpu().numpy(), *pref.rotate(t.double().cpu().numpy(), pos, freq, False, w.double().numpy(), 1e-6), dtype, True)
    major = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)  # noqa: E731
    odd = lambda t: torch.empty(t.shape[:-1] + (dim + 3,), dtype=t.dtype, device=DEV)[..., 1:-2].copy_(t)  # noqa: E731
    for change, near in ((major, False), (odd, True)):
        out = plan(change(q), change(k), _dev(base), q_out=change(torch.zeros_like(want[0])), k_out=change(torch.zeros_like(want[1])))
        for o, w in zip(out, want):
            if near:  # element by element: sums in the same order, products of other instructions
                d = (o.double() - w.double()).abs().max()
                assert float(d) <= 2 * ts.U[dtype] * float(w.double().abs().max()) + 2.0**-19 * 20
            else:
                assert torch.equal(o, w)
    same = plan(q[:, :, :1].expand(-1, -1, hq, -1), k[:, :, :1].expand(-1, -1, hkv, -1), _dev(base))
    assert torch.equal(same[0][:, :, 0], want[0][:, :, 0]) and torch.equal(same[0][:, :, 3], want[0][:, :, 0]) and torch.equal(same[1][:, :, 1], want[1][:, :, 0])


@pytest.mark.gpu
def test_rotation_keeps_rows_that_are_not_finite_to_themselves():
    import torch
    from paper_2506_04708_b200 import serving
    q = torch.ones((1, 4, 4, 64), device=DEV)
    k = torch.ones((1, 4, 2, 64), device=DEV)
    plan = serving.HeadRotation(1, 4, 4, 2, 64, torch.float32, freq=torch.ones(32, device=DEV), norm=True)
    clean = [t.clone() for t in plan(q, k)]
    q[0, 1, 2, 5], q[0, 3, 3, 6], k[0, 2, 1, 63] = float("nan"), float("inf"), float("-inf")
    out = plan(q, k)
    assert torch.isnan(out[0][0, 1, 2]).all() and torch.isnan(out[1][0, 2, 1, 63])
    keep = torch.ones((4, 4), dtype=torch.bool, device=DEV)
    keep[1, 2] = keep[3, 3] = False
    assert torch.equal(out[0][0][keep], clean[0][0][keep]) and torch.equal(out[1][0, :2], clean[1][0, :2]) and torch.equal(out[1][0, 2, 0], clean[1][0, 2, 0])


# ---------------------------------------------------------------- appends and reads
def _append_case(seed, dtype, L, B, N, H, dim, page, width, packed, path, spare=2):
    import torch
    from paper_2506_04708_b200 import serving
    rng = np.random.default_rng(seed)
    dt = ts._dtype(dtype)
    pool = -(-B * width // page) + spare
    kv = torch.from_numpy(rng.standard_normal((L, B, N, 2 * H, dim)).astype(np.float32) * np.exp(rng.standard_normal(dim)).astype(np.float32)).to(dt).to(DEV)
    slots = rng.permutation(pool * page)[: B * width].reshape(B, width).astype(np.int64)
    drop = rng.random((B, width)) < 0.25
    slots[drop] = rng.choice([-1, -9, pool * page, 1 << 40], drop.sum())
    places = rng.integers(-1, N + 1, (B, width)).astype(np.int32) if path else None
    if packed:
        caches = [torch.from_numpy(rng.integers(0, 256, (L, pool, H, serving.packed_block_bytes(page, dim))).astype(np.uint8)).to(DEV) for _ in range(2)]
    else:
        caches = [torch.from_numpy(rng.standard_normal((L, pool, H, page, dim)).astype(np.float32)).to(dt).to(DEV) for _ in range(2)]
    return kv[:, :, :, :H], kv[:, :, :, H:], slots, places, caches, pool


def _stored(before, rows, places, slots, page, dim, packed):
    """Caches with rows [L, B, N, H, dim] (numpy, exact) stored: bytes (packed) or values."""
    out = before.copy()
    L, pool, H = before.shape[:3]
    for b in range(slots.shape[0]):
        for j in range(slots.shape[1]):
            node, s = (j if places is None else int(places[b, j])), int(slots[b, j])
            if not (0 <= s < pool * page and 0 <= node < rows.shape[2]):
                continue
            if packed:
                codes, scales = pref.pack(rows[:, b, node])
                at, cut = s % page, page * dim // 2
                out[:, s // page, :, at * dim // 2:(at + 1) * dim // 2] = codes
                out[:, s // page, :, cut + at * dim // 16: cut + (at + 1) * dim // 16] = scales
            else:
                out[:, s // page, :, s % page] = rows[:, b, node]
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("L,B,N,H,dim,page,width,path", [
    (1, 1, 1, 8, 128, 16, 1, False), (3, 5, 9, 2, 64, 16, 4, True), (2, 2, 40, 3, 80, 48, 40, False), (28, 3, 6, 4, 128, 32, 5, True), (1, 7, 3, 1, 16, 64, 2, True),
    (2, 1, 300, 2, 256, 16, 300, False), (5, 90, 2, 2, 96, 16, 2, True)])
def test_append_stores_the_rows_and_nothing_else(dtype, packed, L, B, N, H, dim, page, width, path):
    import torch
    from paper_2506_04708_b200 import serving
    k, v, slots, places, caches, pool = _append_case(dim + N, dtype, L, B, N, H, dim, page, width, packed, path)
    before = [c.clone() for c in caches]
    op = serving.KvAppend(L, B, N, H, dim, k.dtype, page, pool, width, packed=packed)
    op(k, v, _dev(slots), caches[0], caches[1], path=_dev(places))
    for c, old, x in zip(caches, before, (k, v)):
        old = old.cpu().numpy() if packed else old.double().cpu().numpy()
        got = c.cpu().numpy() if packed else c.double().cpu().numpy()
        assert np.array_equal(got, _stored(old, x.double().cpu().numpy(), places, slots, page, dim, packed))
    # and back
    read = serving.KvRead(L, B, H, dim, k.dtype, page, pool, width, packed=packed)
    back = read(_dev(slots), caches[0], caches[1])
    there = (slots >= 0) & (slots < pool * page)
    s = np.where(there, slots, 0)
    for got, c in zip(back, caches):
        full = pref.block_values(c.cpu().numpy(), page, dim) if packed else c.double().cpu().numpy()
        want = np.where(there[None, ..., None, None], full[:, s // page, :, s % page].transpose(2, 0, 1, 3, 4), 0.0)
        want = torch.from_numpy(want).to(k.dtype).double().numpy()
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("dim,rotary,pairs,norm,offsets", [(128, 128, False, True, "shared"), (64, 64, True, False, "none"), (80, 40, False, True, "own"),
                                                           (96, 96, True, True, "shared"), (64, 32, False, False, "own"), (128, 0, False, True, "none")])
def test_append_turns_keys_as_head_rotation_does(dtype, packed, dim, rotary, pairs, norm, offsets):
    """The cache holds what it would hold had the keys been turned first; values are not turned."""
    import torch
    from paper_2506_04708_b200 import serving
    L, B, N, H, page, width = 3, 4, 12, 2, 16, 5
    k, v, slots, places, caches, pool = _append_case(rotary + dim, dtype, L, B, N, H, dim, page, width, packed, True)
    _, freq, _, offset, base = _heads(dim, dtype, B, N, H, H, dim, rotary, "", offsets if rotary else "none", 50000)
    rng = np.random.default_rng(1)
    weight = torch.from_numpy((1 + 0.3 * rng.standard_normal((L, dim))).astype(np.float32)).to(k.dtype).to(DEV) if norm else None
    turn = dict(freq=_dev(freq), offset=_dev(offset), interleaved=pairs, norm=norm)
    want = [c.clone() for c in caches]
    turned = []
    for l in range(L):
        w = weight[l].contiguous() if norm else None
        plan = serving.HeadRotation(B, N, H, H, dim, k.dtype, weight_q=w, weight_k=w, **turn)
        turned.append(plan(k[l], k[l], _dev(base))[1].clone())
    serving.KvAppend(L, B, N, H, dim, k.dtype, page, pool, width, packed=packed)(torch.stack(turned), v, _dev(slots), want[0], want[1], path=_dev(places))
    op = serving.KvAppend(L, B, N, H, dim, k.dtype, page, pool, width, packed=packed, weight_k=weight, **turn)
    op(k, v, _dev(slots), caches[0], caches[1], base=_dev(base), path=_dev(places))
    for got, w in zip(caches, want):
        assert torch.equal(got, w)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
def test_every_magnitude_tie_and_odd_value_is_stored_as_defined(dtype):
    """Groups whose largest element runs through all magnitudes of the type; exact ties; zeros; values that are not finite."""
    import torch
    from paper_2506_04708_b200 import serving
    rng = np.random.default_rng(6)
    N, dim, page = 2000, 64, 16
    x = rng.standard_normal((1, 1, N, 1, dim)) * 2.0 ** rng.integers(-30, 16, (1, 1, N, 1, 1))
    s = pref.SCALES[rng.integers(8, 8 * 25, (N // 2, dim // 16))]
    ties = (rng.integers(-7, 7, (N // 2, dim // 16, 16)) + 0.5) * s[..., None]  # half steps
    ties[..., 0] = 7 * s
    x[0, 0, : N // 2, 0] = ties.reshape(N // 2, dim)
    x[0, 0, 0, 0, :16], x[0, 0, 1, 0, 3], x[0, 0, 2, 0, 20], x[0, 0, 3, 0, 40] = 0, np.nan, np.inf, -np.inf
    x[0, 0, 4, 0] = 1e-8
    x[0, 0, 5, 0] = 6e4
    if dtype != "f16":
        x[0, 0, 6, 0, :40], x[0, 0, 7, 0, 3], x[0, 0, 8, 0, 8] = 430080.0, 1e30, -500000.0
    k = torch.from_numpy(x).to(ts._dtype(dtype)).to(DEV)
    pool = N // page
    caches = [torch.zeros((1, pool, 1, serving.packed_block_bytes(page, dim)), dtype=torch.uint8, device=DEV) for _ in range(2)]
    slots = np.arange(N)[None]
    serving.KvAppend(1, 1, N, 1, dim, k.dtype, page, pool, N, packed=True)(k, k, _dev(slots), caches[0], caches[1])
    rows = k.double().cpu().numpy()
    want = _stored(np.zeros(caches[0].shape, np.uint8), rows, None, slots, page, dim, True)
    assert np.array_equal(caches[0].cpu().numpy(), want) and np.array_equal(caches[1].cpu().numpy(), want)
    for out in ("bf16", "f16", "f32"):  # bfloat16 holds every value
        read = serving.KvRead(1, 1, 1, dim, ts._dtype(out), page, pool, N, packed=True)
        got = read(_dev(slots), *caches)[0].double().cpu().numpy().reshape(pool, page, dim)
        v = pref.block_values(want, page, dim)[0, :, 0]
        rounded = torch.from_numpy(v).to(ts._dtype(out)).double().numpy()
        assert np.array_equal(got, rounded, equal_nan=True)
        if out != "f16":
            assert np.array_equal(rounded, v, equal_nan=True)


@pytest.mark.gpu
@pytest.mark.parametrize("packed", [False, True])
def test_appends_and_reads_pass_32_bits(packed):
    """Slots at the far end of a pool of more than 2^32 bytes."""
    import torch
    from paper_2506_04708_b200 import serving
    H, page, dim = 8, 64, 128
    unit = serving.packed_block_bytes(page, dim) if packed else page * dim * 2
    pool = (2**32 + 2**28) // (H * unit)
    shape = (1, pool, H, unit) if packed else (1, pool, H, page, dim)
    cache = torch.zeros(shape, dtype=torch.uint8 if packed else torch.bfloat16, device=DEV)
    k = torch.randn((1, 1, 3, H, dim), dtype=torch.bfloat16, device=DEV)
    slots = torch.tensor([[pool * page - 1, 5, (pool - 1) * page]], device=DEV)
    serving.KvAppend(1, 1, 3, H, dim, torch.bfloat16, page, pool, 3, packed=packed)(k, k, slots, cache, cache)
    back = serving.KvRead(1, 1, H, dim, torch.bfloat16, page, pool, 3, packed=packed)(slots, cache, cache)[0]
    rows = k.double().cpu().numpy()
    want = pref.values(*pref.pack(rows)) if packed else rows
    assert np.array_equal(back.double().cpu().numpy(), want)
    assert int((cache[0].reshape(pool, -1).any(1)).sum()) == 2


# ---------------------------------------------------------------- attention over packed caches
def _check(c, got, want=None, scale=None):
    want = ts._reference(c, scale) if want is None else want
    if c["dtype"] == "bf16":  # what test_serving's tolerance lacks here, in units that it knows: u (weight + 2^-24 spread) >= u weight + 2^-32 spread
        r_out, r_lse, weight, spread, reach = want
        want = r_out, r_lse, weight + 2.0**-24 * spread, spread, reach
    if c["dtype"] == "f16":  # halves below 2^-14 lie 2^-24 apart, so a result there is off by up to 2^-25: its unit of spread is 2^-25.  (Of 4-bit values
        r_out, r_lse, weight, spread, reach = want  # many are zero, and results are small where the large weights meet those.)
        want = r_out, r_lse, weight, spread + 1.0, reach
    ts._check_attention(c, got, want=want)


def _packed_case(*a, **kw):
    """test_serving's case with caches in the 4-bit form beside what they stand for."""
    import torch
    c = ts._attention_case(*a, **kw)
    return _repacked(c)


def _repacked(c):
    import torch
    for name in ("ck", "cv"):
        c[name + "_packed"] = torch.from_numpy(pref.blocks(c[name].float().numpy()))
        c[name] = torch.from_numpy(pref.block_values(c[name + "_packed"].numpy(), c["page"], c["dim"]))
    return c


def _run_packed(c, stream=None, scale=None, move=None, plan=None):
    import torch
    from paper_2506_04708_b200 import serving
    B, N, hq, hkv = len(c["len"]), c["N"], c["hq"], c["hkv"]
    qkv, ck, cv = c["qkv"].to(DEV), c["ck_packed"].to(DEV), c["cv_packed"].to(DEV)
    q, k, v = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:]
    if move is not None:
        q, k, v, ck, cv = move(q, k, v, ck, cv)
    mask = None if c["mask"] is None else torch.from_numpy(ts._bits(c["mask"])).to(DEV)
    if plan is None:
        plan = serving.PackedTreeAttention(B, N, hq, hkv, c["dim"], ts._dtype(c["dtype"]), c["page"], ck.shape[0], c["table"].shape[1], scale=scale,
                                           parent=c["parent"], mask=mask)
    plan.out.fill_(float("nan"))
    plan.lse.fill_(float("nan"))
    tree = None if c["tree"] is None else torch.from_numpy(c["tree"]).to(DEV)
    args = (q, k, v, ck, cv, torch.from_numpy(c["table"]).to(DEV), torch.from_numpy(c["len"]).to(DEV))
    torch.cuda.synchronize()
    out, lse = plan(*args, tree_tokens=tree, stream=stream)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("N,D,kb,hq,hkv,dim,page", [
    (1, 0, 1, 8, 2, 128, 16), (1, 0, 1, 3, 3, 64, 32), (1, 0, 1, 16, 1, 128, 48), (1, 0, 1, 8, 1, 64, 16), (2, 1, 1, 16, 2, 128, 64), (8, 4, 2, 8, 2, 64, 16),
    (24, 6, 3, 12, 3, 128, 64), (64, 8, 4, 7, 1, 128, 48), (13, 4, 3, 6, 2, 80, 16), (33, 6, 4, 5, 1, 96, 128), (9, 4, 2, 4, 2, 256, 16), (40, 6, 4, 4, 1, 192, 32),
    (5, 2, 2, 2, 1, 16, 16), (3, 2, 1, 5, 1, 128, 16), (4, 3, 1, 4, 1, 64, 16), (1, 0, 1, 4, 1, 256, 16), (1, 0, 1, 130, 1, 64, 16), (3, 1, 2, 6, 1, 128, 16)])
def test_packed_attention_matches_the_definition(dtype, N, D, kb, hq, hkv, dim, page):
    """Lengths around page and tile boundaries, a sequence without text, one with a single token; single tokens."""
    lens = [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 517]
    if N > 30:
        lens = [0, 1, 64, 130, 517]
    c = _packed_case(N * dim, dtype, lens, N, hq, hkv, dim, page, parent=inputs.topology(N, D, kb))
    _check(c, _run_packed(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("B,length,N,hq,hkv,dim", [(1, 5000, 8, 8, 2, 128), (2, 4097, 64, 7, 1, 128), (1, 9000, 1, 16, 2, 128), (3, 2500, 24, 8, 1, 128),
                                                   (1, 7000, 1, 4, 4, 64), (30, 900, 1, 8, 2, 64)])
def test_long_packed_texts_are_split_and_joined(dtype, B, length, N, hq, hkv, dim):
    parent = inputs.topology(N, min(8, N - 1), 4)
    c = _packed_case(length, dtype, [length - 27 * b for b in range(B)], N, hq, hkv, dim, 16, parent=parent)
    _check(c, _run_packed(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("N,hq,hkv,dim", [(70, 4, 1, 64), (200, 4, 2, 64), (700, 2, 1, 128), (129, 16, 1, 128), (5, 3, 1, 128)])
def test_packed_chains_and_prompts_without_a_mask(dtype, N, hq, hkv, dim):
    c = _packed_case(N, dtype, [0, 33, 150], N, hq, hkv, dim, 16)
    _check(c, _run_packed(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("N,hq,hkv,dim", [(24, 8, 2, 128), (4, 4, 1, 64), (2, 4, 1, 128)])
def test_packed_undrafted_nodes_get_empty_rows(dtype, N, hq, hkv, dim):
    c = _packed_case(11, dtype, [0, 100, 64, 700], N, hq, hkv, dim, 16, parent=inputs.topology(N, min(6, N - 1), 3), undrafted=0.4)
    c["tree"][1, N - 1] = -1
    _check(c, _run_packed(c))
    c["tree"][:] = -1
    out, lse = _run_packed(c)
    assert not out.any() and np.isneginf(lse).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("N,hq,hkv,dim", [(45, 6, 2, 64), (3, 4, 1, 128), (2, 8, 1, 64)])
@pytest.mark.parametrize("shared", [True, False])
def test_packed_masks_and_rows_that_see_nothing(dtype, shared, N, hq, hkv, dim):
    rng = np.random.default_rng(3)
    lens = [0, 0, 17, 200]
    seen = rng.random((len(lens), N, N)) < 0.3
    seen[:, ::5] = False
    c = _packed_case(12, dtype, lens, N, hq, hkv, dim, 16, mask=seen[0] if shared else seen)
    out, lse = _run_packed(c)
    assert np.isneginf(lse[0, 0]).all()
    _check(c, (out, lse))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("N,D,kb,hq,hkv,dim", [(24, 6, 3, 4, 2, 64), (4, 2, 2, 4, 2, 128), (24, 6, 3, 4, 2, 128), (3, 1, 2, 4, 2, 64), (9, 3, 2, 4, 2, 256)])
def test_packed_a_node_value_that_is_not_finite_reaches_only_the_rows_that_see_it(dtype, N, D, kb, hq, hkv, dim):
    parent = inputs.topology(N, D, kb)
    c = _packed_case(21, dtype, [0, 90], N, hq, hkv, dim, 16, parent=parent)
    bad = N // 2
    clean = ts._reference(c)
    c["qkv"][:, bad, hq + hkv + 1, 7] = float("inf")   # value head 1, element 7
    c["qkv"][0, bad, hq + hkv, 3] = float("nan")       # value head 0, element 3, first sequence
    out, lse = _run_packed(c)
    below = ts.ref.ancestors(parent)[:, bad]
    assert np.isposinf(out[:, below, 2:, 7]).all() and np.isnan(out[0, below, :2, 3]).all()
    hit = np.zeros_like(out, bool)
    hit[:, below, 2:, 7] = True
    hit[0, below, :2, 3] = True
    assert np.isfinite(out[~hit]).all()
    _check(c, (np.where(hit, clean[0], out), lse), want=clean)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("N,hq,hkv,dim", [(3, 2, 2, 64), (24, 4, 2, 64), (1, 4, 2, 128), (24, 4, 2, 128), (8, 8, 2, 256)])
def test_packed_groups_that_are_not_finite(dtype, N, hq, hkv, dim):
    """A value's group that reads as NaN makes these 16 elements of all rows of its head NaN, however small its weight; a key's makes the
    rows NaN; in pages that are not the sequence's, or past its end, it touches nothing."""
    c = _packed_case(dim + N, dtype, [1, 70, 300, 300], N, hq, hkv, dim, 16, parent=inputs.topology(N, min(2, N - 1), 6))
    clean, g, group = ts._reference(c), hkv - 1, hq // hkv
    cut = 16 * dim // 2

    def spoil(name, b, pos, head, element, byte):
        c[name + "_packed"][int(c["table"][b, pos // 16]), head, cut + pos % 16 * (dim // 16) + element // 16] = byte
    spoil("cv", 1, 69, g, 20, 0xFF)
    spoil("cv", 2, 17, 0, 3, 0xF8)  # an infinite scale: the same
    spoil("ck", 3, 200, g, 40, 0xFC)
    out, lse = _run_packed(c)
    hit = np.zeros_like(out, bool)
    hit[1, :, g * group:, 16:32] = True
    hit[2, :, :group, :16] = True
    hit[3, :, g * group:] = True
    assert np.isnan(out[hit]).all() and np.isnan(lse[3, :, g * group:]).all()
    lse[3, :, g * group:] = clean[1][3, :, g * group:]
    _check(c, (np.where(hit, clean[0], out), lse), want=clean)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("N,hq", [(8, 8), (1, 8)])
@pytest.mark.parametrize("how", ["page-major heads", "contiguous nodes", "odd offsets", "padded blocks"])
def test_packed_strides_and_alignment(dtype, how, N, hq):
    import torch
    c = _packed_case(31, dtype, [0, 1, 77, 300], N, hq, 2, 64, 32, parent=inputs.topology(N, min(4, N - 1), 2))

    def move(q, k, v, ck, cv):
        if how == "page-major heads":  # [heads, pages, block]
            return (q, k, v) + tuple(x.transpose(0, 1).contiguous().transpose(0, 1) for x in (ck, cv))
        if how == "contiguous nodes":
            return q.contiguous(), k.contiguous(), v.contiguous(), ck, cv
        if how == "odd offsets":
            shift = lambda x: torch.empty(x.numel() + 1, dtype=x.dtype, device=x.device)[1:].view(x.shape).copy_(x)  # noqa: E731
            return tuple(shift(x) for x in (q, k, v)) + (ck, cv)
        pad = lambda x: torch.empty(x.shape[:-1] + (x.shape[-1] + 48,), dtype=x.dtype, device=x.device)[..., 16:-32].copy_(x)  # noqa: E731
        return q, k, v, pad(ck), pad(cv)

    _check(c, _run_packed(c, move=move))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("N,hq,dim", [(8, 4, 64), (1, 4, 128), (24, 4, 128)])
def test_packed_steep_and_flat_scores(dtype, N, hq, dim):
    """Scores that grow along the text, large ones, all equal ones, all far below zero."""
    import torch
    c = ts._attention_case(41, dtype, [400, 700], N, hq, 1, dim, 16, parent=inputs.topology(N, min(4, N - 1), 2), nan=False)
    for b, n in enumerate(c["len"]):
        for pos in range(n):
            c["ck"][int(c["table"][b, pos // 16]), :, pos % 16] *= 8.0 * pos / n
    raw = c["ck"].clone()
    c = _repacked(c)
    _check(c, _run_packed(c))
    _check(c, _run_packed(c, scale=1.0), want=ts._reference(c, 1.0))
    c["qkv"][:, :, :hq] = 0
    _check(c, _run_packed(c))
    c["ck"] = -torch.abs(raw) - 4
    c = _repacked(dict(c, cv=c["cv"]))
    c["qkv"][:, :, hq] = -6
    c["qkv"][:, :, :hq] = 3
    _check(c, _run_packed(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("N,dim", [(8, 64), (1, 64), (1, 128), (30, 128)])
def test_packed_lengths_and_tables_out_of_range_do_not_fault(dtype, N, dim):
    """A length below 0 counts as 0, one beyond the table as the table; entries outside the pool read as zeros."""
    c = _packed_case(51, dtype, [40, 64, 64], N, 4, 2, dim, 16, parent=inputs.topology(N, min(4, N - 1), 2), nan=False)
    c["len"][:] = [-5, 10**12, 60]
    c["table"][2, 1] = 10**9
    c["table"][2, 2] = -3
    _check(c, _run_packed(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("N", [1, 24])
def test_a_packed_cache_whose_offsets_pass_32_bits(dtype, N):
    import torch
    from paper_2506_04708_b200 import serving
    H, page, dim = 8, 64, 128
    c = _packed_case(5, dtype, [300], N, 8, H, dim, page, parent=inputs.topology(N, min(3, N - 1), 3), nan=False, spare=0)
    block = serving.packed_block_bytes(page, dim)
    pool = (2**32 + 2**28) // (H * block)
    big = [torch.zeros((pool, H, block), dtype=torch.uint8, device=DEV) for _ in range(2)]
    n = c["ck_packed"].shape[0]
    for b, name in zip(big, ("ck_packed", "cv_packed")):
        b[pool - n:] = c[name].to(DEV)
    want = ts._reference(c)
    c["table"] = c["table"] + (pool - n)
    _check(c, _run_packed(c, move=lambda q, k, v, ck, cv: (q, k, v, big[0], big[1])), want=want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("N,dim", [(1, 128), (24, 128), (8, 64)])
def test_packed_attention_gives_the_same_bits_every_time_and_on_another_stream(dtype, N, dim):
    import torch
    c = _packed_case(61, dtype, [900, 0, 333, 1800], N, 8, 2, dim, 16, parent=inputs.topology(N, min(6, N - 1), 3))
    first = _run_packed(c)
    for stream in (None, torch.cuda.Stream(), None):
        again = _run_packed(c, stream=stream)
        assert np.array_equal(first[0], again[0]) and np.array_equal(first[1], again[1])


@pytest.mark.gpu
def test_no_packed_cache_at_all_and_pages_of_the_largest_size():
    for dtype in ts.ALL_TYPES:
        for N in (1, 8):
            c = _packed_case(9, dtype, [0, 0], N, 4, 2, 64, 16, parent=inputs.topology(N, min(3, N - 1), 2), spare=0, cols=0)
            _check(c, _run_packed(c))
            c = _packed_case(9, dtype, [1, 4096, 5000], N, 4, 2, 64, 4096, parent=inputs.topology(N, min(3, N - 1), 2))
            _check(c, _run_packed(c))


# ---------------------------------------------------------------- bindings, streams, graphs
@pytest.mark.gpu
def test_bindings_refuse_wrong_tensors():
    import torch
    from paper_2506_04708_b200 import serving
    bf, f32 = torch.bfloat16, torch.float32
    z = lambda *s, dtype=bf, device=DEV: torch.zeros(s, dtype=dtype, device=device)  # noqa: E731
    Err = binding.StandError
    for bad in (dict(dim=72), dict(page_size=24), dict(dim=0)):
        d = dict(dict(dim=64, page_size=16), **bad)
        with pytest.raises(Err):
            serving.PackedTreeAttention(1, 2, 2, 2, d["dim"], bf, d["page_size"], 4, 4)
    plan = serving.PackedTreeAttention(1, 2, 2, 2, 64, bf, 16, 4, 4)
    q, cache = z(1, 2, 2, 64), z(4, 2, 576, dtype=torch.uint8)
    rest = z(1, 4, dtype=torch.int32), z(1, dtype=torch.int64)
    plan(q, q, q, cache, cache, *rest)
    for bad in (z(4, 2, 16, 64), z(4, 2, 16 * 64, dtype=torch.uint8), z(3, 2, 576, dtype=torch.uint8), cache.cpu(), z(4, 2, 580, dtype=torch.uint8)[..., :576],
                z(4, 576, 2, dtype=torch.uint8).transpose(1, 2), z(4 * 2 * 576 + 8, dtype=torch.uint8)[8:].view(4, 2, 576)):
        with pytest.raises(Err):
            plan(q, q, q, bad, bad, *rest)
    with pytest.raises(Err):
        plan(q, q, q, cache, z(4, 2, 592, dtype=torch.uint8)[..., :576], *rest)
    freq = z(32, dtype=f32)
    for bad in (dict(freq=z(32)), dict(freq=z(33, dtype=f32)), dict(freq=freq.cpu()), dict(freq=freq, offset=z(3, dtype=torch.int32)),
                dict(offset=z(2, dtype=torch.int32)), dict(weight_q=z(64)), dict(norm=True, weight_q=z(64, dtype=f32)), dict(norm=True, weight_k=z(32)),
                dict(norm=True, eps=0.0)):
        with pytest.raises(Err):
            serving.HeadRotation(1, 2, 2, 2, 64, bf, **bad)
    rot = serving.HeadRotation(1, 2, 2, 2, 64, bf, freq=freq)
    rot(q, q)
    for bad in (dict(q=z(1, 2, 2, 32)), dict(k=z(1, 2, 2, 64, dtype=f32)), dict(base=z(1, dtype=torch.int32)), dict(base=z(2, dtype=torch.int64)), dict(q=q.cpu()),
                dict(q_out=q.cpu()), dict(k_out=z(1, 2, 1, 64)), dict(q=z(1, 2, 64, 2).transpose(2, 3))):
        with pytest.raises(Err):
            rot(**dict(dict(q=q, k=q), **bad))
    for bad in (dict(dim=72), dict(page_size=8), dict(layers=0), dict(weight_k=z(64)), dict(norm=True, weight_k=z(64))):
        d = dict(dict(layers=1, dim=64, page_size=16), **bad)
        with pytest.raises(Err):
            serving.KvAppend(d.pop("layers"), 1, 2, 2, d.pop("dim"), bf, d.pop("page_size"), 4, 2, packed=True, **d)
    add, read = serving.KvAppend(1, 1, 2, 2, 64, bf, 16, 4, 2, packed=True), serving.KvRead(1, 1, 2, 64, bf, 16, 4, 2, packed=True)
    rows, slots, caches = z(1, 1, 2, 2, 64), z(1, 2, dtype=torch.int64) + torch.arange(2, device=DEV), z(1, 4, 2, 576, dtype=torch.uint8)
    add(rows, rows, slots, caches, caches.clone())
    read(slots, caches, caches)
    for bad in (dict(k=rows.cpu()), dict(v=z(1, 1, 2, 2, 64, dtype=f32)), dict(slots=slots.int()), dict(cache_k=z(1, 4, 2, 16, 64)), dict(path=slots),
                dict(base=slots[0, :1].int()), dict(cache_v=z(1, 4, 2, 592, dtype=torch.uint8)[..., :576])):
        with pytest.raises(Err):
            add(**dict(dict(k=rows, v=rows, slots=slots, cache_k=caches, cache_v=caches), **bad))
    for bad in (dict(slots=slots.int()), dict(cache_k=z(1, 4, 2, 16, 64)), dict(k=rows.cpu()), dict(v=rows.float()), dict(k=z(1, 1, 2, 64, 2).transpose(3, 4))):
        with pytest.raises(Err):
            read(**dict(dict(slots=slots, cache_k=caches, cache_v=caches), **bad))


@pytest.mark.gpu
def test_a_run_of_all_operators_in_a_graph():
    """Rotation, attention, append and read-back of a step, captured once and replayed as the texts grow: each replay equals the same calls made one
    by one, on another stream."""
    import torch
    from paper_2506_04708_b200 import serving
    B, N, hq, hkv, dim, page, cols, steps = 3, 4, 8, 2, 128, 16, 6, 12
    bf = torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(4)
    freq = (10000.0 ** (-torch.arange(64, device=DEV) / 64)).float()

    class Loop:
        def __init__(self):
            self.rot = serving.HeadRotation(B, N, hq, hkv, dim, bf, freq=freq, norm=True)
            self.att = serving.PackedTreeAttention(B, N, hq, hkv, dim, bf, page, B * cols, cols)
            self.map = serving.PageMap(B, N, page, cols, B * cols)
            self.add = serving.KvAppend(1, B, N, hkv, dim, bf, page, B * cols, N, packed=True, freq=freq, norm=True)
            self.read = serving.KvRead(1, B, hkv, dim, bf, page, B * cols, N, packed=True)
            self.cache = [torch.zeros((1, B * cols, hkv, serving.packed_block_bytes(page, dim)), dtype=torch.uint8, device=DEV) for _ in range(2)]
            self.table = torch.full((B, cols), -1, dtype=torch.int32, device=DEV)
            self.free, self.n_free = torch.arange(B * cols, dtype=torch.int32, device=DEV), torch.tensor([B * cols], dtype=torch.int32, device=DEV)
            self.len = torch.zeros(B, dtype=torch.int64, device=DEV)
            self.qkv = torch.zeros((B, N, hq + 2 * hkv, dim), dtype=bf, device=DEV)
            self.new = torch.zeros(B, dtype=torch.int32, device=DEV)

        def step(self):
            q, k, v = self.qkv.split([hq, hkv, hkv], 2)
            qr, kr = self.rot(q, k, self.len)
            out, lse = self.att(qr, kr, v, self.cache[0][0], self.cache[1][0], self.table, self.len)
            slots, granted, length, n_free = self.map(self.len, self.new, self.table, self.free, self.n_free)
            self.add(k[None], v[None], slots, self.cache[0], self.cache[1], base=self.len)
            back = self.read(slots, *self.cache)
            self.len.copy_(length)
            self.n_free.copy_(n_free)
            return out, lse, back[0], back[1]

    a, b = Loop(), Loop()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        res = a.step()
    for i in range(steps):
        x = torch.randn(a.qkv.shape, generator=g, device=DEV).to(bf)
        n = torch.tensor([i % 5, 4, 1], dtype=torch.int32, device=DEV)
        for loop in (a, b):
            loop.qkv.copy_(x)
            loop.new.copy_(n)
        graph.replay()
        want = b.step()
        torch.cuda.synchronize()
        for r, w in zip(res, want):
            assert torch.equal(r, w)
        assert torch.equal(a.cache[0], b.cache[0]) and torch.equal(a.cache[1], b.cache[1]) and torch.equal(a.len, b.len)
    # and the last step's rows are what attention over the values says
    vals = [torch.from_numpy(pref.block_values(c[0].cpu().numpy(), page, dim)) for c in b.cache]
    c = dict(qkv=torch.cat([b.rot.q_out, b.rot.k_out, b.qkv[:, :, hq + hkv:]], 2).cpu(), ck=vals[0], cv=vals[1], table=b.table.cpu().numpy(),
             len=(b.len - torch.tensor([(steps - 1) % 5, 4, 1], device=DEV)).cpu().numpy(), tree=None, parent=None, mask=None, hq=hq, hkv=hkv, dim=dim, page=page, N=N, dtype="bf16")
    _check(c, (want[0].double().cpu().numpy(), want[1].double().cpu().numpy()))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N,dim", [(1, 128), (2, 64), (4, 128), (24, 128), (24, 64), (9, 256)])
def test_packed_a_wait_that_runs_out_gives_nan_and_leaves_the_gpu_usable(lib, dtype, N, dim):
    c = _packed_case(71, dtype, [300, 20, 0], N, 4, 2, dim, 16, parent=inputs.topology(N, min(4, N - 1), 3))
    assert lib.stand_set_wait_limit(0) == 0
    try:
        out, lse = _run_packed(c)
    finally:
        lib.stand_set_wait_limit(-1)
    assert np.isnan(out).all() and np.isnan(lse).all()
    _check(c, _run_packed(c))


# ---------------------------------------------------------------- all of them together: examples/tree_decode.py
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,head_norm", [(1, False), (4, True)])
def test_a_decoding_loop_over_a_cache_in_4_bits(dtype, batch, head_norm):
    """Per step and layer, attention over the packed cache against attention over its values in a cache of the model's type (bfloat16
    and single precision hold them exactly): two kernels, each within u (|o| + sum p|v|) and single-precision sums of
    the definition, so within 4 u max |v| + 2^-12 max |v| of one another (scores here are below 2^5 and e below 2^-13)."""
    import torch
    from examples import tree_decode as td
    from paper_2506_04708_b200 import serving
    model = td.Model(dtype=ts._dtype(dtype), V=300, head_norm=head_norm)
    dec = td.Decoder(model, td.prompts_for(batch, model.V, seed=batch), most=256, packed=True)
    pool, page, L = dec.cache_k.shape[1], dec.page, model.layers
    every = serving.KvRead(L, 1, model.hkv, model.dim, model.dtype, page, pool, pool * page, packed=True)
    slots = torch.arange(pool * page, device=DEV)[None]
    plain = serving.TreeAttention(batch, dec.N, model.hq, model.hkv, model.dim, model.dtype, page, pool, dec.table.shape[1], parent=dec.parent)
    worst, deepest = 0.0, 0

    def attend(attention):
        caches = [c.view(L, pool, page, model.hkv, model.dim).transpose(2, 3) for c in every(slots, dec.cache_k, dec.cache_v)]

        def f(layer, q, k, v):
            nonlocal worst
            out = attention(q, k, v, dec.cache_k[layer], dec.cache_v[layer], dec.table, dec.len, tree_tokens=dec.seen)[0]
            want = plain(q, k, v, caches[0][layer], caches[1][layer], dec.table, dec.len, tree_tokens=dec.seen)[0]
            top = max(float(v.abs().max()), float(caches[1][layer].abs().max()))
            worst = max(worst, float((out.float() - want.float()).abs().max()) / top)
            return out
        return f
    dec.attend = attend
    for _ in range(16):
        _, _, n = dec.step()
        deepest = max(deepest, int(n.max()))
    assert worst <= 4 * ts.U[dtype] + 2.0**-12, worst
    assert deepest >= 2 or batch == 1
    assert torch.equal(dec.len + 1, dec.n_text) and not dec.short.any()
    # the cache holds what the model's keys are, in 4 bits: the text run through the first layer's projections
    n = int(dec.len[0])
    tokens, pos = dec.text[:1, :n], torch.arange(n, device=DEV)[None]
    qkv = (model.norm(model.embed[tokens.long()]) @ model.blocks[0]["qkv"]).unflatten(-1, (-1, model.dim))
    q, k, v = qkv.split([model.hq, model.hkv, model.hkv], 2)
    w = None if not head_norm else model.weight_k[0]
    turned = serving.HeadRotation(1, n, model.hq, model.hkv, model.dim, model.dtype, freq=model.freq, interleaved=True, norm=head_norm, weight_q=w, weight_k=w)(q, k)[1]
    at = dec.table[0, pos[0] // page].long() * page + pos[0] % page
    read = serving.KvRead(L, 1, model.hkv, model.dim, torch.float32, page, pool, n, packed=True)
    got = read(at[None], dec.cache_k, dec.cache_v)
    for rows, x in ((got[0][0, 0], turned[0]), (got[1][0, 0], v[0])):
        want = torch.from_numpy(pref.values(*pref.pack(x.float().cpu().numpy()))).to(DEV)
        # products of other shapes may round otherwise: a code may differ by one there, and few do
        step = want.abs().unflatten(-1, (-1, 16)).amax(-1, keepdim=True).expand(*want.shape[:-1], -1, 16).flatten(-2) / 7 * 1.26
        assert ((rows - want).abs() <= step + 1e-12).all() and float(((rows - want).abs() > 1e-6).double().mean()) < 0.05


# ---------------------------------------------------------------- at the ends
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("B", [193, 700])
@pytest.mark.parametrize("N,dim", [(1, 64), (1, 128), (3, 64), (20, 128)])
def test_packed_batches_of_more_sequences_than_threads(dtype, B, N, dim):
    """Many short texts, among them empty ones: a range of tiles covers dozens of sequences."""
    rng = np.random.default_rng(B)
    lens = [int(n) for n in np.where(rng.random(B) < 0.2, 0, rng.integers(1, 90 if N < 20 else 40, B))]
    lens[B // 2] = 700
    c = _packed_case(B, dtype, lens, N, 4, 2, dim, 16, parent=inputs.topology(N, min(2, N - 1), 4 if N > 3 else 2), nan=False)
    _check(c, _run_packed(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,size,scale", [("bf16", 2.0**-40, 2.0**37), ("bf16", 2.0**80, 2.0**-83), ("f16", 2.0**-8, 2.0**5), ("f16", 2.0**10, 2.0**-13), ("f32", 2.0**60, 2.0**-63)])
@pytest.mark.parametrize("N,hq,dim", [(1, 4, 128), (1, 4, 64), (3, 8, 128), (24, 8, 64)])
def test_packed_queries_of_any_size(dtype, size, scale, N, hq, dim):
    """Queries far from 1, rows of different sizes, elements of a row 2^-12 times the others: the scores are ordinary ones."""
    c = _packed_case(91, dtype, [300, 5, 0], N, hq, 2, dim, 16, parent=inputs.topology(N, min(3, N - 1), 3), nan=False)
    q = c["qkv"][:, :, :hq].float()
    q[..., ::3] *= 2.0**-12 if dtype != "f16" else 2.0**-4
    q[:, :, 1] *= 2.0**-3
    c["qkv"][:, :, :hq] = (q * size).to(c["qkv"].dtype)
    _check(c, _run_packed(c, scale=scale), want=ts._reference(c, scale))


@pytest.mark.gpu
def test_launches_of_all_packed_kernels_in_a_row_and_on_two_streams():
    """Launches that follow one another closely, of the kernels with and without tensor memory, over packed caches and others, on two streams at
    the same time: the same bits as each by itself."""
    import torch
    from paper_2506_04708_b200 import serving
    work = []
    for i, (dim, N, hq, hkv, packed) in enumerate(((64, 8, 4, 2, True), (128, 24, 8, 2, True), (128, 1, 8, 2, True), (256, 9, 4, 2, True), (64, 40, 4, 2, False),
                                                   (80, 3, 2, 1, True), (64, 1, 8, 8, True), (128, 4, 8, 2, True), (128, 24, 8, 2, False))):
        c = _packed_case(i, "bf16", [700, 0, 129, 3000], N, hq, hkv, dim, 16, parent=inputs.topology(N, min(4, N - 1), 3), nan=False)
        qkv = c["qkv"].to(DEV)
        caches = [c[n + "_packed"].to(DEV) if packed else c[n].to(torch.bfloat16).to(DEV) for n in ("ck", "cv")]
        args = (qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:], *caches, torch.from_numpy(c["table"]).to(DEV), torch.from_numpy(c["len"]).to(DEV))
        kind = serving.PackedTreeAttention if packed else serving.TreeAttention
        plans = [kind(4, N, hq, hkv, dim, torch.bfloat16, 16, caches[0].shape[0], args[5].shape[1], parent=c["parent"]) for _ in range(2)]
        alone = [t.clone() for t in plans[0](*args)]
        torch.cuda.synchronize()
        _check(c, tuple(t.double().cpu().numpy() for t in alone))
        work.append((args, plans, alone))
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(20):
        for args, plans, _ in work:
            for plan, stream in zip(plans, streams):
                plan(*args, stream=stream)
        torch.cuda.synchronize()
        for _, plans, alone in work:
            for plan in plans:
                assert torch.equal(plan.out, alone[0]) and torch.equal(plan.lse, alone[1])
                plan.out.fill_(7)
        torch.cuda.synchronize()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N,hq,hkv,dim", [(1, 4, 1, 128), (3, 4, 1, 64), (5, 6, 2, 128), (9, 6, 2, 64), (64, 7, 1, 128), (7, 3, 1, 96), (3, 2, 1, 256)])
def test_packed_results_do_not_depend_on_what_shared_memory_held(dtype, N, hq, hkv, dim):
    """Rows that do not fill their tiles, after launches whose queries and keys leave large scores, infinities and NaN behind."""
    import torch
    from paper_2506_04708_b200 import serving
    c = _packed_case(dim * N, dtype, [700, 40, 2000], N, hq, hkv, dim, 16, parent=inputs.topology(N, min(4, N - 1), 3), nan=False)
    c["qkv"][:, :, :hq] *= 3
    qkv, ck, cv = c["qkv"].to(DEV), c["ck_packed"].to(DEV), c["cv_packed"].to(DEV)
    table, length = torch.from_numpy(c["table"]).to(DEV), torch.from_numpy(c["len"]).to(DEV)
    dt = ts._dtype(dtype)
    plan = serving.PackedTreeAttention(3, N, hq, hkv, dim, dt, 16, ck.shape[0], table.shape[1], parent=c["parent"])
    spoilers = [serving.PackedTreeAttention(3, n, hq, hkv, dim, dt, 16, ck.shape[0], table.shape[1]) for n in (128 // (hq // hkv), max(1, 16 // (hq // hkv)))]
    first = None
    for fill in (0.0, 1.0, -30.0, 1000.0, float("inf"), float("nan")):
        for s in spoilers:
            q = torch.full((3, s.out.shape[1], hq, dim), fill, dtype=dt, device=DEV)
            kv = torch.full((3, s.out.shape[1], hkv, dim), fill, dtype=dt, device=DEV)
            s(q, kv, kv, ck, cv, table, length)
        out, lse = plan(qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:], ck, cv, table, length)
        if first is None:
            first = out.clone(), lse.clone()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1]), fill
    _check(c, tuple(t.double().cpu().numpy() for t in first))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("N,dim", [(1, 128), (24, 128), (4, 64)])
def test_one_undrafted_nodes_queries_do_not_touch_other_rows(dtype, N, dim):
    """What queries of undrafted nodes hold changes no bit of the other rows."""
    import torch
    c = _packed_case(33, dtype, [700, 90], N, 8, 2, dim, 16, parent=inputs.topology(N, min(4, N - 1), 3), nan=False)
    c["tree"] = np.zeros((2, N), np.int32)
    c["tree"][:, N // 2:] = -1
    want = None
    for fill in (0.0, 3.0, 1000.0, float("nan"), float("inf")):
        c["qkv"][:, N // 2:, :8] = fill
        got = _run_packed(c)
        want = got if want is None else want
        assert np.array_equal(got[0][:, :N // 2], want[0][:, :N // 2]) and np.array_equal(got[1][:, :N // 2], want[1][:, :N // 2])
        assert not got[0][:, N // 2:].any() and np.isneginf(got[1][:, N // 2:]).all()


def test_rotations_of_too_many_tokens_are_refused(lib):
    assert lib.stand_rotate_heads(C.byref(_rotation(B=1 << 16, N=1 << 16)), A, A, A, A, A, A, A, A, A, None) == -1


@pytest.mark.gpu
def test_rotation_and_append_of_many_tokens_of_short_sequences():
    """One node per sequence (every token another sequence), and heads so many that a block takes some of them."""
    import torch
    from paper_2506_04708_b200 import serving
    freq = (10000.0 ** (-np.arange(32) / 32)).astype(np.float32)
    for B, N, hq, hkv in ((5000, 1, 2, 1), (3, 1, 300, 100), (700, 3, 8, 8)):
        x = torch.randn((B, N, hq + hkv, 64), device=DEV)
        base = torch.randint(0, 100000, (B,), device=DEV)
        q, k = serving.HeadRotation(B, N, hq, hkv, 64, torch.float32, freq=_dev(freq), norm=True)(x[:, :, :hq], x[:, :, hq:], base)
        pos = _where(base.cpu().numpy(), None, B, N)[..., None]
        want, size = pref.rotate(x.double().cpu().numpy(), pos, freq, False, None, 1e-6)
        _near(torch.cat([q, k], 2).double().cpu().numpy(), want, size, "f32", True)


@pytest.mark.gpu
def test_rotation_offsets_pass_32_bits():
    """Rows more than 2^31 elements apart."""
    import torch
    from paper_2506_04708_b200 import serving
    big = torch.zeros(2**31 + 2**20, dtype=torch.bfloat16, device=DEV)
    rows = torch.as_strided(big, (2, 3, 2, 64), (2**31, 256, 64, 1))
    x = torch.randn((2, 3, 2, 64), device=DEV).bfloat16()
    rows.copy_(x)
    freq = torch.ones(32, device=DEV)
    op = serving.HeadRotation(2, 3, 2, 2, 64, torch.bfloat16, freq=freq)
    want = [t.clone() for t in op(x, x)]
    got = op(rows, rows)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    op(x, x, q_out=rows, k_out=rows)
    assert torch.equal(rows, want[0]) and not big[2**20:2**31 - 2**20].any()


@pytest.mark.gpu
def test_a_refused_rotation_leaves_the_next_call_as_it_was():
    """Strides of a call whose last argument is refused are forgotten with it."""
    import torch
    from paper_2506_04708_b200 import serving
    x = torch.randn((2, 3, 4, 64), device=DEV)
    op = serving.HeadRotation(2, 3, 4, 4, 64, torch.float32, freq=torch.ones(32, device=DEV))
    want = [t.clone() for t in op(x, x)]
    wide = torch.randn((2, 3, 8, 64), device=DEV)[:, :, ::2]
    with pytest.raises(binding.StandError):
        op(wide, x, k_out=torch.zeros((2, 3, 64, 4), device=DEV).transpose(2, 3))
    got = op(x, x)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.gpu
def test_expanded_tensors_are_read_but_not_written():
    import torch
    from paper_2506_04708_b200 import serving
    x = torch.randn((2, 1, 1, 64), device=DEV)
    many = x.expand(2, 3, 4, 64)
    op = serving.HeadRotation(2, 3, 4, 4, 64, torch.float32, freq=torch.ones(32, device=DEV))
    want = [t.clone() for t in op(many.contiguous(), many.contiguous())]
    got = op(many, many)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    for bad in (dict(q_out=many), dict(k_out=many)):
        with pytest.raises(binding.StandError):
            op(many, many, **bad)
    slots = torch.arange(6, device=DEV).view(2, 3)
    for packed, shape, dtype in ((False, (1, 1, 64, 64), torch.float32), (True, (1, 1, 2304), torch.uint8)):
        add = serving.KvAppend(1, 2, 3, 4, 64, torch.float32, 64, 1, 3, packed=packed)
        cache = torch.zeros((1,) + shape, dtype=dtype, device=DEV).expand((1, 1, 4) + shape[2:])
        with pytest.raises(binding.StandError):
            add(many[None], many[None], slots, cache, cache.clone(memory_format=torch.contiguous_format))
        assert not cache.any()


@pytest.mark.gpu
@pytest.mark.parametrize("packed", [False, True])
def test_rows_at_multiples_of_16_bytes_that_are_none_of_32(packed):
    """Sources and results whose rows begin 16 bytes behind a multiple of 32 (accesses are narrower there) give the same."""
    import torch
    from paper_2506_04708_b200 import serving
    dt, L, B, N, H, D = torch.bfloat16, 3, 2, 5, 2, 64
    shape, slots = (L, B, N, H, D), torch.arange(10, device=DEV).view(B, N)

    def shifted(x=None):
        t = torch.empty(L * B * N * H * D + 8, dtype=dt, device=DEV)[8:].view(shape)
        return t if x is None else t.copy_(x)

    k, v = (torch.randn(shape, device=DEV).to(dt) for _ in range(2))
    add = serving.KvAppend(L, B, N, H, D, dt, 16, 1, N, packed=packed)
    back = serving.KvRead(L, B, H, D, dt, 16, 1, N, packed=packed)
    cache = [torch.zeros((L, 1, H, 576) if packed else (L, 1, H, 16, D), dtype=torch.uint8 if packed else dt, device=DEV) for _ in range(4)]
    add(k, v, slots, *cache[:2])
    add(shifted(k), shifted(v), slots, *cache[2:])
    assert torch.equal(cache[0], cache[2]) and torch.equal(cache[1], cache[3])
    want = [t.clone() for t in back(slots, *cache[:2])]
    got = back(slots, *cache[:2], k=shifted(), v=shifted())
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    if not packed:
        assert torch.equal(got[0], k) and torch.equal(got[1], v)
