"""The operators around the decoding step at the ends of their arguments: bounds, devices, values that are not finite, small
weights, layouts, aliases, streams.  Tolerances as in test_serving.py unless a test derives its own.
"""
import os
import subprocess

import numpy as np
import pytest

from paper_2506_04708_b200 import binding, build as lib_build, inputs
from tests import test_serving as ts

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


# ---------------------------------------------------------------- the visibility mask
@pytest.fixture(scope="module")
def bounds_program(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("bounds") / "attention_bounds")
    subprocess.run([lib_build.NVCC, "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-o", exe,
                    os.path.join(ROOT, "tests", "attention_bounds.cu")], check=True)
    return exe


@pytest.mark.parametrize("N,group", [(1, 1), (64, 7), (200, 2), (513, 1), (33, 5), (640, 1), (640, 5), (18, 7), (19, 7), (3, 128), (2, 130), (65, 3)])
@pytest.mark.parametrize("own", [0, 1])
def test_the_mask_is_read_for_existing_nodes_only(bounds_program, N, group, own):
    """Both kernels ask attn_nodes_seen for each row of their row tiles, rows beyond the last node among them.  The mask ends
    where the mapping does; the words are those of the definition."""
    for masked in (1, 0):
        run = subprocess.run([bounds_program, str(N), str(group), "3", str(own), str(masked)], capture_output=True, text=True, timeout=60)
        assert run.returncode == 0, (run.returncode, run.stdout)


# ---------------------------------------------------------------- result tensors
class _Tensor:
    """What the binding asks of a tensor, without a device."""

    def __init__(self, shape, dtype, device=0, contiguous=True, stride=None):
        steps = [1]
        for n in reversed(shape[1:]):
            steps.insert(0, steps[0] * n)
        self.shape, self.dtype, self.device, self._d, self._c, self._s = tuple(shape), dtype, device, device, contiguous, stride or tuple(steps)

    def get_device(self):
        return self._d

    def is_contiguous(self):
        return self._c

    def stride(self):
        return self._s

    def data_ptr(self):
        return 0x1000


def _hostless_attention(B=1, N=4, hq=2, hkv=2, dim=64, page=16, pages=4, cols=4):
    """A TreeAttention whose launches are counted, not made, and the arguments of a call that it takes."""
    import ctypes as C

    import torch
    from paper_2506_04708_b200 import serving
    bf = torch.bfloat16
    p = object.__new__(serving.TreeAttention)
    p.torch, p.dtype, p.dev, p._index = torch, bf, "cuda:0", 0
    p.cfg = binding.StandAttention(B, N, hq, hkv, dim, binding.DTYPE_BF16, page, pages, cols, 0.125)
    p._cfg_ptr, p._strides, p._mask_ptr, p.mask_stride, p._scratch, p._scratch_bytes = C.addressof(p.cfg), None, None, 0, 0, 0
    p._q_shape, p._kv_shape, p._cache_shape = (B, N, hq, dim), (B, N, hkv, dim), (pages, hkv, page, dim)
    p._table_shape, p._len_shape, p._tree_shape = (B, cols), (B,), (B, N)
    p.out, p.lse = _Tensor(p._q_shape, bf), _Tensor((B, N, hq), torch.float32)
    p._lib = type("Lib", (), {"stand_tree_attention": None})
    p.launches = 0

    def launch(*a):
        p.launches += 1
    p._launch = launch
    args = [_Tensor(p._q_shape, bf)] + [_Tensor(p._kv_shape, bf) for _ in range(2)] + [_Tensor(p._cache_shape, bf) for _ in range(2)]
    return p, args + [_Tensor((B, cols), torch.int32), _Tensor((B,), torch.int64)]


def test_results_go_to_this_device_only():
    """An `out` or `lse` on the CPU or another GPU, of another type or shape, or with gaps is refused before a launch."""
    import torch
    p, args = _hostless_attention()
    bf, f32, q, rows = torch.bfloat16, torch.float32, p._q_shape, (1, 4, 2)
    p(*args)
    p(*args, out=_Tensor(q, bf), lse=_Tensor(rows, f32))
    assert p.launches == 2
    for bad in (dict(out=_Tensor(q, bf, device=-1)), dict(out=_Tensor(q, bf, device=1)), dict(out=_Tensor(q, torch.float16)),
                dict(out=_Tensor((1, 4, 2, 32), bf)), dict(out=_Tensor(q, bf, contiguous=False)), dict(lse=_Tensor(rows, f32, device=-1)),
                dict(lse=_Tensor(rows, f32, device=1)), dict(lse=_Tensor(rows, bf)), dict(lse=_Tensor((1, 4), f32)),
                dict(lse=_Tensor(rows, f32, contiguous=False))):
        with pytest.raises(binding.StandError):
            p(*args, **bad)
    assert p.launches == 2


@pytest.mark.gpu
def test_results_on_the_host_are_refused():
    import torch
    from paper_2506_04708_b200 import serving
    dev = "cuda:0"
    plan = serving.TreeAttention(1, 4, 2, 2, 64, torch.bfloat16, 16, 4, 4)
    q, cache = torch.zeros((1, 4, 2, 64), dtype=torch.bfloat16, device=dev), torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16, device=dev)
    args = q, q, q, cache, cache, torch.zeros((1, 4), dtype=torch.int32, device=dev), torch.zeros(1, dtype=torch.int64, device=dev)
    for bad in (dict(out=torch.empty(q.shape, dtype=q.dtype)), dict(out=torch.empty(q.shape, device=dev)), dict(lse=torch.empty((1, 4, 2)))):
        with pytest.raises(binding.StandError):
            plan(*args, **bad)
    mine = torch.full_like(q, 7)
    out, _ = plan(*args, out=mine)
    assert out is mine and not mine.any()


# ---------------------------------------------------------------- cached values that are not finite
def _plant(c, b, pos, head, element, value):
    c["cv"][int(c["table"][b, pos // c["page"]]), head, pos % c["page"], element] = value


def _check_planted(c, clean, hits, got):
    """hits: (sequence, element, key head, value): what that element of all rows of these heads has to be."""
    out, lse = got
    group, hit = c["hq"] // c["hkv"], np.zeros_like(out, bool)
    for b, d, g, value in hits:
        rows = out[b, :, g * group:(g + 1) * group, d]
        assert (np.isnan(rows) if np.isnan(value) else rows == value).all(), (b, d, g, value, rows)
        hit[b, :, g * group:(g + 1) * group, d] = True
    ts._check_attention(c, (np.where(hit, clean[0], out), lse), want=clean)


INF, NAN = float("inf"), float("nan")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("N,hq,hkv,dim", [(3, 2, 2, 64), (24, 4, 2, 64), (33, 4, 2, 64), (24, 3, 1, 40), (8, 8, 2, 128), (5, 2, 1, 256)])
def test_cached_values_that_are_not_finite(dtype, N, hq, hkv, dim):
    """One infinity, two of a sign, two of opposite signs, a NaN: in all forms of the kernels the element is what the sum is.
    (Rows of heads up to 64 are held several times, for parts of the keys: an infinity in one part is no NaN in another.)"""
    c = ts._attention_case(dim + N, dtype, [1, 70, 300], N, hq, hkv, dim, 16, parent=inputs.topology(N, 2, 6))
    clean, g = ts._reference(c), hkv - 1
    hits = [(0, 0, 0, -INF)]
    _plant(c, 0, 0, 0, 0, -INF)
    for pos in (3, 69):
        _plant(c, 1, pos, g, 5, INF)
    hits.append((1, 5, g, INF))
    for pos, value in ((17, INF), (200, -INF)):
        _plant(c, 2, pos, g, 6, value)
    hits.append((2, 6, g, NAN))
    _plant(c, 2, 250, 0, 7, NAN)
    hits.append((2, 7, 0, NAN))
    for pos in range(300):
        _plant(c, 2, pos, 0, 9, -INF)
    hits.append((2, 9, 0, -INF))
    _check_planted(c, clean, hits, ts._run_attention(c))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("hq,hkv,dim", [(2, 2, 64), (4, 1, 128)])
def test_infinities_whose_weight_is_below_the_type(dtype, hq, hkv, dim):
    """Scores rise by 260 nats along a text that is cut into pieces: a 32-bit weight of its early tokens is zero, the definition's is not."""
    n = 3000
    c = ts._attention_case(7, dtype, [n, 100], 4, hq, hkv, dim, 16, parent=inputs.topology(4, 2, 2), nan=False)
    c["qkv"][0, :, :hq] = 0
    c["qkv"][0, :, :hq, 0] = 4.0
    c["qkv"][0, :, hq:hq + hkv] = 0  # the nodes' scores are in the middle of it
    for pos in range(n):
        c["ck"][int(c["table"][0, pos // 16]), :, pos % 16, 0] = (pos / n - 0.5) * 260.0 / 4.0
    clean = ts._reference(c, scale=1.0)
    hits = []
    for d, (pos, value) in enumerate([(0, INF), (40, -INF), (700, INF), (2990, -INF), (1500, NAN)]):
        _plant(c, 0, pos, 0, 2 * d, value)
        hits.append((0, 2 * d, 0, value))
    _plant(c, 0, 5, 0, 21, INF)
    _plant(c, 0, 2995, 0, 21, -INF)
    hits.append((0, 21, 0, NAN))
    _check_planted(c, clean, hits, ts._run_attention(c, scale=1.0))


# ---------------------------------------------------------------- small weights of half precision
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("n,N,hq,hkv,dim,B", [(40000, 1, 2, 2, 64, 24), (40000, 4, 4, 1, 128, 40), (9000, 40, 1, 1, 64, 150), (20000, 1, 1, 1, 256, 60)])
@pytest.mark.parametrize("last", [False, True])
def test_many_small_weights_beside_a_dominant_one(dtype, n, N, hq, hkv, dim, B, last):
    """One key takes nearly all weight and has the value 0; tens of thousands of others, near 2^-26 of it each, make the result.
    So many sequences (over the same pages) that thousands of keys are summed relative to the dominant one.  Half: none of them may be lost.  Tolerance of test_serving.py with weights that keep all bits down to 2^-21 and 2^-32 of the
    largest weight below that: 2^-32 sum |v| in place of 2^-25 sum |v|."""
    c = ts._attention_case(n + dim, dtype, [n], N, hq, hkv, dim, 64, parent=inputs.topology(N, 3, 4), nan=False)
    rng = np.random.default_rng(5)
    import torch
    c["qkv"][:] = 0
    c["qkv"][:, :, :hq, 0] = 4.0
    c["qkv"][:, :, hq:hq + hkv, 0] = -10.0  # the nodes themselves: next to nothing
    flat = torch.from_numpy((-26 * np.log(2.0) / 4 + 0.05 * rng.standard_normal(n)).astype(np.float32))
    at = n - 1 if last else 3
    flat[at] = 0.0
    ids = torch.from_numpy(c["table"][0].astype(np.int64))
    keys = torch.zeros((len(ids) * 64,))
    keys[:n] = flat
    c["ck"][:] = 0
    c["ck"][ids, :, :, 0] = keys.view(-1, 64)[:, None].expand(-1, hkv, -1).to(c["ck"].dtype)
    c["cv"] = (1 + 0.25 * c["cv"].float()).to(c["cv"].dtype)
    c["cv"][int(c["table"][0, at // 64]), :, at % 64] = 0
    r_out, r_lse, weight, spread, reach = ts._reference(c, scale=1.0)
    c.update(len=c["len"].repeat(B), table=c["table"].repeat(B, 0), qkv=c["qkv"].expand(B, -1, -1, -1).contiguous())
    out, lse = ts._run_attention(c, scale=1.0)
    u, e = ts.U[dtype], (dim + 8) * 2.0**-24 * reach
    lost = 2.0**-32 * spread if dtype == "f16" else 0
    tol = u * np.abs(r_out) + (u + 2 * e[..., None] + 2.0**-19) * weight + lost
    if dtype == "f16":
        tol = np.maximum(tol, 2.0**-25)  # the result's own type
    assert np.median(np.abs(r_out)) > 1e-4
    assert (np.abs(out - r_out) <= tol).all(), np.max(np.abs(out - r_out) / tol)
    assert (np.abs(lse - r_lse) <= e + 2.0**-19 * (1 + np.abs(r_lse))).all()


# ---------------------------------------------------------------- layouts of keys and values
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("how", ["rotated keys", "rotated keys, odd", "head-major values", "one value row for all heads"])
def test_keys_and_values_of_different_layouts(dtype, how):
    """Keys in a tensor of their own after a rotation, values still a slice of the projection, and the like."""
    import torch
    c = ts._attention_case(131, dtype, [0, 90, 300], 24, 4, 2, 64, 16, parent=inputs.topology(24, 6, 3), nan=False)
    if how == "one value row for all heads":
        c["qkv"][:, :, 5] = c["qkv"][:, :, 4]
        c["qkv"][:, :, 6:] = c["qkv"][:, :, 6:7]
    heads = 2 if how == "one value row for all heads" else 1  # value heads with an infinity: those are read again at the end
    clean = dict(c, qkv=c["qkv"].clone())
    clean["qkv"][1, 3, 6:6 + heads, 5] = 0.0
    c["qkv"][1, 3, 6:6 + heads, 5] = INF

    def move(q, k, v, ck, cv):
        if how == "rotated keys":
            return q, k.contiguous(), v, ck, cv
        if how == "rotated keys, odd":
            wide = torch.empty(k.shape[:-1] + (k.shape[-1] + 5,), dtype=k.dtype, device=k.device)[..., 2:-3]
            return q, wide.copy_(k), v, ck, cv
        if how == "head-major values":
            return q, k, v.transpose(1, 2).contiguous().transpose(1, 2), ck, cv
        return q, k, v[:, :, :1].contiguous().expand(-1, -1, 2, -1), ck, cv

    out, lse = ts._run_attention(c, move=move)
    want = ts._reference(clean)
    hit = np.zeros_like(out, bool)
    hit[1, ts.ref.ancestors(c["parent"])[:, 3], :2 * heads, 5] = True
    assert (out[hit] == INF).all()
    ts._check_attention(c, (np.where(hit, want[0], out), lse), want=want)


@pytest.mark.gpu
def test_strides_of_single_elements_do_not_matter():
    """Dimensions of one element may have any stride: one sequence, one node, one key head, one page, a head size of one."""
    import torch
    from paper_2506_04708_b200 import serving
    for dim in (64, 1):
        c = ts._attention_case(17 + dim, "bf16", [13], 1, 2, 1, dim, 16, parent=np.array([-1], np.int32), spare=0, nan=False)

        def odd(x):
            return torch.as_strided(x.contiguous(), x.shape, [s if n > 1 else 7 * s + 3 for n, s in zip(x.shape, x.contiguous().stride())])

        def move(q, k, v, ck, cv):
            return q, odd(k), v, odd(ck), cv
        ts._check_attention(c, ts._run_attention(c, move=move))


def test_strides_are_given_for_keys_and_values_apart():
    import torch
    bf = torch.bfloat16
    p, args = _hostless_attention(B=2, N=3)
    args[0], args[1] = _Tensor((2, 3, 2, 64), bf, stride=(2400, 800, 64, 1)), _Tensor((2, 3, 2, 64), bf, stride=(384, 128, 64, 1))
    args[2] = _Tensor((2, 3, 2, 64), bf, stride=(2400, 800, 64, 1))
    p(*args)
    assert list(p.cfg.kv_stride) == [384, 128, 64] and list(p.cfg.v_stride) == [2400, 800, 64] and p.cfg.own_v_stride == 1
    for i in (0, 1, 2, 3, 4):  # elements that do not lie side by side
        bad = list(args)
        bad[i] = _Tensor(args[i].shape, bf, stride=(9000, 3000, 1, 2))
        with pytest.raises(binding.StandError):
            p(*bad)
    bad = list(args)
    bad[4] = _Tensor(args[4].shape, bf, stride=(4096, 2048, 64, 1))
    with pytest.raises(binding.StandError):
        p(*bad)


def test_value_strides_are_checked():
    lib_build.build()
    import ctypes as C
    size = binding.lib().stand_tree_attention_scratch_bytes
    good = ts._shape()
    assert size(C.byref(good)) > 0
    good.own_v_stride = 1
    assert size(C.byref(good)) > 0
    for field, value in (("own_v_stride", 2), ("own_v_stride", -1), ("reserved", 1)):
        bad = ts._shape()
        setattr(bad, field, value)
        assert size(C.byref(bad)) == 0
    bad = ts._shape()
    bad.own_v_stride, bad.v_stride[2] = 1, -3
    assert size(C.byref(bad)) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("how", ["slice of a projection", "head-major", "odd rows", "one row for all heads"])
def test_commit_of_keys_and_values_of_different_layouts(dtype, how):
    import torch
    from paper_2506_04708_b200 import serving
    L, B, N, H, D, page, pool, width = 3, 2, 9, 3, 24, 16, 5, 4
    rng = np.random.default_rng(8)
    dt = ts._dtype(dtype)
    make = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(dt).to("cuda:0")  # noqa: E731
    k, ck, cv = make(L, B, N, H, D), make(L, pool, H, page, D), make(L, pool, H, page, D)
    v = {"slice of a projection": lambda: make(L, B, N, 3 * H, D)[:, :, :, 2 * H:], "head-major": lambda: make(L, B, H, N, D).transpose(2, 3),
         "odd rows": lambda: make(L, B, N, H, D + 3)[..., 1:-2], "one row for all heads": lambda: make(L, B, N, 1, D).expand(-1, -1, -1, H, -1)}[how]()
    slots = rng.permutation(pool * page)[: B * width].reshape(B, width).astype(np.int64)
    path = np.sort(rng.integers(0, N, (B, width)), 1).astype(np.int32)
    want = [ts.ref.kv_commit(s.float().cpu().numpy(), path, slots, c.float().cpu().numpy()) for s, c in ((k, ck), (v, cv))]
    op = serving.KvCommit(L, B, N, H, D, dt, page, pool, width)
    op(k, v, torch.from_numpy(slots).to("cuda:0"), ck, cv, path=torch.from_numpy(path).to("cuda:0"))
    assert np.array_equal(ck.float().cpu().numpy(), want[0]) and np.array_equal(cv.float().cpu().numpy(), want[1])
    for bad in ((k, v, ck, cv.transpose(2, 3).contiguous().transpose(2, 3)), (k.transpose(3, 4).contiguous().transpose(3, 4), v, ck, cv)):
        with pytest.raises(binding.StandError):
            op(bad[0], bad[1], torch.from_numpy(slots).to("cuda:0"), bad[2], bad[3])


def test_commit_value_strides_are_checked():
    lib_build.build()
    import ctypes as C
    at = C.c_void_p(0x100000)  # never touched: every call here is refused before a launch
    for fields in (dict(own_v_stride=2), dict(own_v_stride=-1), dict(reserved2=1), dict(own_v_stride=1, v=(0, 0, -1, 0))):
        s = binding.StandKvShape(1, 1, 4, 2, 64, 1, 16, 3, 2, 0)
        s.v_stride[:] = fields.pop("v", (0, 0, 0, 0))
        for name, value in fields.items():
            setattr(s, name, value)
        assert binding.lib().stand_kv_commit(C.byref(s), at, at, None, at, at, at, None) == -1


# ---------------------------------------------------------------- page maps: arrays that overlap
def test_page_maps_refuse_outputs_that_overlap_inputs():
    """Each array at a place of its own, then one output laid over an input, whole or in part: refused before a launch."""
    import ctypes as C
    lib_build.build()
    L = binding.lib()
    at = {n: 0x100000 * (i + 1) for i, n in enumerate(("length", "new", "free", "n_free", "table", "slots", "granted", "len_out", "n_out", "done"))}
    B = 5

    def page_map(**kw):
        p = {k: C.c_void_p(v) for k, v in dict(at, **kw).items()}
        return L.stand_page_map(p["length"], p["new"], B, 3, 16, 4, p["free"], 9, p["n_free"], p["table"], p["slots"], p["granted"], p["len_out"],
                                p["n_out"], None)

    def release(**kw):
        p = {k: C.c_void_p(v) for k, v in dict(at, **kw).items()}
        return L.stand_page_release(p["length"], p["done"], B, 16, 4, p["table"], 9, p["free"], p["n_free"], p["len_out"], p["n_out"], None)

    for bad in (dict(granted=at["new"]), dict(granted=at["new"] + 4), dict(granted=at["new"] - 16), dict(granted=at["n_free"]),
                dict(granted=at["n_free"] - 16), dict(len_out=at["length"]), dict(len_out=at["length"] + 32), dict(n_out=at["n_free"]),
                dict(n_out=at["new"] + 16)):
        assert page_map(**bad) == -1, bad
    for bad in (dict(len_out=at["length"]), dict(len_out=at["length"] - 32), dict(n_out=at["n_free"]), dict(n_out=at["done"] + 16)):
        assert release(**bad) == -1, bad


@pytest.mark.gpu
def test_granted_counts_are_no_request():
    """What a map granted may not be the next call's request in place; a copy of it may.  Neighbours in memory are no overlap."""
    import torch
    from paper_2506_04708_b200 import serving
    dev = "cuda:0"
    plan = serving.PageMap(4, 3, 16, 4, 8)
    i32, i64 = dict(dtype=torch.int32, device=dev), dict(dtype=torch.int64, device=dev)
    table, free, n_free = torch.full((4, 4), -1, **i32), torch.arange(8, **i32), torch.full((1,), 8, **i32)
    _, granted, length, n_free = plan(torch.zeros(4, **i64), torch.full((4,), 2, **i32), table, free, n_free)
    with pytest.raises(binding.StandError):
        plan(length, granted, table, free, n_free)
    _, again, length, n_free = plan(length, granted.clone(), table, free, n_free)
    assert again.tolist() == [2] * 4 and length.tolist() == [4] * 4 and int(n_free) == 4
    both = torch.full((8,), 2, **i32)
    plan.granted = both[4:]
    assert plan(length, both[:4], table, free, n_free)[1].tolist() == [2] * 4


# ---------------------------------------------------------------- streams
@pytest.mark.gpu
def test_objects_made_on_a_busy_stream_and_used_on_another():
    """Nothing that making an object queues on the current stream may run after, and over, a call on another stream."""
    import torch
    from paper_2506_04708_b200 import serving
    dev = "cuda:0"
    i32, i64 = dict(dtype=torch.int32, device=dev), dict(dtype=torch.int64, device=dev)
    table, free, n_free = torch.full((3, 4), 5, **i32), torch.arange(20, 32, **i32), torch.full((1,), 12, **i32)
    length, new = torch.tensor([0, 15, 16], **i64), torch.tensor([2, 3, 0], **i32)
    done = torch.tensor([0, 1, 0], **i32)
    c = ts._attention_case(3, "bf16", [40, 0, 100], 8, 4, 2, 64, 16, nan=False)
    qkv, ck, cv = c["qkv"].to(dev), c["ck"].to(dev), c["cv"].to(dev)
    pages, lens = torch.from_numpy(c["table"]).to(dev), torch.from_numpy(c["len"]).to(dev)
    x = torch.randn((2, 4, 1000), device=dev)
    presence = torch.ones(2, device=dev)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()

    def make():
        return (serving.PageMap(3, 3, 16, 4, 12), serving.PageMap(3, 3, 16, 4, 12),
                serving.TreeAttention(3, 8, 4, 2, 64, torch.bfloat16, 16, ck.shape[0], pages.shape[1]),
                serving.LogitsProcessor(2, 4, 1000, torch.float32, parent=[-1, 0, 0, 1]))

    y = torch.empty_like(x)

    def call(plan, back, attend, op, table, free):
        slots, granted, ln, nf = plan(length, new, table, free, n_free, stream=side)
        ln2, nf2 = back.release(ln, done, table, free, nf, stream=side)
        out, lse = attend(qkv[:, :, :4], qkv[:, :, 4:6], qkv[:, :, 6:], ck, cv, pages, lens, stream=side)
        op(x, presence=presence, out=y, stream=side)
        return slots, granted, ln, nf, ln2, nf2, out, lse

    other = table.clone(), free.clone()
    torch.cuda.synchronize()
    call(*make(), *other)  # memory is at hand and kernels are loaded then
    torch.cuda.synchronize()
    torch.cuda._sleep(int(4e8))  # some 0.2 s
    slots, granted, ln, nf, ln2, nf2, out, lse = call(*make(), table, free)
    side.synchronize()
    assert not torch.cuda.current_stream().query()  # still busy
    torch.cuda.synchronize()
    assert slots.tolist() == [[31 * 16, 31 * 16 + 1, -1], [5 * 16 + 15, 30 * 16, 30 * 16 + 1], [-1] * 3]
    assert granted.tolist() == [2, 3, 0] and ln.tolist() == [2, 18, 16] and int(nf) == 10
    assert ln2.tolist() == [2, 0, 16] and int(nf2) == 12
    ts._check_attention(c, (out.double().cpu().numpy(), lse.double().cpu().numpy()))
    assert torch.equal(y, x)


@pytest.mark.gpu
def test_a_view_of_a_returned_length_is_the_next_input():
    """What a call returned may come back as it is or as a view of it, and as a copy."""
    import torch
    from paper_2506_04708_b200 import serving
    i32, i64 = dict(dtype=torch.int32, device="cuda:0"), dict(dtype=torch.int64, device="cuda:0")
    plan = serving.PageMap(3, 2, 16, 4, 12)
    table, free, n_free = torch.full((3, 4), -1, **i32), torch.arange(12, **i32), torch.full((1,), 12, **i32)
    length, new = torch.zeros(3, **i64), torch.full((3,), 2, **i32)
    for i, again in enumerate((lambda t: t, lambda t: t[:], lambda t: t.view(-1), lambda t: t.detach(), lambda t: t.clone(), lambda t: t[:])):
        _, _, length, n_free = plan(again(length), new, table, free, again(n_free))
        assert length.tolist() == [2 * i + 2] * 3 and n_free.tolist() == [9]
    length, n_free = plan.release(length[:], torch.tensor([0, 1, 0], **i32), table, free, n_free[:])
    assert length.tolist() == [12, 0, 12] and n_free.tolist() == [10]


def test_results_of_a_page_map_take_turns():
    import torch
    from paper_2506_04708_b200 import serving
    p = object.__new__(serving.PageMap)
    p._len, p._n_free = [torch.zeros(3), torch.zeros(3)], [torch.zeros(1), torch.zeros(1)]
    for k in (0, 1):
        for same in (lambda t: t, lambda t: t[:], lambda t: t.view(-1)):
            length, n_free = p._outs(same(p._len[k]), same(p._n_free[1 - k]))
            assert length is p._len[1 - k] and n_free is p._n_free[k]
    length, n_free = p._outs(torch.zeros(3), torch.zeros(1))
    assert length is p._len[0] and n_free is p._n_free[0]


# ---------------------------------------------------------------- alignment
def test_arrays_off_their_elements_are_refused():
    """Each array in turn a byte, and half an element, off its element's boundary: refused before a launch."""
    import ctypes as C
    lib_build.build()
    L = binding.lib()

    def places(sizes):  # (name, bytes of an element) -> a call's pointers with one of them off
        for name, size in sizes.items():
            for off in {1, size // 2}:
                yield name, {n: C.c_void_p(0x100000 * (i + 1) + (off if n == name else 0)) for i, n in enumerate(sizes)}

    for dtype, es in ((binding.DTYPE_BF16, 2), (binding.DTYPE_F32, 4)):
        shape = ts._shape(dtype=dtype)
        sizes = dict(q=es, k=es, v=es, ck=es, cv=es, table=4, length=8, mask=4, tree=4, out=es, lse=4)
        for name, p in places(sizes):
            assert L.stand_tree_attention(C.byref(shape), p["q"], p["k"], p["v"], p["ck"], p["cv"], p["table"], p["length"], p["mask"], 0, p["tree"],
                                          C.c_void_p(0x2000000), 1 << 40, p["out"], p["lse"], None) == -1, name
        kv = binding.StandKvShape(1, 1, 4, 2, 64, dtype, 16, 3, 2, 0)
        for name, p in places(dict(k=es, v=es, path=4, slots=8, ck=es, cv=es)):
            assert L.stand_kv_commit(C.byref(kv), p["k"], p["v"], p["path"], p["slots"], p["ck"], p["cv"], None) == -1, name
        s = binding.StandLogits(2, 1, 100, dtype, None, 100, 100, 5, 1, 1, 0)
        names = [n for n, _ in binding.StandLogitsInputs._fields_]
        sizes = dict({n: 8 if n in ("n_text", "n_prompt") else 4 for n in names}, x_in=es, x_out=es)
        for name, p in places(sizes):
            x = binding.StandLogitsInputs(*[p[n] for n in names])
            assert L.stand_process_logits(C.byref(s), C.byref(x), p["x_in"], p["x_out"], None) == -1, name
    for name, p in places(dict(length=8, new=4, free=4, n_free=4, table=4, slots=8, granted=4, len_out=8, n_out=4)):
        assert L.stand_page_map(p["length"], p["new"], 2, 3, 16, 4, p["free"], 9, p["n_free"], p["table"], p["slots"], p["granted"], p["len_out"],
                                p["n_out"], None) == -1, name
    for name, p in places(dict(length=8, done=4, free=4, n_free=4, table=4, len_out=8, n_out=4)):
        assert L.stand_page_release(p["length"], p["done"], 2, 16, 4, p["table"], 9, p["free"], p["n_free"], p["len_out"], p["n_out"], None) == -1, name


# ---------------------------------------------------------------- launches in a row
@pytest.mark.gpu
def test_launches_of_all_head_sizes_in_a_row_and_on_two_streams():
    """Launches that follow one another closely, with different shares of an SM's tensor memory, some on another stream at the same
    time: the same bits as each by itself."""
    import torch
    from paper_2506_04708_b200 import serving
    dev, work = "cuda:0", []
    for i, (dim, N, hq, hkv) in enumerate(((64, 8, 4, 2), (128, 24, 8, 2), (256, 9, 4, 2), (64, 40, 4, 2), (200, 3, 2, 1), (128, 1, 8, 8))):
        c = ts._attention_case(i, "bf16", [700, 0, 129, 3000], N, hq, hkv, dim, 16, parent=inputs.topology(N, min(4, N - 1), 3), nan=False)
        qkv = c["qkv"].to(dev)
        args = (qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:], c["ck"].to(dev), c["cv"].to(dev), torch.from_numpy(c["table"]).to(dev),
                torch.from_numpy(c["len"]).to(dev))
        make = lambda: serving.TreeAttention(4, N, hq, hkv, dim, torch.bfloat16, 16, args[3].shape[0], args[5].shape[1], parent=c["parent"])  # noqa: E731
        plans = make(), make()
        alone = [t.clone() for t in plans[0](*args)]
        torch.cuda.synchronize()
        ts._check_attention(c, tuple(t.double().cpu().numpy() for t in alone))
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
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("N,hq,hkv,dim", [(1, 4, 1, 128), (5, 4, 2, 64), (9, 6, 2, 64), (64, 7, 1, 128), (3, 2, 1, 256), (50, 1, 1, 64), (7, 3, 1, 96)])
def test_results_do_not_depend_on_what_shared_memory_held(dtype, N, hq, hkv, dim):
    """Rows that do not fill their tiles, after launches whose queries and keys leave large scores, infinities and NaN behind."""
    import torch
    from paper_2506_04708_b200 import serving
    c = ts._attention_case(dim * N, dtype, [700, 40, 2000], N, hq, hkv, dim, 16, parent=inputs.topology(N, min(4, N - 1), 3), nan=False)
    c["qkv"][:, :, :hq] *= 3  # the maximum rises along the text
    dev = "cuda:0"
    qkv, ck, cv = c["qkv"].to(dev), c["ck"].to(dev), c["cv"].to(dev)
    table, length = torch.from_numpy(c["table"]).to(dev), torch.from_numpy(c["len"]).to(dev)
    plan = serving.TreeAttention(3, N, hq, hkv, dim, ts._dtype(dtype), 16, ck.shape[0], table.shape[1], parent=c["parent"])
    # as many rows as a tile has, the same pages and lengths: all CTAs leave theirs behind
    full = 128 // (hq // hkv)
    spoil = serving.TreeAttention(3, full, hq, hkv, dim, ts._dtype(dtype), 16, ck.shape[0], table.shape[1])
    first = None
    for fill in (0.0, 1.0, -30.0, 1000.0, INF, NAN):
        q = torch.full((3, full, hq, dim), fill, dtype=ts._dtype(dtype), device=dev)
        kv = torch.full((3, full, hkv, dim), fill, dtype=ts._dtype(dtype), device=dev)
        spoil(q, kv, kv, ck, cv, table, length)
        out, lse = plan(qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:], ck, cv, table, length)
        if first is None:
            first = out.clone(), lse.clone()
        assert torch.equal(out, first[0]) and torch.equal(lse, first[1]), fill
    ts._check_attention(c, tuple(t.double().cpu().numpy() for t in first))


# ---------------------------------------------------------------- the example
@pytest.mark.gpu
def test_the_loop_tells_when_a_sequence_outgrows_its_pages():
    from examples import tree_decode as td
    model = td.Model(V=300)
    prompts = [np.arange(6, dtype=np.int32), np.arange(30, dtype=np.int32)]
    dec = td.Decoder(model, prompts, most=48)  # three pages of 16 each
    for _ in range(60):
        before = int(dec.n_text[1])
        dec.step()
        if int(dec.n_text[1]) - 1 > 48:  # does not fit any more
            break
        assert not dec.short.any()
    assert before <= 49 and dec.short.tolist()[1]
    assert int(dec.len[1]) == before - 1


# ---------------------------------------------------------------- page release by itself
@pytest.mark.gpu
@pytest.mark.parametrize("B", [1, 3, 300])
@pytest.mark.parametrize("room", ["plenty", "short", "none"])
def test_release_pushes_whole_pages_in_order(B, room):
    """Lengths of zero and below, at and past a page's end, beyond the table (its columns count); a list that takes all, some or none."""
    import torch
    from paper_2506_04708_b200 import serving
    rng = np.random.default_rng(B)
    page, cols = 16, 5
    length = rng.choice([-4, 0, 1, 15, 16, 17, 33, 79, 80, 81, 10**12], B).astype(np.int64)
    done = (rng.random(B) < 0.6).astype(np.int32) * rng.integers(-3, 4, B).astype(np.int32)
    table = rng.permutation(B * cols).reshape(B, cols).astype(np.int32)
    pages = [list(table[b, : min(-(-max(int(length[b]), 0) // page), cols)]) if done[b] else [] for b in range(B)]
    given, held = sum(pages, []), 7
    capacity = held + {"plenty": len(given) + 3, "short": len(given) // 2, "none": 0}[room]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")  # noqa: E731
    free = np.full(capacity, -9, np.int32)
    free[:held] = 1000 + np.arange(held)
    t_free = dev(free)
    plan = serving.PageMap(B, 1, page, cols, capacity)
    ln, nf = plan.release(dev(length), dev(done), dev(table), t_free, dev(np.array([held], np.int32)))
    n = min(held + len(given), capacity)
    free[held:n] = given[: n - held]
    assert int(nf) == n and np.array_equal(t_free.cpu().numpy(), free)
    assert np.array_equal(ln.cpu().numpy(), np.where(done != 0, 0, length))


# ---------------------------------------------------------------- large values
@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,hq,hkv,dim", [(1, 2, 2, 64), (8, 8, 2, 128), (40, 4, 2, 64), (3, 2, 1, 256)])
def test_values_near_the_end_of_the_range(dtype, N, hq, hkv, dim):
    """Values of up to 2^117 under scores that rise by 5 nats after the first tile: 700 of them fit the range with room, and so does any
    weighted mean of them."""
    c = ts._attention_case(dim, dtype, [700] * 150, N, hq, hkv, dim, 16, parent=inputs.topology(N, min(N - 1, 3), 4), nan=False, spare=0)
    c["qkv"][:, :, :hq] = 0
    c["qkv"][:, :, :hq, 0] = 1.0
    c["ck"][:, :, :, 0] = 5.0
    for b in range(150):
        for page in c["table"][b, :4]:
            c["ck"][int(page), :, :, 0] = 0.0
    big = 2.0**117
    c["cv"] = (c["cv"].float().clamp(-1, 1) * 0.25 + 0.5).mul(big).to(c["cv"].dtype)
    c["qkv"][:, :, hq + hkv:] = 0
    few = dict(c, len=c["len"][:2], table=c["table"][:2], qkv=c["qkv"][:2])
    want = ts._reference(few, scale=1.0)
    out, lse = ts._run_attention(c, scale=1.0)
    assert np.isfinite(out).all()
    ts._check_attention(few, (out[:2] / big, lse[:2]), want=(want[0] / big, want[1], want[2] / big, want[3] / big, want[4]))


# ---------------------------------------------------------------- logits: rows over rows
def test_logits_rows_laid_over_others_are_refused():
    import ctypes as C
    lib_build.build()
    x = binding.StandLogitsInputs()
    parent = np.array([-1, 0, 0], np.int32)

    def call(out, in_stride=100, out_stride=100, at=0x1000000, dtype=binding.DTYPE_F32):
        s = binding.StandLogits(2, 3, 100, dtype, parent.ctypes.data, in_stride, out_stride, 0, 0, 0, 0)
        return binding.lib().stand_process_logits(C.byref(s), C.byref(x), C.c_void_p(at), C.c_void_p(out), None)

    at = 0x1000000
    for bad in (dict(out=at + 4), dict(out=at - 4), dict(out=at + 400), dict(out=at - 400 * 5), dict(out=at + 400 * 5 + 396),
                dict(out=at + 396, in_stride=300, out_stride=300), dict(out=at + 804, in_stride=300, out_stride=300),
                dict(out=at + 400, in_stride=200, out_stride=300), dict(out=at + 2, dtype=binding.DTYPE_BF16)):
        assert call(**bad) == -1, bad


@pytest.mark.gpu
@pytest.mark.parametrize("where", ["between", "behind", "before"])
def test_logits_rows_between_others_are_taken(where):
    """Output rows in the gaps between the input's, and right behind or before all of them, in one buffer."""
    import torch
    from paper_2506_04708_b200 import serving
    B, N, V = 3, 4, 1001
    op = serving.LogitsProcessor(B, N, V, torch.float32, parent=[-1, 0, 0, 1])
    pen = torch.ones(B, device="cuda:0")
    text, n = torch.arange(7, dtype=torch.int32, device="cuda:0").expand(B, 7).contiguous(), torch.full((B,), 7, dtype=torch.int64, device="cuda:0")
    if where == "between":
        both = torch.randn((B, N, 2 * V), device="cuda:0")
        x, y = both[..., :V], both[..., V:]
    else:
        both = torch.randn((2, B, N, V), device="cuda:0")
        x, y = (both[0], both[1]) if where == "behind" else (both[1], both[0])
    want = x.clone()
    want[..., :7] -= 1
    assert op(x, text, n, presence=pen, out=y) is y and torch.equal(y, want)
    flat = torch.randn(B * N * V + 5, device="cuda:0")
    with pytest.raises(binding.StandError):
        op(flat[:-5].view(B, N, V), out=flat[5:].view(B, N, V))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("hq,hkv,dim", [(4, 2, 64), (8, 2, 128), (4, 4, 64), (2, 1, 256)])
def test_queries_of_undrafted_nodes_do_not_touch_other_rows(dtype, hq, hkv, dim):
    """Bit for bit, whatever the projection left in the rows of nodes that were not drafted."""
    N = 24
    c = ts._attention_case(dim, dtype, [300, 40, 1000], N, hq, hkv, dim, 16, parent=inputs.topology(N, 6, 3), undrafted=0.4, nan=False)
    dead = np.argwhere(c["tree"] < 0)
    assert len(dead) > 3
    c["qkv"][:, :, :hq] *= 3
    first = None
    for fill in (0.0, 5.0, -40.0, 3000.0, INF, NAN):
        for b, u in dead:
            c["qkv"][int(b), int(u), :hq] = fill
        got = ts._run_attention(c)
        first = first or got
        assert np.array_equal(got[0], first[0]) and np.array_equal(got[1], first[1]), fill
    ts._check_attention(c, first)


# ---------------------------------------------------------------- a sequence full of such values beside others
@pytest.mark.gpu
@pytest.mark.parametrize("how", ["prompt, one NaN", "prompt, all infinite", "cached infinities, heads of 64", "cached NaN, heads of 64"])
def test_one_sequence_that_is_not_finite_does_not_hold_up_others(how):
    """What is done for values that are not finite stays within waits of a few milliseconds (a sixty-fourth of what they
    may last), so that no warp gives up and no other sequence is touched."""
    import torch
    from paper_2506_04708_b200 import serving
    dev, dt = "cuda:0", torch.bfloat16
    g = torch.Generator(device=dev).manual_seed(4)
    prompt = how.startswith("prompt")
    B, N, hq, hkv, dim, L, page = (3, 4096, 8, 2, 128, 0, 16) if prompt else (6, 32, 16, 16, 64, 8192, 64)
    pool, cols = B * L // page, L // page
    ck, cv = (torch.randn((pool, hkv, page, dim), generator=g, device=dev, dtype=dt) for _ in range(2))
    table = torch.arange(pool, dtype=torch.int32, device=dev).view(B, cols)
    length = torch.full((B,), L, dtype=torch.int64, device=dev)
    qkv = torch.randn((B, N, hq + 2 * hkv, dim), generator=g, device=dev, dtype=dt)
    plan = serving.TreeAttention(B, N, hq, hkv, dim, dt, page, pool, cols, parent=None if prompt else inputs.topology(N, 4, 4))
    args = qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], qkv[:, :, hq + hkv:], ck, cv, table, length
    clean = plan(*args)[0].clone()
    touched = torch.zeros_like(clean, dtype=torch.bool)
    if how == "prompt, one NaN":
        qkv[1, 5, hq + hkv + 1, 9] = NAN
        touched[1, 5:, hq // hkv:, 9] = True
        value = NAN
    elif how == "prompt, all infinite":
        qkv[1, :, hq + hkv:] = -INF
        touched[1] = True
        value = -INF
    else:
        value = INF if "infinities" in how else NAN
        for tile in range(cols):  # one token of every page
            cv[int(table[1, tile]), :, tile % page] = value
        touched[1] = True
    torch.cuda.synchronize()
    binding.set_wait_limit(2**16)
    try:
        out = plan(*args)[0]
        torch.cuda.synchronize()
    finally:
        binding.set_wait_limit(-1)
    assert torch.equal(out[~touched], clean[~touched])
    assert (torch.isnan(out[touched]) if np.isnan(value) else out[touched] == value).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ts.ALL_TYPES)
@pytest.mark.parametrize("N,hq,hkv,dim", [(150, 2, 1, 64), (20, 2, 2, 64), (700, 2, 1, 128), (90, 1, 1, 200)])
def test_values_of_a_prompt_that_are_not_finite(dtype, N, hq, hkv, dim):
    """Several in a column: of one sign, of both (NaN from the second on), NaN first; over a cached text that has some too."""
    c = ts._attention_case(N, dtype, [0, 40], N, hq, hkv, dim, 16)
    clean, v0 = ts._reference(c), hq + hkv
    expect = {}

    def put(b, node, d, value):
        c["qkv"][b, node, v0, d] = value
        with np.errstate(invalid="ignore"):
            expect.setdefault((b, d), np.zeros(N))[node:] += value

    for b in (0, 1):
        put(b, 3, 0, INF)
        put(b, 9, 0, INF)
        put(b, N - 1, 0, -INF)
        put(b, 5, 1, -INF)
        put(b, 6, 1, NAN)
        put(b, 2, 2, NAN)
        put(b, 4, 2, INF)
        put(b, 0, 5, -INF)
    for node in range(7, N):
        put(1, node, dim - 1, INF)
    _plant(c, 1, 20, 0, 0, INF)
    expect[1, 0] += INF
    _plant(c, 1, 21, 0, 5, INF)
    expect[1, 5] = np.full(N, NAN)
    _plant(c, 1, 22, 0, 6, -INF)
    expect[1, 6] = np.full(N, -INF)
    out, lse = ts._run_attention(c)
    hit = np.zeros_like(out, bool)
    group = hq // hkv
    for (b, d), want in expect.items():
        odd = ~np.isfinite(want) | (want != 0)
        got = out[b, :, :group, d]
        assert np.array_equal(got[odd], np.repeat(want[odd, None], group, 1), equal_nan=True), (b, d)
        hit[b, odd, :group, d] = True
    ts._check_attention(c, (np.where(hit, clean[0], out), lse), want=clean)
