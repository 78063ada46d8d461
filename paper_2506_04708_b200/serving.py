"""Thin binding of the operators around the decoding step (include/stand.h, second half).

`TreeAttention`, `PageMap`, `KvCommit` and `LogitsProcessor`, and for positions and a cache in 4 bits `HeadRotation`, `KvAppend`,
`KvRead` and `PackedTreeAttention`, hold what stays the same from step to step - shapes, the
tree, workspaces, result tensors - and are called with the step's device tensors.  Argument marshalling only: the work
runs in the CUDA kernels of libstand.so.  Calls only enqueue work on the current stream (or `stream`) and return; the
result tensors of an object are overwritten by its next call unless the caller passes its own.  An object, and tensors given
to it, must live until the work on the stream is done; calls of one object that may overlap need an order of their own.
"""
import ctypes as C
import math

import numpy as np

from .binding import (DTYPE_BF16, DTYPE_F16, DTYPE_F32, StandAttention, StandError, StandKvRows, StandKvShape, StandLogits,
                      StandLogitsInputs, StandRotation, _check, lib)


def _dtype_code(dtype):
    import torch
    code = {torch.float32: DTYPE_F32, torch.bfloat16: DTYPE_BF16, torch.float16: DTYPE_F16}.get(dtype)
    if code is None:
        raise StandError(f"unsupported dtype {dtype}")
    return code


def _need(cond, what):
    if not cond:
        raise StandError(what)


def _steps(x, what):
    """The strides of all dimensions but the last, whose elements lie side by side.  A dimension of one element has none, an empty
    tensor neither."""
    shape, strides = x.shape, x.stride()
    if 0 in shape:
        return [0] * (len(shape) - 1)
    _need(shape[-1] == 1 or strides[-1] == 1, f"{what}: a contiguous last dimension")
    return [s if n > 1 else 0 for n, s in zip(shape[:-1], strides)]


def _apart(x, what):
    """Refuses tensors to write whose rows share memory by a stride of 0 (expanded ones)."""
    _need(not any(s == 0 and n > 1 for s, n in zip(x.stride(), x.shape)), f"{what}: wants rows of its own for every place")


class _Op:
    """Device, stream and workspace handling of the operators."""

    def _init_device(self, device):
        import torch
        self.torch = torch
        self.dev = torch.device(device)
        if self.dev.index is None:
            self.dev = torch.device(self.dev.type, torch.cuda.current_device())
        self._index = self.dev.index
        self._raw_stream, self._current_device = torch._C._cuda_getCurrentRawStream, torch.cuda.current_device
        self._lib = lib()

    def _launch(self, stream, call, *args):
        """One library call on `stream` (or the device's current one), with the operator's device current."""
        st = self._raw_stream(self._index) if stream is None else stream.cuda_stream
        if self._current_device() == self._index:
            rc = call(*args, st)
        else:
            with self.torch.cuda.device(self.dev):
                rc = call(*args, st)
        if rc:
            _check(rc, call.__name__)

    def _ints(self, t, dtype, shape, what):
        if t.dtype is not dtype or t.shape != shape or t.get_device() != self._index or not t.is_contiguous():
            raise StandError(f"{what}: wants a contiguous {dtype} tensor {tuple(shape)} on {self.dev}, "
                             f"got {t.dtype} {tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    def _opt(self, t, dtype, shape, what):
        return None if t is None else self._ints(t, dtype, shape, what)

    def _floats(self, x, shape, what):
        if x.dtype is not self.dtype or x.shape != shape or x.get_device() != self._index:
            raise StandError(f"{what}: wants a {self.dtype} tensor {shape} on {self.dev}, "
                             f"got {x.dtype} {tuple(x.shape)} on {x.device}")
        return x.data_ptr()


def tree_mask(parent):
    """Ancestor bits of a static tree, uint32 [n, ceil(n/32)] (numpy): bit v of row u is set if v is u or above it."""
    par = np.ascontiguousarray(parent, np.int32)
    out = np.zeros((len(par), (len(par) + 31) // 32), np.uint32)
    _check(lib().stand_tree_mask(par.ctypes.data, len(par), out.ctypes.data), "stand_tree_mask")
    return out


class TreeAttention(_Op):
    """Attention of draft trees over a paged cache (stand_tree_attention).

    parent: the static tree (its ancestor mask is used for all sequences); or mask: int32 device tensor
    [N, ceil(N/32)] or [B, N, ceil(N/32)] of visibility bits; neither: node u sees nodes 0..u (a chain, a prompt).
    max_pages: columns of the block table.  scale: default 1 / sqrt(dim)."""

    def __init__(self, B, N, heads_q, heads_kv, dim, dtype, page_size, pages, max_pages, scale=None, parent=None, mask=None,
                 device="cuda:0"):
        self._init_device(device)
        t = self.torch
        self.cfg = StandAttention(B, N, heads_q, heads_kv, dim, _dtype_code(dtype), page_size, pages, max_pages,
                                  1.0 / math.sqrt(dim) if scale is None else float(scale))
        self.dtype = dtype
        need = self._lib.stand_tree_attention_scratch_bytes(C.byref(self.cfg))
        _need(need > 0, "TreeAttention: invalid shapes")
        _need(parent is None or mask is None, "TreeAttention: parent or mask, not both")
        words = (N + 31) // 32
        self.mask, self.mask_stride = None, 0
        if parent is not None:
            _need(len(parent) == N, "TreeAttention: parent has N entries")
            self.mask = t.from_numpy(tree_mask(parent).view(np.int32)).to(self.dev)
        elif mask is not None:
            _need(mask.dtype == t.int32 and mask.device == self.dev and mask.is_contiguous()
                  and tuple(mask.shape) in ((N, words), (B, N, words)), "TreeAttention: mask")
            self.mask, self.mask_stride = mask, N * words if mask.dim() == 3 else 0
        self._mask_ptr = None if self.mask is None else self.mask.data_ptr()
        self._q_shape, self._kv_shape = (B, N, heads_q, dim), (B, N, heads_kv, dim)
        self._cache_shape = self._block(pages, heads_kv, page_size, dim)
        self._table_shape, self._len_shape, self._tree_shape = (B, max_pages), (B,), (B, N)
        self.scratch = t.empty(need + 256, dtype=t.uint8, device=self.dev)
        self._scratch = self.scratch.data_ptr() + (-self.scratch.data_ptr()) % 256
        self._scratch_bytes = need
        self.out = t.empty(self._q_shape, dtype=dtype, device=self.dev)
        self.lse = t.empty((B, N, heads_q), dtype=t.float32, device=self.dev)
        self._cfg_ptr, self._strides = C.addressof(self.cfg), None

    _entry = "stand_tree_attention"

    @staticmethod
    def _block(pages, heads, page_size, dim):
        return (pages, heads, page_size, dim)

    def _cached(self, x, what):
        return self._floats(x, self._cache_shape, what)

    def __call__(self, q, k, v, cache_k, cache_v, table, length, tree_tokens=None, out=None, lse=None, stream=None):
        """q [B, N, heads_q, dim], k / v [B, N, heads_kv, dim] (any strides: slices of one projection will do, keys rotated
        into a tensor of their own too), caches [pages, heads_kv, page_size, dim] (any strides, the same for both), table [B, max_pages] int32, length [B] int64, tree_tokens
        [B, N] int32 or None (nodes below 0 get empty rows).  Returns (out [B, N, heads_q, dim], lse [B, N, heads_q])."""
        t, c = self.torch, self.cfg
        pq, pk, pv = self._floats(q, self._q_shape, "q"), self._floats(k, self._kv_shape, "k"), self._floats(v, self._kv_shape, "v")
        pck, pcv = self._cached(cache_k, "cache_k"), self._cached(cache_v, "cache_v")
        strides = q.stride(), k.stride(), v.stride(), cache_k.stride(), cache_v.stride()
        if strides != self._strides:
            qs, ks, vs, cs = _steps(q, "q"), _steps(k, "k"), _steps(v, "v"), _steps(cache_k, "cache_k")
            _need(_steps(cache_v, "cache_v") == cs, "TreeAttention: both caches have the same strides")
            c.q_stride[:], c.kv_stride[:], c.v_stride[:], c.cache_stride[:] = qs, ks, vs, cs + [0] * (3 - len(cs))
            c.own_v_stride, self._strides = 1, strides
        ptab = self._ints(table, t.int32, self._table_shape, "table")
        plen = self._ints(length, t.int64, self._len_shape, "length")
        ptree = self._opt(tree_tokens, t.int32, self._tree_shape, "tree_tokens")
        if out is None:
            out = self.out
        else:
            self._floats(out, self._q_shape, "out")
            _need(out.is_contiguous(), "out: wants a contiguous tensor")
        if lse is None:
            lse = self.lse
        plse = self._ints(lse, t.float32, self.lse.shape, "lse")
        self._launch(stream, getattr(self._lib, self._entry), self._cfg_ptr, pq, pk, pv, pck, pcv, ptab, plen, self._mask_ptr,
                     self.mask_stride, ptree, self._scratch, self._scratch_bytes, out.data_ptr(), plse)
        return out, lse


def packed_block_bytes(page_size, dim):
    """Bytes of a page of one head in the 4-bit form: codes of all its tokens, then their scales (include/stand.h)."""
    return page_size * dim // 16 * 9


def _packed_shapes(page_size, dim, what):
    _need(dim >= 16 and dim % 16 == 0 and page_size >= 16 and page_size % 16 == 0, f"{what}: the 4-bit form wants dim and page_size to be multiples of 16")


class PackedTreeAttention(TreeAttention):
    """TreeAttention over caches in the 4-bit form (stand_packed_tree_attention): cache_k / cache_v are uint8
    [pages, heads_kv, packed_block_bytes(page_size, dim)], page and head at multiples of 16 bytes.  All else is the same."""

    _entry = "stand_packed_tree_attention"

    def __init__(self, B, N, heads_q, heads_kv, dim, dtype, page_size, *args, **kw):
        _packed_shapes(page_size, dim, "PackedTreeAttention")
        super().__init__(B, N, heads_q, heads_kv, dim, dtype, page_size, *args, **kw)

    @staticmethod
    def _block(pages, heads, page_size, dim):
        return (pages, heads, packed_block_bytes(page_size, dim))

    def _cached(self, x, what):
        return _packed_cache(self, x, self._cache_shape, what)


def _packed_cache(op, x, shape, what):
    if x.dtype is not op.torch.uint8 or x.shape != shape or x.get_device() != op._index:
        raise StandError(f"{what}: wants a uint8 tensor {shape} on {op.dev}, got {x.dtype} {tuple(x.shape)} on {x.device}")
    return x.data_ptr()


class HeadRotation(_Op):
    """Norms of queries and keys per head and the position rotation, in one pass (stand_rotate_heads).

    freq: float32 [rotary_dim / 2], the angle per position of each pair (None: no rotation); interleaved: pairs are neighbours
    (else half of rotary_dim apart); offset: int32 [N] or [B, N], what a node's position adds to its sequence's (None: its
    number); norm with weight_q, weight_k [dim] (None: ones)."""

    def __init__(self, B, N, heads_q, heads_kv, dim, dtype, freq=None, offset=None, interleaved=False, norm=False, weight_q=None,
                 weight_k=None, eps=1e-6, device="cuda:0"):
        self._init_device(device)
        t = self.torch
        self.dtype = dtype
        _need(B >= 1 and N >= 1 and heads_q >= 1 and heads_kv >= 1 and 1 <= dim <= 256, "HeadRotation: invalid shapes")
        self._turn = _Turn(self, B, N, dim, freq, offset, norm, (weight_q, weight_k), (dim,), eps, "HeadRotation")
        self.cfg = StandRotation(B, N, heads_q, heads_kv, dim, _dtype_code(dtype), self._turn.rotary, int(bool(interleaved)), int(bool(norm)),
                                 float(eps) if norm else 0.0)
        self.cfg.offset_stride = self._turn.offset_stride
        self._q, self._k, self._b = (B, N, heads_q, dim), (B, N, heads_kv, dim), (B,)
        self.q_out = t.empty(self._q, dtype=dtype, device=self.dev)
        self.k_out = t.empty(self._k, dtype=dtype, device=self.dev)
        self._cfg_ptr, self._strides = C.addressof(self.cfg), None

    def __call__(self, q, k, base=None, q_out=None, k_out=None, stream=None):
        """q [B, N, heads_q, dim], k [B, N, heads_kv, dim] (any strides), base [B] int64: the position that each sequence's nodes
        begin at (None: 0).  q_out / k_out: tensors to write (q and k themselves: in place); None: tensors kept by this object.
        Returns (q_out, k_out)."""
        c = self.cfg
        q_out, k_out = self.q_out if q_out is None else q_out, self.k_out if k_out is None else k_out
        pq, pk = self._floats(q, self._q, "q"), self._floats(k, self._k, "k")
        pqo, pko = self._floats(q_out, self._q, "q_out"), self._floats(k_out, self._k, "k_out")
        strides = q.stride(), k.stride(), q_out.stride(), k_out.stride()
        if strides != self._strides:
            _apart(q_out, "q_out"), _apart(k_out, "k_out")
            qs, ks, qo, ko = _steps(q, "q"), _steps(k, "k"), _steps(q_out, "q_out"), _steps(k_out, "k_out")
            c.q_stride[:], c.k_stride[:], c.q_out_stride[:], c.k_out_stride[:] = qs, ks, qo, ko
            self._strides = strides
        r = self._turn
        pb = self._opt(base, self.torch.int64, self._b, "base")
        self._launch(stream, self._lib.stand_rotate_heads, self._cfg_ptr, pq, pk, r.weights[0], r.weights[1], r.freq, pb, r.offset, pqo, pko)
        return q_out, k_out


class _Turn:
    """What rotations are made with: device pointers of freq, offset and weights, whose tensors are kept."""

    def __init__(self, op, B, N, dim, freq, offset, norm, weights, weight_shape, eps, what):
        t = op.torch
        self.rotary = 0
        self.freq = self.offset = None
        self.offset_stride = 0
        self.kept = freq, offset, weights
        if freq is not None:
            _need(freq.dim() == 1 and 1 <= freq.shape[0] <= dim // 2, f"{what}: freq has 1 .. dim / 2 entries")
            self.freq, self.rotary = op._ints(freq, t.float32, freq.shape, "freq"), 2 * freq.shape[0]
        if offset is not None:
            _need(freq is not None, f"{what}: offset goes with freq")
            self.offset = op._ints(offset, t.int32, (N,) if offset.dim() == 1 else (B, N), "offset")
            self.offset_stride = 0 if offset.dim() == 1 else N
        _need(not norm or (eps > 0.0 and math.isfinite(eps)), f"{what}: eps > 0")
        _need(norm or all(w is None for w in weights), f"{what}: weights go with norm")
        self.weights = [op._opt(w, op.dtype, weight_shape, "weight") for w in weights]


class KvAppend(_Op):
    """Keys and values of chosen nodes into the cache, all layers at once, with the keys' norm and position rotation and the
    4-bit form on the way (stand_kv_append).

    packed: the caches are uint8 [layers, pages, heads, packed_block_bytes(page_size, dim)], else [layers, pages, heads, page_size, dim]
    of `dtype`.  freq, offset, interleaved, norm, eps as in HeadRotation; weight_k [layers, dim]."""

    def __init__(self, layers, B, N, heads, dim, dtype, page_size, pages, width, packed=False, freq=None, offset=None, interleaved=False,
                 norm=False, weight_k=None, eps=1e-6, device="cuda:0"):
        self._init_device(device)
        self.dtype, self.packed = dtype, bool(packed)
        _need(1 <= layers <= 4096 and B >= 1 and N >= 1 and 1 <= heads <= 4096 and 1 <= dim <= 256 and width >= 1 and 1 <= page_size <= 4096
              and pages >= 0, "KvAppend: invalid shapes")
        if packed:
            _packed_shapes(page_size, dim, "KvAppend")
        self._turn = _Turn(self, B, N, dim, freq, offset, norm, (weight_k,), (layers, dim), eps, "KvAppend")
        self.cfg = StandKvRows(layers, B, N, heads, dim, _dtype_code(dtype), page_size, pages, width, int(self.packed), self._turn.rotary,
                               int(bool(interleaved)), int(bool(norm)), float(eps) if norm else 0.0)
        self.cfg.offset_stride = self._turn.offset_stride
        self._src, self._places, self._b = (layers, B, N, heads, dim), (B, width), (B,)
        self._cache = (layers, pages, heads, packed_block_bytes(page_size, dim)) if packed else (layers, pages, heads, page_size, dim)
        self._cfg_ptr, self._strides = C.addressof(self.cfg), None

    def __call__(self, k, v, slots, cache_k, cache_v, base=None, path=None, stream=None):
        """k / v [layers, B, N, heads, dim] (any strides), slots [B, width] int64 (PageMap), base [B] int64: the position that
        each sequence's nodes begin at (None: 0), path [B, width] int32 (None: node j goes to slot j), caches of any strides, the
        same for both."""
        t, c, r = self.torch, self.cfg, self._turn
        pk, pv = self._floats(k, self._src, "k"), self._floats(v, self._src, "v")
        if self.packed:
            pck, pcv = _packed_cache(self, cache_k, self._cache, "cache_k"), _packed_cache(self, cache_v, self._cache, "cache_v")
        else:
            pck, pcv = self._floats(cache_k, self._cache, "cache_k"), self._floats(cache_v, self._cache, "cache_v")
        strides = k.stride(), v.stride(), cache_k.stride(), cache_v.stride()
        if strides != self._strides:
            _apart(cache_k, "cache_k"), _apart(cache_v, "cache_v")
            ks, vs, cs = _steps(k, "k"), _steps(v, "v"), _steps(cache_k, "cache_k")
            _need(_steps(cache_v, "cache_v") == cs, "KvAppend: both caches have the same strides")
            c.k_stride[:], c.v_stride[:], c.cache_stride[:] = ks, vs, cs + [0] * (4 - len(cs))
            self._strides = strides
        ps, pp = self._ints(slots, t.int64, self._places, "slots"), self._opt(path, t.int32, self._places, "path")
        pb = self._opt(base, t.int64, self._b, "base")
        self._launch(stream, self._lib.stand_kv_append, self._cfg_ptr, pk, pv, r.weights[0], r.freq, pb, r.offset, pp, ps, pck, pcv)


class KvRead(_Op):
    """Rows of the cache back as values (stand_kv_read), from the 4-bit form (packed) in any `dtype`, else in the cache's own."""

    def __init__(self, layers, B, heads, dim, dtype, page_size, pages, width, packed=False, device="cuda:0"):
        self._init_device(device)
        t = self.torch
        self.dtype, self.packed = dtype, bool(packed)
        _need(1 <= layers <= 4096 and B >= 1 and 1 <= heads <= 4096 and 1 <= dim <= 256 and width >= 1 and 1 <= page_size <= 4096 and pages >= 0,
              "KvRead: invalid shapes")
        if packed:
            _packed_shapes(page_size, dim, "KvRead")
        self.cfg = StandKvRows(layers, B, 0, heads, dim, _dtype_code(dtype), page_size, pages, width, int(self.packed))
        self._places, self._out = (B, width), (layers, B, width, heads, dim)
        self._cache = (layers, pages, heads, packed_block_bytes(page_size, dim)) if packed else (layers, pages, heads, page_size, dim)
        self.k, self.v = (t.empty(self._out, dtype=dtype, device=self.dev) for _ in range(2))
        self._cfg_ptr, self._strides = C.addressof(self.cfg), None

    def __call__(self, slots, cache_k, cache_v, k=None, v=None, stream=None):
        """slots [B, width] int64 (a place without one: zeros), caches as KvAppend takes them.  k / v: contiguous tensors
        [layers, B, width, heads, dim] to write; None: tensors kept by this object.  Returns (k, v)."""
        c = self.cfg
        k, v = self.k if k is None else k, self.v if v is None else v
        pk, pv = self._floats(k, self._out, "k"), self._floats(v, self._out, "v")
        _need(k.is_contiguous() and v.is_contiguous(), "KvRead: contiguous results")
        if self.packed:
            pck, pcv = _packed_cache(self, cache_k, self._cache, "cache_k"), _packed_cache(self, cache_v, self._cache, "cache_v")
        else:
            pck, pcv = self._floats(cache_k, self._cache, "cache_k"), self._floats(cache_v, self._cache, "cache_v")
        strides = cache_k.stride(), cache_v.stride()
        if strides != self._strides:
            cs = _steps(cache_k, "cache_k")
            _need(_steps(cache_v, "cache_v") == cs, "KvRead: both caches have the same strides")
            c.cache_stride[:], self._strides = cs + [0] * (4 - len(cs)), strides
        ps = self._ints(slots, self.torch.int64, self._places, "slots")
        self._launch(stream, self._lib.stand_kv_read, self._cfg_ptr, pck, pcv, ps, pk, pv)
        return k, v


class PageMap(_Op):
    """Pages and slots for new tokens, and pages of finished sequences back (stand_page_map, stand_page_release).

    width: most new tokens of a sequence per call; max_pages: columns of the block table; capacity: size of the free
    list."""

    def __init__(self, B, width, page_size, max_pages, capacity, device="cuda:0"):
        self._init_device(device)
        t = self.torch
        _need(B >= 1 and width >= 1 and page_size >= 1 and max_pages >= 0 and capacity >= 0, "PageMap: invalid shapes")
        self.B, self.width, self.page_size, self.max_pages, self.capacity = B, width, page_size, max_pages, capacity
        self._b, self._table, self._list, self._one = (B,), (B, max_pages), (capacity,), (1,)
        # every call writes all of these; nothing is queued for them here, which could run after a call on another stream
        self.slots = t.empty((B, width), dtype=t.int64, device=self.dev)
        self.granted = t.empty(B, dtype=t.int32, device=self.dev)
        # two sets: what a call returned may be the next call's input
        self._len = [t.empty(B, dtype=t.int64, device=self.dev) for _ in range(2)]
        self._n_free = [t.empty(1, dtype=t.int32, device=self.dev) for _ in range(2)]

    def _outs(self, length, n_free):
        return [own[own[0].data_ptr() == given.data_ptr()] for own, given in ((self._len, length), (self._n_free, n_free))]

    def __call__(self, length, new, table, free, n_free, stream=None):
        """length [B] int64, new [B] int32, table [B, max_pages] int32 (gets the new pages), free [capacity] int32,
        n_free [1] int32.  Returns (slots [B, width] int64, granted [B] int32, length, n_free); the last two replace
        the arguments of the same names in the next call."""
        t = self.torch
        len_out, n_out = self._outs(length, n_free)
        args = (self._ints(length, t.int64, self._b, "length"), self._ints(new, t.int32, self._b, "new"), self.B, self.width,
                self.page_size, self.max_pages, self._ints(free, t.int32, self._list, "free"), self.capacity,
                self._ints(n_free, t.int32, self._one, "n_free"), self._ints(table, t.int32, self._table, "table"),
                self.slots.data_ptr(), self.granted.data_ptr(), len_out.data_ptr(), n_out.data_ptr())
        self._launch(stream, self._lib.stand_page_map, *args)
        return self.slots, self.granted, len_out, n_out

    def release(self, length, done, table, free, n_free, stream=None):
        """Pushes the pages of the sequences with done [B] int32 != 0 on the free list.  Returns (length, n_free)."""
        t = self.torch
        len_out, n_out = self._outs(length, n_free)
        args = (self._ints(length, t.int64, self._b, "length"), self._ints(done, t.int32, self._b, "done"), self.B,
                self.page_size, self.max_pages, self._ints(table, t.int32, self._table, "table"), self.capacity,
                self._ints(free, t.int32, self._list, "free"), self._ints(n_free, t.int32, self._one, "n_free"),
                len_out.data_ptr(), n_out.data_ptr())
        self._launch(stream, self._lib.stand_page_release, *args)
        return len_out, n_out


class KvCommit(_Op):
    """Keys and values of chosen nodes into the cache, all layers at once (stand_kv_commit)."""

    def __init__(self, layers, B, N, heads, dim, dtype, page_size, pages, width, device="cuda:0"):
        self._init_device(device)
        self.cfg = StandKvShape(layers, B, N, heads, dim, _dtype_code(dtype), page_size, pages, width, 0)
        self.dtype = dtype
        self._src, self._cache = (layers, B, N, heads, dim), (layers, pages, heads, page_size, dim)
        self._places = (B, width)
        self._cfg_ptr, self._strides = C.addressof(self.cfg), None

    def __call__(self, k, v, slots, cache_k, cache_v, path=None, stream=None):
        """k / v [layers, B, N, heads, dim] (any strides), slots [B, width] int64 (stand_page_map), path [B, width] int32
        (stand_last_path; None: node j goes to slot j), caches [layers, pages, heads, page_size, dim] (any
        strides, the same for both)."""
        t, c = self.torch, self.cfg
        pk, pv = self._floats(k, self._src, "k"), self._floats(v, self._src, "v")
        pck, pcv = self._floats(cache_k, self._cache, "cache_k"), self._floats(cache_v, self._cache, "cache_v")
        strides = k.stride(), v.stride(), cache_k.stride(), cache_v.stride()
        if strides != self._strides:
            ks, vs, cs = _steps(k, "k"), _steps(v, "v"), _steps(cache_k, "cache_k")
            _need(_steps(cache_v, "cache_v") == cs, "KvCommit: both caches have the same strides")
            c.src_stride[:], c.v_stride[:], c.cache_stride[:] = ks, vs, cs
            c.own_v_stride, self._strides = 1, strides
        ps = self._ints(slots, t.int64, self._places, "slots")
        pp = self._opt(path, t.int32, self._places, "path")
        self._launch(stream, self._lib.stand_kv_commit, self._cfg_ptr, pk, pv, pp, ps, pck, pcv)


class LogitsProcessor(_Op):
    """Penalties, biases and grammar masks on the logits of every node (stand_process_logits)."""

    def __init__(self, B, N, V, dtype, parent=None, device="cuda:0"):
        self._init_device(device)
        t = self.torch
        _need(dtype in (t.float32, t.bfloat16), "LogitsProcessor: float32 or bfloat16 logits")
        _need(B >= 1 and N >= 1 and V >= 2 and (parent is not None or N == 1) and (parent is None or len(parent) == N),
              "LogitsProcessor: invalid shapes")
        self.dtype = dtype
        self._parent = None if parent is None else np.ascontiguousarray(parent, np.int32)
        self.cfg = StandLogits(B, N, V, _dtype_code(dtype), None if parent is None else self._parent.ctypes.data)
        self.inputs = StandLogitsInputs()
        self._shape, self._b, self._nodes, self._starts = (B, N, V), (B,), (B, N), (B + 1,)
        self._rows, self._words = (B * N,), (V + 31) // 32
        self._out = None
        self._cfg_ptr, self._in_ptr = C.addressof(self.cfg), C.addressof(self.inputs)

    def _logits(self, x, what):
        """Address and row stride of [B, N, V] logits whose rows are evenly spaced."""
        B, N, V = self._shape
        if x.dtype is not self.dtype or x.shape != self._shape or x.get_device() != self._index:
            raise StandError(f"{what}: wants a {self.dtype} tensor {self._shape} on {self.dev}")
        sb, sn, sv = x.stride()
        row = sn if N > 1 else (sb if B > 1 else V)
        if sv != 1 or row < V or (B > 1 and N > 1 and sb != N * sn):
            raise StandError(f"{what}: rows of V contiguous logits, evenly spaced")
        return x.data_ptr(), row

    def __call__(self, logits, text=None, n_text=None, n_prompt=None, tree_tokens=None, repetition=None, frequency=None,
                 presence=None, bias_start=None, bias_id=None, bias_value=None, mask=None, mask_row=None, out=None, stream=None):
        """logits [B, N, V]; text [B, any] int32 with n_text / n_prompt [B] int64; tree_tokens [B, N] int32; penalties
        [B] float32; biases in CSR form; mask [masks, ceil(V/32)] int32 bits with mask_row [B, N] (or [B * N]) int32.
        out: the tensor to write (`logits` itself: in place); None: a tensor kept by this object.  Returns it."""
        t, c, x = self.torch, self.cfg, self.inputs
        src, c.in_stride = self._logits(logits, "logits")
        if out is None:
            if self._out is None:
                self._out = t.empty(self._shape, dtype=self.dtype, device=self.dev)
            out = self._out
        dst, c.out_stride = self._logits(out, "out")
        i32, i64, f32 = t.int32, t.int64, t.float32
        c.text_stride = 0
        if text is not None:
            _need(text.dim() == 2 and n_text is not None, "text: [B, any], with n_text")
            c.text_stride = text.shape[1]
            x.text = self._ints(text, i32, (self._b[0], c.text_stride), "text")
        else:
            _need(n_text is None and n_prompt is None, "n_text and n_prompt go with text")
            x.text = None
        x.n_text = self._opt(n_text, i64, self._b, "n_text")
        x.n_prompt = self._opt(n_prompt, i64, self._b, "n_prompt")
        x.tree_tokens = self._opt(tree_tokens, i32, self._nodes, "tree_tokens")
        x.repetition = self._opt(repetition, f32, self._b, "repetition")
        x.frequency = self._opt(frequency, f32, self._b, "frequency")
        x.presence = self._opt(presence, f32, self._b, "presence")
        x.bias_start = self._opt(bias_start, i32, self._starts, "bias_start")
        if bias_start is not None:
            _need(bias_id is not None and bias_value is not None and bias_id.dim() == 1 and bias_id.shape == bias_value.shape,
                  "biases: bias_start, bias_id and bias_value go together")
            x.bias_id = self._ints(bias_id, i32, bias_id.shape, "bias_id")
            x.bias_value = self._ints(bias_value, f32, bias_id.shape, "bias_value")
        else:
            _need(bias_id is None and bias_value is None, "biases: bias_start, bias_id and bias_value go together")
            x.bias_id = x.bias_value = None
        c.biases = 0 if bias_id is None else bias_id.shape[0]
        c.masks = 0
        if mask is not None:
            _need(mask_row is not None and mask.dim() == 2, "mask: [masks, ceil(V/32)], with mask_row")
            c.masks = mask.shape[0]
            x.mask = self._ints(mask, i32, (c.masks, self._words), "mask")
            x.mask_row = self._ints(mask_row, i32, self._rows if mask_row.dim() == 1 else self._nodes, "mask_row")
        else:
            _need(mask_row is None, "mask_row goes with mask")
            x.mask = x.mask_row = None
        self._launch(stream, self._lib.stand_process_logits, self._cfg_ptr, self._in_ptr, src, dst)
        return out
