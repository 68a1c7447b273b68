"""Verification of a tree of drafted tokens over a paged key/value cache: torch-tensor arguments for the
``dflare_cache_*``, ``dflare_rope*`` and ``dflare_tree_*`` calls of include/dflare.h, which says what each
computes. Tensors are CUDA tensors of one device: the cache's, or the current one for calls without a cache. Calls are
enqueued on that device's current torch stream unless one of its streams is given, and a tensor that was made on
another stream must be ready there. Nothing is computed here.

A block step of a target model:

    tree_plan(parents, n_nodes, mask, depth)
    cache.reserve(n_nodes)
    for layer in range(n_layers):
        cache.append(layer, q, k, v, n_nodes, phase, q, depth=depth)      # q rotated in place
        cache.attend(layer, q, n_nodes, out, mask=mask)
    tree_accept(tokens, parents, choice, n_nodes, accept_len, path, next_token)
    cache.commit(accept_len, path)
"""
from __future__ import annotations

import ctypes

import torch

from . import _lib

_I32, _I64, _F32, _BF16 = torch.int32, torch.int64, torch.float32, torch.bfloat16


# These calls take a few microseconds on the device, so the host's part counts: torch.cuda.current_stream()
# makes a Stream object in 2.9 us (measured on the host's Arm cores), the plain handle is there in 0.2.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _current():
    return torch.cuda.current_device() if _device is None else _device()


def _stream(stream, device):
    if stream is None:
        return torch.cuda.current_stream(device).cuda_stream if _raw_stream is None else _raw_stream(device)
    if getattr(stream, "device_index", device) != device:
        raise ValueError(f"stream must be one of cuda:{device}, got one of cuda:{stream.device_index}")
    return stream.cuda_stream


def _on(name, t, device):
    """Memory of another device must not reach a kernel."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.get_device() != device:
        raise ValueError(f"{name} must be on cuda:{device}, got {t.device}")


def _check(status):
    if status:
        _lib.check(status, None)


def _ints(name, t, numel, device):
    """An int32 tensor on the device of at least numel elements, without gaps; its address."""
    if t.dtype is _I32 and t.get_device() == device and t.is_contiguous() and t.numel() >= numel:
        return t.data_ptr()
    _on(name, t, device)
    if t.dtype is not _I32:
        raise ValueError(f"{name} must be torch.int32, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    raise ValueError(f"{name} holds {t.numel()} elements, needs at least {numel}")


def _typed(name, t, dtype, device):
    if t.dtype is dtype and t.get_device() == device:
        return
    _on(name, t, device)
    raise ValueError(f"{name} must be {dtype}, got {t.dtype}")


def _rows(name, t, dtype, shape, device):
    """A [batch][rows][heads][head_dim] tensor whose heads are adjacent and whose rows are evenly spaced
    (a part of a fused projection's rows, for one); its address and row stride in elements."""
    _typed(name, t, dtype, device)
    if t.shape != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(t.shape)}")
    b, n, heads, hd = shape
    sb, sn, sh, sd = t.stride()
    if n == 1:
        sn = sb if b > 1 else heads * hd       # one row per sequence: their distance is the stride
    if (sd != 1 and hd > 1) or (sh != hd and heads > 1) or (b > 1 and sb != n * sn):
        raise ValueError(f"{name}: heads must be adjacent and rows evenly spaced, got strides {list(t.stride())}")
    return t.data_ptr(), sn


def rope_phases(rot_dim, theta=1e6, scaling="none", factor=1.0, trained=4096, beta_fast=32.0, beta_slow=1.0,
                device="cuda"):
    """The phases of ``rot_dim`` rotated elements (int64 [rot_dim / 2], what the rotary calls take) and the
    factor on the rotated values. scaling: "none", "linear", "ntk" or "yarn"."""
    if scaling not in _lib.ROPE_SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(_lib.ROPE_SCALINGS)}, got {scaling!r}")
    g = _lib.RopeConfig(rot_dim, _lib.ROPE_SCALINGS[scaling], theta, factor, trained, beta_fast, beta_slow)
    out = torch.zeros(max(int(rot_dim) // 2, 1), dtype=_I64)
    magnitude = ctypes.c_float(0.0)
    _check(_lib.load().dflare_rope_phases(ctypes.byref(g), out.data_ptr(), ctypes.byref(magnitude)))
    return out.to(device), magnitude.value


def _phase(phase, device):
    _typed("phase", phase, _I64, device)
    if not phase.is_contiguous():
        raise ValueError("phase must be contiguous")
    return phase.data_ptr()


def _layout(layout):
    if layout not in _lib.ROPE_LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(_lib.ROPE_LAYOUTS)}, got {layout!r}")
    return _lib.ROPE_LAYOUTS[layout]


def rope(x, positions, phase, out, *, layout="half", magnitude=1.0, backward=False, stream=None):
    """Rotary embedding of x [rows][heads][head_dim] at int32 positions [rows] into out (x itself: in place).
    The first 2 * len(phase) elements of each head are rotated, the others copied. ``backward=True`` applies
    the transposed map, the gradient's."""
    if x.dim() != 3 or out.shape != x.shape:
        raise ValueError(f"x and out must be [rows][heads][head_dim], got {list(x.shape)} and {list(out.shape)}")
    dtype = x.dtype
    if dtype is not _BF16 and dtype is not _F32:
        raise ValueError(f"x must be torch.bfloat16 or torch.float32, got {dtype}")
    dev = _current()
    _typed("x", x, dtype, dev)
    _typed("out", out, dtype, dev)
    rows, heads, hd = x.shape
    x0, x1, x2 = x.stride()
    o0, o1, o2 = out.stride()
    if (x2 != 1 or o2 != 1) and hd > 1:
        raise ValueError("the elements of a head must be adjacent")
    _check(_lib.load().dflare_rope(x.data_ptr(), x0, x1, out.data_ptr(), o0, o1, _ints("positions", positions, rows, dev), _phase(phase, dev),
                                   rows, heads, hd, 2 * phase.numel(), _layout(layout), magnitude, backward,
                                   _lib.DFLARE_BF16 if dtype is _BF16 else _lib.DFLARE_F32, _stream(stream, dev)))


def tree_plan(parents, n_nodes, mask, depth, error=None, stream=None):
    """Ancestor bits (int32 [batch][n][ceil(n / 32)]) and depths (int32 [batch][n]) of the trees with parent
    numbers ``parents`` int32 [batch][n]. error: optional int32 [1] that gets DEVERR_TREE for an impossible tree."""
    if parents.dim() != 2:
        raise ValueError(f"parents must be [batch][n], got {list(parents.shape)}")
    batch, n = parents.shape
    dev = _current()
    pp = _ints("parents", parents, 0, dev)
    _check(_lib.load().dflare_tree_plan(pp, _ints("n_nodes", n_nodes, batch, dev), batch, n,
                                        _ints("mask", mask, batch * n * ((n + 31) // 32), dev), _ints("depth", depth, batch * n, dev),
                                        None if error is None else _ints("error", error, 1, dev), _stream(stream, dev)))


def tree_accept(tokens, parents, choice, n_nodes, accept_len, path, next_token, error=None, stream=None):
    """Greedy acceptance in drafted trees: tokens, parents and choice (the target's argmax after each node)
    int32 [batch][n]; writes accept_len [batch], path [batch][n], next_token [batch]. error: as in tree_plan."""
    if parents.dim() != 2:
        raise ValueError(f"parents must be [batch][n], got {list(parents.shape)}")
    batch, n = parents.shape
    dev = _current()
    pp = _ints("parents", parents, 0, dev)
    _check(_lib.load().dflare_tree_accept(
        _ints("tokens", tokens, batch * n, dev), pp, _ints("choice", choice, batch * n, dev), _ints("n_nodes", n_nodes, batch, dev), batch, n,
        _ints("accept_len", accept_len, batch, dev), _ints("path", path, batch * n, dev), _ints("next_token", next_token, batch, dev),
        None if error is None else _ints("error", error, 1, dev), _stream(stream, dev)))


class PagedCache:
    """Keys and values of a model in pages that sequences share (see dflare_cache_create).

    ``PagedCache.allocate`` makes an empty one; the constructor takes a caller's tensors:
    k, v [n_layers][n_pages][n_kv_heads][page_size][head_dim] (bf16 or fp32) and the int32 tables. The
    tensors stay the caller's to read between calls.
    """

    def __init__(self, *, k, v, table, lens, held, refs, free, n_free, n_q_heads, max_nodes):
        self._cache = ctypes.c_void_p()
        if not k.is_cuda:
            raise ValueError("k must be a CUDA tensor")
        self.device_index = dev = k.get_device()
        if k.dim() != 5 or v.shape != k.shape:
            raise ValueError("k and v must be [n_layers][n_pages][n_kv_heads][page_size][head_dim]")
        if k.dtype is not _BF16 and k.dtype is not _F32:
            raise ValueError(f"k must be torch.bfloat16 or torch.float32, got {k.dtype}")
        for name, t in (("k", k), ("v", v)):
            _typed(name, t, k.dtype, dev)
            if not t.is_contiguous():
                raise ValueError(f"{name} must be contiguous")
        if table.dim() != 2:
            raise ValueError("table must be [max_batch][max_pages]")
        self._L = _lib.load()
        self.n_layers, self.n_pages, self.n_kv_heads, self.page_size, self.head_dim = k.shape
        self.max_batch, self.max_pages = table.shape
        self.n_q_heads, self.max_nodes, self.dtype = n_q_heads, max_nodes, k.dtype
        b = _lib.CacheBuffers(k.data_ptr(), v.data_ptr(), _ints("table", table, 0, dev), _ints("lens", lens, self.max_batch, dev),
                              _ints("held", held, self.max_batch, dev), _ints("refs", refs, self.n_pages, dev),
                              _ints("free", free, self.n_pages, dev), _ints("n_free", n_free, 1, dev))
        self.cfg = _lib.CacheConfig(self.n_layers, self.n_pages, self.page_size, n_q_heads, self.n_kv_heads, self.head_dim,
                                    self.max_batch, self.max_pages, max_nodes,
                                    _lib.DFLARE_BF16 if k.dtype is _BF16 else _lib.DFLARE_F32)
        self.k, self.v, self.table, self.lens, self.held = k, v, table, lens, held
        self.refs, self.free, self.n_free = refs, free, n_free
        with torch.cuda.device(k.device):
            _check(self._L.dflare_cache_create(ctypes.byref(self.cfg), ctypes.byref(b), ctypes.byref(self._cache)))

    @classmethod
    def allocate(cls, *, n_layers, n_pages, page_size, n_q_heads, n_kv_heads, head_dim, max_batch, max_pages, max_nodes,
                 dtype="bf16", device="cuda"):
        """An empty cache with memory of its own."""
        t = _BF16 if dtype == "bf16" else _F32
        shape = (n_layers, n_pages, n_kv_heads, page_size, head_dim)

        def ints(*s):
            return torch.zeros(s, dtype=_I32, device=device)

        return cls(k=torch.empty(shape, dtype=t, device=device), v=torch.empty(shape, dtype=t, device=device),
                   table=ints(max_batch, max_pages) - 1, lens=ints(max_batch), held=ints(max_batch), refs=ints(n_pages),
                   free=torch.arange(n_pages - 1, -1, -1, dtype=_I32, device=device), n_free=ints(1) + n_pages,
                   n_q_heads=n_q_heads, max_nodes=max_nodes)

    def close(self):
        if self._cache:
            self._L.dflare_cache_destroy(self._cache)
            self._cache = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def error(self, stream=None) -> int:
        """DEVERR_* bits that kernels have set since the last call (synchronises the stream)."""
        bits = ctypes.c_uint32(0)
        st = self._L.dflare_cache_error(self._cache, ctypes.byref(bits), _stream(stream, self.device_index))
        if st not in (_lib.DFLARE_OK, _lib.DFLARE_EDEVICE):
            _check(st)
        return bits.value

    def reserve(self, n_new, stream=None):
        """Room for n_new [batch] tokens behind every sequence's length (all sequences or none)."""
        dev = self.device_index
        _check(self._L.dflare_cache_reserve(self._cache, _ints("n_new", n_new, 1, dev), n_new.numel(), _stream(stream, dev)))

    def append(self, layer, q, k, v, n_new, phase, q_out, *, depth=None, layout="half", magnitude=1.0, stream=None):
        """A layer's new tokens: q [batch][n][n_q_heads][head_dim] rotated into q_out (q itself: in place), k
        and v [batch][n][n_kv_heads][head_dim] into the pages. q and q_out None: keys and values only. phase
        None: no rotation. depth int32 [batch][n]: positions relative to lens (None: 0, 1, 2, ...)."""
        dev = self.device_index
        batch, n = k.shape[:2]
        kv = (batch, n, self.n_kv_heads, self.head_dim)
        kp, ks = _rows("k", k, self.dtype, kv, dev)
        vp, vs = _rows("v", v, self.dtype, kv, dev)
        qp = op = None
        qs = os_ = 0
        if q is not None or q_out is not None:
            if q is None or q_out is None:
                raise ValueError("q and q_out go together")
            shape = (batch, n, self.n_q_heads, self.head_dim)
            qp, qs = _rows("q", q, self.dtype, shape, dev)
            op, os_ = (qp, qs) if q_out is q else _rows("q_out", q_out, self.dtype, shape, dev)
        _check(self._L.dflare_cache_append(
            self._cache, layer, qp, qs, kp, ks, vp, vs, op, os_,
            None if depth is None else _ints("depth", depth, batch * n, dev), _ints("n_new", n_new, batch, dev), batch, n,
            None if phase is None else _phase(phase, dev), 0 if phase is None else 2 * phase.numel(), _layout(layout), magnitude,
            _stream(stream, dev)))

    def attend(self, layer, q, n_nodes, out, *, mask=None, scale=None, lse=None, stream=None):
        """Attention of q [batch][n][n_q_heads][head_dim] over the pages into out (contiguous). mask: the
        ancestor bits of tree_plan (None: node i sees nodes 0 .. i). scale: head_dim^-0.5 if None. lse: optional
        fp32 [batch][n][n_q_heads]."""
        dev = self.device_index
        if q.dim() != 4:
            raise ValueError(f"q must be [batch][n][n_q_heads][head_dim], got {list(q.shape)}")
        batch, n = q.shape[:2]
        qp, qs = _rows("q", q, self.dtype, (batch, n, self.n_q_heads, self.head_dim), dev)
        _typed("out", out, self.dtype, dev)
        if out.shape != q.shape or not out.is_contiguous():
            raise ValueError(f"out must be contiguous {list(q.shape)}, got {list(out.shape)}")
        lp = None
        if lse is not None:
            _typed("lse", lse, _F32, dev)
            if lse.numel() < batch * n * self.n_q_heads or not lse.is_contiguous():
                raise ValueError(f"lse must be contiguous and hold {batch * n * self.n_q_heads} elements")
            lp = lse.data_ptr()
        _check(self._L.dflare_cache_attend(
            self._cache, layer, qp, qs, None if mask is None else _ints("mask", mask, batch * n * ((n + 31) // 32), dev),
            _ints("n_nodes", n_nodes, batch, dev), batch, n, self.head_dim ** -0.5 if scale is None else scale, out.data_ptr(), lp,
            _stream(stream, dev)))

    def commit(self, accept_len, path, stream=None):
        """Keep the nodes path[b][: accept_len[b]] (int32 [batch], [batch][n]) behind every length, moved
        together, and give the other pages back."""
        dev = self.device_index
        if path.dim() != 2:
            raise ValueError(f"path must be [batch][n], got {list(path.shape)}")
        batch, row = path.shape
        _check(self._L.dflare_cache_commit(self._cache, _ints("accept_len", accept_len, batch, dev), _ints("path", path, 0, dev), row, batch,
                                           _stream(stream, dev)))

    def truncate(self, new_len, stream=None):
        """Cut sequences to new_len [batch] tokens at most; 0 ends one. Pages past that are given back."""
        dev = self.device_index
        _check(self._L.dflare_cache_truncate(self._cache, _ints("new_len", new_len, 1, dev), new_len.numel(), _stream(stream, dev)))

    def fork(self, src, dst, stream=None):
        """Sequences dst [n] (which hold nothing) become copies of sequences src [n] that share their pages."""
        dev = self.device_index
        _check(self._L.dflare_cache_fork(self._cache, _ints("src", src, 1, dev), _ints("dst", dst, src.numel(), dev), src.numel(),
                                         _stream(stream, dev)))

    def copy_pages(self, src, dst, stream=None):
        """Copy pages src [n] to pages dst [n] in every layer."""
        dev = self.device_index
        _check(self._L.dflare_cache_copy_pages(self._cache, _ints("src", src, 1, dev), _ints("dst", dst, src.numel(), dev), src.numel(),
                                               _stream(stream, dev)))
