"""Binding of the key/value cache and the attention over it (include/fbq.h): argument marshalling only.

A `Cache` is a pool of pages and, on the device like it, the table that says which pages hold which row's tokens:

    pool    [layers, pages, 2 (K, V), kv_heads, page_size, head_dim]   fp16 or bf16
    table   [rows, max_pages] int32, -1: none        lengths [rows] int32        refs [pages] int32

A cache in 4 bits has a pool of uint8, [layers, pages, 2, kv_heads, page_size, token_bytes(head_dim)], and everything else alike (layout: include/fbq.h); what goes in and comes out
is fp16 or bf16, its `dtype`.

`cache_reserve` gives rows pages for new tokens, `cache_append` writes a layer's keys and values there, `attention` reads them; `cache_fork`, `cache_free`,
`cache_copy` and `cache_compact` move whole sequences and pages about; `cache_read` gives tokens back as fp32.  Nothing here waits for the device or asks it anything, so all of it can be captured
in a graph; what could not be served stands in the `info` tensors.
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass, field
from typing import Optional

from . import fbq
from .fbq import FbqError, _check, _dev_ptr, _on, _result, _stream  # noqa: F401


class _CCacheDesc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("layers", "pages", "page_size", "kv_heads", "head_dim", "type")]


class _CCache(ctypes.Structure):
    _fields_ = [("desc", _CCacheDesc), ("rows", ctypes.c_int32), ("max_pages", ctypes.c_int32), ("pool", ctypes.c_void_p), ("table", ctypes.c_void_p),
                ("lengths", ctypes.c_void_p), ("refs", ctypes.c_void_p)]


class _CAttentionCall(ctypes.Structure):
    _fields_ = [("cache", _CCache), ("layer", ctypes.c_int32), ("heads", ctypes.c_int32), ("T", ctypes.c_int32), ("max_q", ctypes.c_int32),
                ("q_start", ctypes.c_void_p), ("q", ctypes.c_void_p), ("q_stride", ctypes.c_int64), ("out", ctypes.c_void_p), ("out_stride", ctypes.c_int64),
                ("lse", ctypes.c_void_p), ("shared", ctypes.c_void_p), ("n_shared", ctypes.c_int32), ("scale", ctypes.c_float)]


_call = None                    # the compiled calls' module and the addresses of what they call, once the library is loaded
_int32 = _float32 = _types = None


def declare(lib) -> None:
    """Argument types of the entry points (called once, when the library is loaded)."""
    vp, sz, i32, i64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int64
    dp, cp, ap = ctypes.POINTER(_CCacheDesc), ctypes.POINTER(_CCache), ctypes.POINTER(_CAttentionCall)
    for name, res, args in (("fbq_check_cache", i32, [dp]), ("fbq_cache_bytes", sz, [dp]), ("fbq_cache_workspace_bytes", sz, [dp, i32]),
                            ("fbq_cache_reserve", i32, [cp, vp, vp, vp, vp]), ("fbq_cache_append", i32, [cp, i32, i32, vp, vp, vp, i64, vp, i64, vp]),
                            ("fbq_cache_free", i32, [cp, i32, vp, vp]), ("fbq_cache_fork", i32, [cp, i32, vp, vp, vp, vp, sz, vp]),
                            ("fbq_cache_copy", i32, [cp, i32, vp, vp, vp]), ("fbq_cache_compact", i32, [cp, vp, vp, vp, vp, sz, vp]),
                            ("fbq_attention_weights", i32, [ap, vp, vp, i32, ctypes.c_float, vp]), ("fbq_cache_evict_workspace_bytes", sz, [cp, i32]),
                            ("fbq_cache_evict", i32, [cp, vp, vp, i64, i32, vp, i32, i32, vp, vp, sz, vp]), ("fbq_cache_read", i32, [cp, i32, i32, vp, vp, vp, vp, vp]),
                            ("fbq_attention_workspace_bytes", sz, [ap]), ("fbq_attention", i32, [ap, vp, sz, vp])):
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    global _call, _int32, _float32, _types
    import torch
    from . import _fbq_call
    _int32, _float32, _types = torch.int32, torch.float32, {torch.float16: 0, torch.bfloat16: 1}
    _call = (_fbq_call, *(ctypes.cast(getattr(lib, n), vp).value for n in ("fbq_attention", "fbq_cache_append")))


def _ints(t, what: str, n: Optional[int] = None):
    """Pointer of a device int32 tensor (None: NULL)."""
    if t is None:
        return None
    if t.dtype != _int32 or (n is not None and t.numel() != n):
        raise ValueError(f"{what}: expected int32" + ("" if n is None else f", {n} of them"))
    return _dev_ptr(t)


def _like(t, stream):
    """A result of t's shape and type, of a call on `stream`."""
    if stream is None:
        return t.new_empty(t.shape)
    with _on(stream):
        result = t.new_empty(t.shape)
    return _result(result, stream)


def _info(t, n: int):
    """Pointer of a tensor that takes n numbers of what could not be served, or is told."""
    if t is not None and t.numel() < n:
        raise ValueError(f"info: expected int32, {n} of them")
    return _ints(t, "info")


def token_bytes(head_dim: int) -> int:
    """Bytes of a token's keys, or values, in one head of a cache in 4 bits: codes of 64, 96, 128, 192 or 256 features, and a word for each 64."""
    features = next((n for n in (64, 96, 128, 192, 256) if n >= head_dim), 0)
    return features // 2 + 4 * -(-features // 64)


@dataclass
class Cache:
    """A cache made of tensors that the caller keeps (see `cache_create`); `rows(a, b)` is the same cache with rows a .. b - 1 alone (compaction wants all of them).
    dtype, dim: of a cache in 4 bits the type of what goes in and comes out, and the features of a head; else the pool says them."""
    pool: "object"
    table: "object"
    lengths: "object"
    refs: "object"
    dtype: "object" = None
    dim: int = 0
    _c: "object" = field(init=False, repr=False, compare=False)
    _at: int = field(init=False, repr=False, compare=False)
    _part: bool = field(init=False, repr=False, compare=False, default=False)             # rows() of another: others hold pages of the pool, too
    _rooms: dict = field(init=False, repr=False, compare=False, default_factory=dict)     # the page operations' workspaces: stream -> [(pairs, workspace)] (see _room)

    def __post_init__(self):
        lib = fbq.load()
        four = self.dtype is not None and self.pool.dtype not in _types
        if self.pool.dim() != 6 or self.pool.shape[2] != 2 or (not four and self.pool.dtype not in _types):
            raise ValueError("pool: expected [layers, pages, 2, kv_heads, page_size, head_dim], float16 or bfloat16")
        if four and (str(self.pool.dtype) != "torch.uint8" or self.dtype not in _types or self.pool.shape[5] != token_bytes(self.dim)):
            raise ValueError("pool: in 4 bits, expected uint8 [layers, pages, 2, kv_heads, page_size, token_bytes(dim)], dtype float16 or bfloat16")
        if not four and (self.dtype not in (None, self.pool.dtype) or self.dim not in (0, self.pool.shape[5])):
            raise ValueError("dtype, dim: expected those of the pool")
        if self.table.dim() != 2:
            raise ValueError("table: expected [rows, max_pages]")
        layers, pages, _, kv_heads, page, dim = self.pool.shape
        rows, width = self.table.shape
        if not four:
            self.dtype, self.dim = self.pool.dtype, int(dim)
        d = _CCacheDesc(layers, pages, page, kv_heads, self.dim, _types[self.dtype] + (4 if four else 0))
        self._c = _CCache(d, rows, width, _dev_ptr(self.pool), _ints(self.table, "table"), _ints(self.lengths, "lengths", rows), _ints(self.refs, "refs", pages))
        _check(lib.fbq_check_cache(ctypes.byref(d)), "Cache")
        self._at = ctypes.addressof(self._c)

    def __setattr__(self, name, value):
        if name in ("pool", "table", "lengths", "refs", "dtype", "dim") and "_at" in self.__dict__:       # (their addresses are in `_c`: calls would go on with the old ones)
            raise AttributeError(f"{name}: a Cache keeps the tensors that it was made of; write into them, or make another Cache")
        object.__setattr__(self, name, value)

    @property
    def heads(self) -> int:
        return int(self.pool.shape[3])

    @property
    def head_dim(self) -> int:
        return self.dim

    @property
    def page_size(self) -> int:
        return int(self.pool.shape[4])

    def rows(self, first: int, end: int) -> "Cache":
        part = Cache(self.pool, self.table[first:end], self.lengths[first:end], self.refs, self.dtype, self.dim)
        part._part = self._part or part.table.shape[0] < self.table.shape[0]
        return part


def cache_create(layers: int, pages: int, page_size: int, kv_heads: int, head_dim: int, rows: int, max_pages: int, dtype=None, device="cuda", bits: int = 16) -> Cache:
    """An empty cache: `rows` sequences of up to max_pages * page_size tokens, out of `pages` pages in all.  dtype: torch.float16 (default) or torch.bfloat16.  bits: 16, or 4."""
    import torch
    if bits not in (4, 16):
        raise ValueError("bits: expected 16 or 4")
    i32 = lambda v, *shape: torch.full(shape, v, dtype=torch.int32, device=device)
    dtype = dtype or torch.float16
    pool = torch.empty((layers, pages, 2, kv_heads, page_size, head_dim if bits == 16 else token_bytes(head_dim)), dtype=dtype if bits == 16 else torch.uint8, device=device)
    return Cache(pool, i32(-1, rows, max_pages), i32(0, rows), i32(0, pages), dtype, head_dim)


def cache_reserve(cache: Cache, count, start=None, info=None, stream=None):
    """fbq_cache_reserve: pages for count[b] more tokens of each row -> start [rows], where they begin (-1: no pages left for this row)."""
    if start is None:
        start = _like(cache.lengths, stream)
    rows = cache._c.rows
    _check(fbq.load().fbq_cache_reserve(cache._c, _ints(count, "count", rows), _ints(start, "start", rows), _info(info, 1), _stream(stream)),
           "fbq_cache_reserve")
    return start


def _tokens(cache: Cache, t, what: str, heads: Optional[int] = None):
    """(pointer, elements between rows, tokens) of a [T, heads, head_dim] tensor of the cache's type whose rows may lie further apart."""
    if t.dim() != 3 or t.dtype != cache.dtype or t.shape[2] != cache.head_dim or (heads is not None and t.shape[1] != heads):
        raise ValueError(f"{what}: expected [T, heads, head_dim] of the cache's type")
    if t.stride(2) != 1 or (t.stride(1) != t.shape[2] and t.shape[1] > 1):
        raise ValueError(f"{what}: a token's heads have to lie in one piece")
    if not t.is_cuda:
        raise ValueError("expected a device tensor")
    T = int(t.shape[0])
    return t.data_ptr(), (t.stride(0) if T > 1 else t.shape[1] * t.shape[2]), T


def cache_append(cache: Cache, layer: int, k, v, start, q_start=None, stream=None) -> None:
    """fbq_cache_append: k, v [T, kv_heads, head_dim] of one layer into the pages of their rows, from position start[b] on (see cache_reserve).
    q_start [rows + 1]: the rows' tokens in k and v; None: one token a row."""
    rc = _call[0].append(_call[2], cache._at, cache.dtype, _int32, layer, k, v, start, q_start, _stream(stream))
    if rc is not None:                                        # (None: something is not as it should be; below it is named)
        return _check(rc, "fbq_cache_append")
    kp, ks, T = _tokens(cache, k, "k", cache.heads)
    vp, vs, Tv = _tokens(cache, v, "v", cache.heads)
    if T != Tv:
        raise ValueError("k and v: as many tokens")
    rows = cache._c.rows
    _check(fbq.load().fbq_cache_append(cache._c, int(layer), T, _ints(q_start, "q_start", rows + 1), _ints(start, "start", rows), kp, ks, vp, vs,
                                       _stream(stream)), "fbq_cache_append")


def cache_read(cache: Cache, layer: int, tokens: int, start, q_start=None, k=None, v=None, stream=None):
    """fbq_cache_read: the tokens from position start[b] on of each row as numbers -> (k, v), float32 [tokens, kv_heads, head_dim].  q_start [rows + 1]: how many of each row, and where
    they go; None: one a row, and `tokens` is the number of rows.  Where start[b] is -1, or there is no page, nothing is written."""
    shape = (tokens, cache.heads, cache.head_dim)
    rows = cache._c.rows
    for t, what in ((k, "k"), (v, "v")):
        if t is not None and (t.dtype != _float32 or tuple(t.shape) != shape):
            raise ValueError(f"{what}: expected float32 [tokens, kv_heads, head_dim]")
    at, places = _ints(start, "start", rows), _ints(q_start, "q_start", rows + 1)
    k, v = (fbq._empty(shape, "float32", cache.pool.device, stream) if t is None else t for t in (k, v))
    _check(fbq.load().fbq_cache_read(cache._c, int(layer), tokens, places, at, _dev_ptr(k), _dev_ptr(v), _stream(stream)), "fbq_cache_read")
    return k, v


def cache_free(cache: Cache, rows, stream=None) -> None:
    """fbq_cache_free: empties the rows of an int32 list."""
    _check(fbq.load().fbq_cache_free(cache._c, rows.numel(), _ints(rows, "rows"), _stream(stream)), "fbq_cache_free")


def _room(cache: Cache, n: int, stream, number: int):
    """Workspace of a page operation that was given none; the cache keeps one for every stream, allocated there, since operations on one cache's rows and reference counts have to
    follow each other anyway.  A smaller one is kept beside a larger: a captured graph may hold it."""
    rooms = cache._rooms.get(number)                          # (number: the stream's)
    if rooms is None or n > rooms[-1][0]:
        import torch
        rooms = cache._rooms.setdefault(number, [])
        pairs, size = max(n, 256), fbq.load().fbq_cache_workspace_bytes
        with _on(stream):
            rooms.append((pairs, torch.empty(max(size(cache._c.desc, min(pairs, 65536)), size(cache._c.desc, 0)), dtype=torch.uint8, device=cache.pool.device)))
    return rooms[-1][1]


def _size(workspace) -> int:
    return 0 if workspace is None else workspace.numel() * workspace.element_size()


def cache_fork(cache: Cache, parent, child, info=None, workspace=None, stream=None) -> None:
    """fbq_cache_fork: row child[i] becomes a second holder of what row parent[i] holds.  info: int32 [2], pages lacking and pairs skipped."""
    n, number = parent.numel(), _stream(stream)
    if workspace is None:
        workspace = _room(cache, n, stream, number)
    _check(fbq.load().fbq_cache_fork(cache._c, n, _ints(parent, "parent"), _ints(child, "child", n), _info(info, 2), _dev_ptr(workspace),
                                     _size(workspace), number), "fbq_cache_fork")


def cache_copy(cache: Cache, src, dst, stream=None) -> None:
    """fbq_cache_copy: page dst[i] = page src[i] in all layers (int32 lists)."""
    n = src.numel()
    _check(fbq.load().fbq_cache_copy(cache._c, n, _ints(src, "src"), _ints(dst, "dst", n), _stream(stream)), "fbq_cache_copy")


def cache_compact(cache: Cache, out: Optional[Cache] = None, info=None, workspace=None, stream=None) -> Cache:
    """fbq_cache_compact: live pages to the low end of the pool.  out: a Cache of the same pool whose table and refs take the new ones (None: in place); its lengths are left
    alone.  info: int32 [2], pages in use and pages moved."""
    out = cache if out is None else out
    if cache._part or out._part:                              # (the other rows' table would name pages that have moved)
        raise ValueError("compaction: of all rows that hold pages, not of a part of them")
    if out.pool.data_ptr() != cache.pool.data_ptr() or out.pool.shape != cache.pool.shape or out.pool.dtype != cache.pool.dtype:
        raise ValueError("out: a cache of the same pool")
    if out.table.shape != cache.table.shape or out.refs.shape != cache.refs.shape:
        raise ValueError("out: a cache of the same shape")
    number = _stream(stream)
    if workspace is None:
        workspace = _room(cache, 0, stream, number)
    _check(fbq.load().fbq_cache_compact(cache._c, out._c.table, out._c.refs, _info(info, 2), _dev_ptr(workspace), _size(workspace),
                                        number), "fbq_cache_compact")
    return out


def _arguments(cache: Cache, layer: int, q, q_start, max_q: int, shared, scale, out, lse) -> _CAttentionCall:
    qp, qs, T = _tokens(cache, q, "q")
    heads = int(q.shape[1])
    op, os_ = (None, heads * cache.head_dim) if out is None else _tokens(cache, out, "out", heads)[:2]
    if out is not None and out.shape[0] != T:
        raise ValueError("out: expected q's shape")
    if lse is not None:
        if lse.dtype != _float32 or tuple(lse.shape) != (T, heads):
            raise ValueError("lse: expected float32 [T, heads]")
    return _CAttentionCall(cache._c, int(layer), heads, T, int(max_q), _ints(q_start, "q_start", cache._c.rows + 1), qp, qs, op, os_, _dev_ptr(lse),
                           _ints(shared, "shared"), 0 if shared is None else shared.numel(), cache.head_dim ** -0.5 if scale is None else float(scale))


def attention_workspace(cache: Cache, q, q_start=None, max_q: int = 1, shared=None):
    """A workspace for attention() calls with queries, rows and shared pages like these.  A T that differs, max_q and the number of shared pages change its size."""
    import torch
    if q_start is None and max_q > 1:                         # (only its presence counts)
        q_start = torch.empty(cache._c.rows + 1, dtype=torch.int32, device=q.device)
    c = _arguments(cache, 0, q, q_start, max_q, shared, None, None, None)
    return torch.empty(max(16, fbq.load().fbq_attention_workspace_bytes(ctypes.byref(c))), dtype=torch.uint8, device=q.device)


def attention(cache: Cache, layer: int, q, q_start=None, max_q: int = 1, shared=None, scale=None, out=None, lse=None, workspace=None, stream=None):
    """fbq_attention: q [T, heads, head_dim], the newest tokens of the rows, over all the rows hold, causal -> out [T, heads, head_dim].

    q_start [rows + 1]: the rows' tokens in q, at most max_q a row; None: one token a row.  shared: the pages that all rows' tables begin with, read once
    for all rows.  scale: head_dim ** -0.5 by default.  lse: float32 [T, heads], takes the logarithm of the softmax's sums.
    """
    if out is None:
        out = _like(q, stream)
    scale = cache.head_dim ** -0.5 if scale is None else float(scale)
    # one row of 33 tokens, us a call: 9.4 by way of ctypes' argument objects, 6.0 this way
    rc = _call[0].attention(_call[1], cache._at, cache.dtype, _int32, _float32, layer, q, q_start, max_q, shared, scale, out, lse, workspace, _stream(stream))
    if rc is not None and (rc != 1 or workspace is not None):  # (1, a null pointer: the workspace, where none was given)
        _check(rc, "fbq_attention")
        return out
    import torch
    c = _arguments(cache, layer, q, q_start, max_q, shared, scale, out, lse)
    lib = fbq.load()
    if workspace is None:
        with _on(stream):
            workspace = torch.empty(max(16, lib.fbq_attention_workspace_bytes(ctypes.byref(c))), dtype=torch.uint8, device=q.device)
    _check(lib.fbq_attention(ctypes.byref(c), _dev_ptr(workspace), _size(workspace), _stream(stream)), "fbq_attention")
    return out


def _weights(t, what: str, shape):
    """Pointer of a float32 device tensor of the shape [rows, kv_heads, ..], the last one any."""
    if t is None:
        return None
    if t.dtype != _float32 or t.dim() != len(shape) + 1 or tuple(t.shape[:-1]) != shape:
        raise ValueError(f"{what}: expected float32 [{', '.join(['layers'] * (len(shape) - 2) + ['rows', 'kv_heads', 'width'])}] of the cache")
    return _dev_ptr(t)


def attention_weights(cache: Cache, layer: int, q, lse, weights, q_start=None, max_q: int = 1, scale=None, decay: float = 1.0, out=None, stream=None):
    """fbq_attention_weights, after attention() of the same q, q_start, max_q and scale, which wrote lse: what each key was attended to, for every key/value head over its queries -> out.

    weights: float32 [rows, kv_heads, width], what earlier calls added up (times decay; the row's new tokens begin at 0), or None; out: the same shape, weights itself by default.
    Tokens from width on are not counted; places without a token, and rows without queries, are left alone.
    A row that cache_reserve left out has no new tokens: it wants a Cache with a length of 0 for it here (decode_loop.py makes one), or the last ones that it holds count as new.
    """
    if out is None:
        out = weights
    if out is None:
        raise ValueError("weights or out: expected one of them")
    heads = (int(cache._c.rows), cache.heads)
    to, at = _weights(out, "out", heads), _weights(weights, "weights", heads)
    if weights is not None and weights.shape != out.shape:
        raise ValueError("out: expected the shape of weights")
    if lse is None:
        raise ValueError("lse: expected what attention() wrote")
    c = _arguments(cache, layer, q, q_start, max_q, None, scale, None, lse)
    _check(fbq.load().fbq_attention_weights(ctypes.byref(c), at, to, out.shape[-1], float(decay), _stream(stream)), "fbq_attention_weights")
    return out


def cache_evict_workspace(cache: Cache, weights):
    """A workspace for cache_evict() calls with weights like these."""
    import torch
    need = fbq.load().fbq_cache_evict_workspace_bytes(cache._c, weights.shape[-1])
    return torch.empty(max(16, need), dtype=torch.uint8, device=cache.pool.device)


def cache_evict(cache: Cache, weights, keep, first: int = 0, recent: int = 0, out=None, info=None, workspace=None, stream=None):
    """fbq_cache_evict: rows cut back to keep[b] tokens (int32 [rows]; -1, or as many as there are: left as it is) in every layer and head: the first `first`, the last `recent`, and of
    the others those with the largest weights.

    weights: float32 [layers, rows, kv_heads, width] (a layer's rows may be a part of more: weights[:, a:b] goes with cache.rows(a, b)); out: takes them as they are afterwards, weights
    itself by default.  info: int32 [2], rows cut back and rows skipped (see the header: what other rows hold too cannot move).
    """
    out = weights if out is None else out
    rows, layers = int(cache._c.rows), int(cache.pool.shape[0])
    stride = None
    for t, what in ((weights, "weights"), (out, "out")):
        if t.dtype != _float32 or t.dim() != 4 or tuple(t.shape[:3]) != (layers, rows, cache.heads) or (stride is not None and t.shape != weights.shape):
            raise ValueError(f"{what}: expected float32 [layers, rows, kv_heads, width] of the cache")
        if not t[0].is_contiguous() or (layers > 1 and stride is not None and t.stride(0) != stride):
            raise ValueError(f"{what}: a layer's have to lie in one piece, and out's layers as far apart as those of weights")
        stride = t.stride(0) if layers > 1 else t[0].numel()
    at, to = (_dev_ptr(t[0]) for t in (weights, out))
    if workspace is None:
        with _on(stream):
            workspace = cache_evict_workspace(cache, weights)
    _check(fbq.load().fbq_cache_evict(cache._c, at, to, stride, weights.shape[3], _ints(keep, "keep", rows), int(first), int(recent), _info(info, 2), _dev_ptr(workspace), _size(workspace),
                                      _stream(stream)), "fbq_cache_evict")
    return out
