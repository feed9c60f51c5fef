"""Binding of the decoding step around the verification: a paged cache of keys and values, attention over it, block tables, and draws
from truncated distributions.  Argument marshalling only, as in ``binding``.

A cache may also hold its entries in 4 bits (``PackedCache``), and pages can be dealt out to requests on the GPU (``PagePool``).

The arguments of a call travel in one C structure (``specgbv_append_args``, ``specgbv_attend_args``), packed by the standard
library's ``struct`` with the C compiler's own alignment: for calls of a few microseconds of GPU time the two dozen conversions of a
long argument list would be most of the call.
"""
from __future__ import annotations

import struct
from typing import Optional

import torch

from .binding import BF16, F32, _check, _scratch, load_library

# specgbv_paged_cache, specgbv_append_args, specgbv_attend_args and so on of the C header, field by field
_CACHE = struct.Struct("@PPP7q8i")
_APPEND = struct.Struct("@PPPPPPPP12qqd4i")
_ATTEND = struct.Struct("@PPPP6qq5if")
_PACKED = struct.Struct("@PPPPP13q8i")
_READ = struct.Struct("@PPP6qq2i")
_POOL = struct.Struct("@PPPPq6i")
_ADVANCE = struct.Struct("@PPPP2i")
_SLOTS = struct.Struct("@PPPPP3q8i")

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


# The handle of a device's current stream without a Stream object around it (1.8 us of a call's 9), where this torch has it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
# (and the current device without a check that CUDA is up, which tensors on it say)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _stream(device, stream: Optional[int]) -> int:
    if stream is not None:
        return stream
    return _raw_stream(device.index) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


def _between(stride: int, rows: int, length: int) -> int:
    """Entries between rows of `length`: the tensor's own, which the library looks at, but of one row, whose stride is of no matter."""
    return stride if rows > 1 else max(stride, length)


def _on(index: int, call, *args):
    """The call with the GPU `index` as the current one, which a launch on its streams needs."""
    if index < 0 or index == _current_device():
        return call(*args)
    with torch.cuda.device(index):
        return call(*args)


class _Cache:
    """What calls look at whatever a cache's entries are: sequences, head_dim, dtype and device."""

    def _heads(self, name, x, heads=None):
        """Tokens, heads and strides of x [sequences, tokens, heads, head_dim]."""
        shape = x.shape
        if len(shape) != 4 or shape[0] != self.sequences or shape[3] != self.head_dim or (heads is not None and shape[2] != heads):
            raise ValueError("%s must be [%d, tokens, %s, %d], got %s" %
                             (name, self.sequences, "heads" if heads is None else heads, self.head_dim, tuple(shape)))
        if x.dtype is not self.dtype:
            raise TypeError("%s must be %s as the cache is, got %s" % (name, self.dtype, x.dtype))
        if x.get_device() != self._index:
            raise ValueError("%s must live on the cache's GPU" % name)
        s = x.stride()
        if s[3] != 1:
            raise ValueError("the last dimension of %s must be dense" % name)
        return shape[1], shape[2], s

    def _positions(self, positions, tokens):
        shape = positions.shape
        if len(shape) != 2 or shape[0] != self.sequences or shape[1] != tokens or positions.dtype is not torch.int32 or \
                positions.get_device() != self._index:
            raise ValueError("positions must be int32 [%d, %d] on the cache's GPU" % (self.sequences, tokens))
        s = positions.stride()
        if tokens > 1 and s[1] != 1:
            raise ValueError("the last dimension of positions must be dense")
        return _between(s[0], shape[0], tokens)


class PagedCache(_Cache):
    """Keys and values in pages: k and v [pages, kv_heads, page_size, head_dim] (bfloat16 or float32, the last dimension
    dense; a page may hold its tokens before its heads: pass the transposed view) and table [sequences, width] int32: token t of sequence
    s lies in slot t % page_size of page table[s, t // page_size] (rows of the table, and of positions, may lie apart, but not overlap).
    The tensors stay the caller's: what is written to them, the table included, is what the next call sees.  A table entry outside
    [0, pages) is a page that is not there."""

    def __init__(self, k, v, table):
        if k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype:
            raise ValueError("k and v must be [pages, kv_heads, page_size, head_dim] of one dtype, got %s and %s" %
                             (tuple(k.shape), tuple(v.shape)))
        if k.dtype not in _DTYPES:
            raise TypeError("a cache holds float32 or bfloat16, got %s" % k.dtype)
        if table.dim() != 2 or table.dtype != torch.int32:
            raise ValueError("table must be int32 [sequences, width]")
        if not (k.is_cuda and v.device == k.device and table.device == k.device):
            raise ValueError("k, v and table must live on one GPU")
        if k.stride(3) != 1 or v.stride(3) != 1 or (table.shape[1] > 1 and table.stride(1) != 1):
            raise ValueError("the last dimension of k, v and table must be dense")
        self.k, self.v, self.table = k, v, table
        self.pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        self.sequences, self.width = table.shape
        self.dtype, self.device, self._index = k.dtype, k.device, k.get_device()
        ks, vs = k.stride(), v.stride()
        self._c = _CACHE.pack(k.data_ptr(), v.data_ptr(), table.data_ptr(), ks[0], ks[1], ks[2], vs[0], vs[1], vs[2],
                              _between(table.stride(0), self.sequences, self.width), self.pages, self.kv_heads, self.page_size, self.head_dim,
                              self.sequences, self.width, _DTYPES[k.dtype], 0)


def _append_args(cache, q, k, v, positions, inv_freq, interleaved, q_weight, k_weight, eps, out):
    T, H, qs = cache._heads("q", q)
    tk, _, ks = cache._heads("k", k, cache.kv_heads)
    tv, _, vs = cache._heads("v", v, cache.kv_heads)
    if tk != T or tv != T:
        raise ValueError("q, k and v must have the same tokens, got %d, %d and %d" % (T, tk, tv))
    ps = cache._positions(positions, T)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    to, _, os = cache._heads("out", out, H)
    if to != T:
        raise ValueError("out must have the shape of q")
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is not None and (w.dim() != 1 or w.shape[0] != cache.head_dim or w.dtype is not cache.dtype or
                              w.device != cache.device or not w.is_contiguous()):
            raise ValueError("%s must be dense [%d] of the cache's dtype on its GPU" % (name, cache.head_dim))
    pairs = 0
    if inv_freq is not None:
        if inv_freq.dim() != 1 or inv_freq.dtype is not torch.float64 or inv_freq.device != cache.device or not inv_freq.is_contiguous():
            raise ValueError("inv_freq must be dense float64 [pairs] on the cache's GPU")
        pairs = inv_freq.shape[0]
    return out, _APPEND.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), positions.data_ptr(),
                             inv_freq.data_ptr() if pairs else 0, q_weight.data_ptr() if q_weight is not None else 0,
                             k_weight.data_ptr() if k_weight is not None else 0, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2],
                             vs[0], vs[1], vs[2], os[0], os[1], os[2], ps, eps, T, H, pairs, 1 if interleaved else 0)


def specgbv_cache_append(cache: PagedCache, q, k, v, positions, *, inv_freq=None, interleaved: bool = False, q_weight=None,
                         k_weight=None, eps: float = 1e-6, out=None, stream: Optional[int] = None):
    """Enqueue the append of new tokens: heads of q [S, T, heads, D] and k [S, T, kv_heads, D] are normalised (where q_weight /
    k_weight [D] are given) and rotated by positions [S, T] * inv_freq (float64, [pairs]; entries behind 2 * pairs stay); k and v
    go to the cache.  Positions below 0 are padding.  Returns the rotated queries (`out`; q itself may be given)."""
    lib = load_library()
    out, args = _append_args(cache, q, k, v, positions, inv_freq, interleaved, q_weight, k_weight, eps, out)
    _check(lib.specgbv_cache_append(cache._c, args, _stream(cache.device, stream)))
    return out


def _attend_args(cache, q, qs, tokens, heads, out_ptr, os, positions_ptr, ps, window, shared_len, max_len, scale):
    prefixes = 0
    if shared_len is not None:
        if shared_len.dim() != 1 or shared_len.dtype is not torch.int32 or shared_len.device != cache.device or \
                not shared_len.is_contiguous():
            raise ValueError("shared_len must be dense int32 [prefixes] on the cache's GPU")
        prefixes = shared_len.shape[0]
        if prefixes == 0 and cache.sequences:
            raise ValueError("%d sequences are not drafts of 0 prefixes" % cache.sequences)
    return _ATTEND.pack(q.data_ptr(), out_ptr, positions_ptr, shared_len.data_ptr() if prefixes else 0,
                        qs[0], qs[1], qs[2], os[0], os[1], os[2], ps, tokens, heads, window, prefixes, max_len or 0, scale or 0.0)


def _attend_call(cache, q, positions, window, shared_len, max_len, scale, out):
    T, H, qs = cache._heads("q", q)
    ps = cache._positions(positions, T)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    to, _, os = cache._heads("out", out, H)
    if to != T:
        raise ValueError("out must have the shape of q")
    return out, _attend_args(cache, q, qs, T, H, out.data_ptr(), os, positions.data_ptr(), ps, window, shared_len, max_len, scale)


def _attend_workspace(cache, args, workspace, need):
    if workspace is None:
        return torch.empty(max(int(need(cache._c, args)), 256), dtype=torch.uint8, device=cache.device)
    return _scratch(workspace, cache.device)


def specgbv_attend_workspace_bytes(cache: PagedCache, q, *, window: int = 0, shared_len=None, max_len: Optional[int] = None) -> int:
    T, H, qs = cache._heads("q", q)
    return int(load_library().specgbv_attend_workspace_bytes(
        cache._c, _attend_args(cache, q, qs, T, H, 0, (0, 0, 0), 0, T, window, shared_len, max_len, None)))


def specgbv_attend_paged(cache: PagedCache, q, positions, *, window: int = 0, shared_len=None, max_len: Optional[int] = None,
                         scale: Optional[float] = None, out=None, workspace=None, stream: Optional[int] = None):
    """Enqueue the attention of queries q [S, T, heads, D] at positions [S, T] (int32, below 0: padding, whose output is 0) over the
    cache: the query at position p sees tokens p - window < j <= p of its sequence (window 0: all up to p).  shared_len [prefixes]
    int32 states that the S sequences are the drafts of as many prefixes and how many first tokens lie in pages that a prefix's drafts
    share: those are read once per prefix.  max_len: how far sequences reach at most, for the choice of the split.  Returns
    (out [S, T, heads, D], workspace); the workspace serves calls of these shapes with any max_len."""
    lib = load_library()
    out, args = _attend_call(cache, q, positions, window, shared_len, max_len, scale, out)
    workspace = _attend_workspace(cache, args, workspace, lib.specgbv_attend_workspace_bytes)
    _check(lib.specgbv_attend_paged(cache._c, args, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                    _stream(cache.device, stream)))
    return out, workspace


class PackedCache(_Cache):
    """Keys and values in pages, each entry held in 4 bits: k and v uint8 [pages, kv_heads, page_size, head_dim / 2] (the last dimension dense; a page
    may hold its tokens before its heads) and the powers of two of 32 adjacent entries, k_scale and v_scale uint8 [pages, kv_heads,
    head_dim / 32, page_size] (the last dimension dense); head_dim is a multiple of 32.  table as in PagedCache.  dtype: that of the queries,
    keys, values and results of the calls (bfloat16 or float32)."""

    def __init__(self, k, v, k_scale, v_scale, table, dtype=torch.bfloat16):
        if k.dim() != 4 or k.shape != v.shape:
            raise ValueError("k and v must be [pages, kv_heads, page_size, head_dim / 2], got %s and %s" % (tuple(k.shape), tuple(v.shape)))
        for x in (k, v, k_scale, v_scale):
            if x.dtype is not torch.uint8:
                raise TypeError("a packed cache is uint8, got %s" % x.dtype)
        if dtype not in _DTYPES:
            raise TypeError("queries are float32 or bfloat16, got %s" % dtype)
        pages, kv_heads, page_size, half = k.shape
        if half % 16:
            raise ValueError("head_dim=%d is not a multiple of 32" % (2 * half))
        blocks = (pages, kv_heads, half // 16, page_size)
        if k_scale.shape != blocks or v_scale.shape != blocks:
            raise ValueError("k_scale and v_scale must be %s, got %s and %s" % (blocks, tuple(k_scale.shape), tuple(v_scale.shape)))
        if table.dim() != 2 or table.dtype != torch.int32:
            raise ValueError("table must be int32 [sequences, width]")
        if not k.is_cuda or any(x.device != k.device for x in (v, k_scale, v_scale, table)):
            raise ValueError("k, v, their scales and table must live on one GPU")
        if any(x.stride(3) != 1 for x in (k, v, k_scale, v_scale)) or (table.shape[1] > 1 and table.stride(1) != 1):
            raise ValueError("the last dimension of k, v, their scales and table must be dense")
        self.k, self.v, self.k_scale, self.v_scale, self.table = k, v, k_scale, v_scale, table
        self.pages, self.kv_heads, self.page_size, self.head_dim = pages, kv_heads, page_size, 2 * half
        self.sequences, self.width = table.shape
        self.dtype, self.device, self._index = dtype, k.device, k.get_device()
        # (the stride of a dimension of one is of no matter)
        strides = [s if n > 1 else 0 for x in (k, v, k_scale, v_scale) for n, s in zip(x.shape[:3], x.stride()[:3])]
        self._c = _PACKED.pack(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), table.data_ptr(), *strides, _between(table.stride(0), self.sequences, self.width),
                               pages, kv_heads, page_size, self.head_dim, self.sequences, self.width, _DTYPES[dtype], 0)

    @classmethod
    def empty(cls, pages, kv_heads, page_size, head_dim, table, dtype=torch.bfloat16):
        """A cache of new memory, all of it zero, beside a table."""
        if head_dim % 32:
            raise ValueError("head_dim=%d is not a multiple of 32" % head_dim)
        k, v = (torch.zeros((pages, kv_heads, page_size, head_dim // 2), dtype=torch.uint8, device=table.device) for _ in range(2))
        ks, vs = (torch.zeros((pages, kv_heads, head_dim // 32, page_size), dtype=torch.uint8, device=table.device) for _ in range(2))
        return cls(k, v, ks, vs, table, dtype)


def specgbv_packed_append(cache: PackedCache, q, k, v, positions, *, inv_freq=None, interleaved: bool = False, q_weight=None,
                          k_weight=None, eps: float = 1e-6, out=None, stream: Optional[int] = None):
    """specgbv_cache_append to a cache that holds its entries in 4 bits: keys are normalised and rotated in float64 before they are
    rounded.  Returns the rotated queries."""
    lib = load_library()
    out, args = _append_args(cache, q, k, v, positions, inv_freq, interleaved, q_weight, k_weight, eps, out)
    _check(_on(cache._index, lib.specgbv_packed_append, cache._c, args, _stream(cache.device, stream)))
    return out


def specgbv_packed_read(cache: PackedCache, positions, *, k=None, v=None, stream: Optional[int] = None):
    """Enqueue the reading of tokens' keys and values as the cache holds them: (k, v), each [S, T, kv_heads, D] of the cache's dtype, for
    positions [S, T]; 0 where there is no token (position below 0, behind the table's width, no page)."""
    lib = load_library()
    if positions.dim() != 2:
        raise ValueError("positions must be int32 [sequences, tokens]")
    T = positions.shape[1]
    ps = cache._positions(positions, T)
    shape = (cache.sequences, T, cache.kv_heads, cache.head_dim)
    strides = []
    made = []
    for name, x in (("k", k), ("v", v)):
        if x is None:
            x = torch.empty(shape, dtype=cache.dtype, device=positions.device)
        t, _, s = cache._heads(name, x, cache.kv_heads)
        if t != T:
            raise ValueError("%s must have the tokens of positions, %d, got %d" % (name, T, t))
        made.append(x)
        strides += s[:3]
    args = _READ.pack(made[0].data_ptr(), made[1].data_ptr(), positions.data_ptr(), *strides, ps, T, 0)
    _check(_on(cache._index, lib.specgbv_packed_read, cache._c, args, _stream(cache.device, stream)))
    return made[0], made[1]


def specgbv_packed_attend_workspace_bytes(cache: PackedCache, q, *, window: int = 0, shared_len=None, max_len: Optional[int] = None) -> int:
    T, H, qs = cache._heads("q", q)
    args = _attend_args(cache, q, qs, T, H, 0, (0, 0, 0), 0, T, window, shared_len, max_len, None)
    return int(_on(cache._index, load_library().specgbv_packed_attend_workspace_bytes, cache._c, args))


def specgbv_packed_attend(cache: PackedCache, q, positions, *, window: int = 0, shared_len=None, max_len: Optional[int] = None,
                          scale: Optional[float] = None, out=None, workspace=None, stream: Optional[int] = None):
    """specgbv_attend_paged over a cache that holds its entries in 4 bits, with the same arguments and results."""
    lib = load_library()
    out, args = _attend_call(cache, q, positions, window, shared_len, max_len, scale, out)
    workspace = _attend_workspace(cache, args, workspace, lambda *a: _on(cache._index, lib.specgbv_packed_attend_workspace_bytes, *a))
    _check(_on(cache._index, lib.specgbv_packed_attend, cache._c, args, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
               _stream(cache.device, stream)))
    return out, workspace


class PagePool:
    """Pages dealt out on the GPU to requests, each a prefix with `drafts` sequences.  table int32 [prefixes * drafts, width] (-1 where a
    sequence has no page; pass it to a cache); held int32 [prefixes, 2]: how many first pages a request's drafts share, and how many each
    draft has in all; ring int32 [pages] and ends int32 [2] (head, count): the free pages are ring[(head + i) % pages] for i < count.
    The tensors stay the caller's.  ``empty`` makes them for a batch without requests."""

    def __init__(self, table, ring, ends, held, *, drafts: int = 1, page_size: int):
        for name, x, dim in (("table", table, 2), ("ring", ring, 1), ("ends", ends, 1), ("held", held, 2)):
            if x.dim() != dim or x.dtype is not torch.int32:
                raise ValueError("%s must be int32 with %d dimensions" % (name, dim))
        if not table.is_cuda or any(x.device != table.device for x in (ring, ends, held)):
            raise ValueError("table, ring, ends and held must live on one GPU")
        if not all(x.is_contiguous() for x in (ring, ends, held)) or (table.shape[1] > 1 and table.stride(1) != 1):
            raise ValueError("ring, ends and held must be dense, and so must the rows of table")
        if drafts < 1 or table.shape[0] % drafts:
            raise ValueError("%d sequences are not prefixes of %d drafts" % (table.shape[0], drafts))
        if ends.shape[0] != 2 or tuple(held.shape) != (table.shape[0] // drafts, 2):
            raise ValueError("ends must be [2] and held [%d, 2], got %s and %s" % (table.shape[0] // drafts, tuple(ends.shape), tuple(held.shape)))
        self.table, self.ring, self.ends, self.held = table, ring, ends, held
        self.drafts, self.page_size, self.pages, self.prefixes, self.width = drafts, page_size, ring.shape[0], table.shape[0] // drafts, table.shape[1]
        self.device, self._index = table.device, table.get_device()
        self._c = _POOL.pack(table.data_ptr(), ring.data_ptr(), ends.data_ptr(), held.data_ptr(), _between(table.stride(0), table.shape[0], self.width),
                             self.pages, page_size, self.prefixes, drafts, self.width, 0)

    @classmethod
    def empty(cls, prefixes, width, pages, *, page_size: int, drafts: int = 1, device="cuda"):
        """A pool of all `pages`, none of them dealt out."""
        table = torch.full((prefixes * drafts, width), -1, dtype=torch.int32, device=device)
        ring = torch.arange(pages, dtype=torch.int32, device=device)
        ends = torch.tensor([0, pages], dtype=torch.int32, device=device)
        return cls(table, ring, ends, torch.zeros((prefixes, 2), dtype=torch.int32, device=device), drafts=drafts, page_size=page_size)


def _numbers(name, x, shape, index, dtype=torch.int32):
    if x.shape != shape or x.dtype is not dtype or x.get_device() != index or not x.is_contiguous():
        raise ValueError("%s must be dense %s %s on the call's GPU" % (name, dtype, list(shape)))
    return x


def specgbv_pages_workspace_bytes(pool: PagePool) -> int:
    return int(load_library().specgbv_pages_workspace_bytes(pool._c))


def specgbv_pages_advance(pool: PagePool, length, *, chosen=None, room: int = 0, shared_len=None, served=None, workspace=None,
                          stream: Optional[int] = None):
    """Enqueue the bringing of every request's pages to its length: length [prefixes] int32 tokens stay (0 and below: the request has ended)
    and `room` more may be written by the next step; chosen [prefixes] int32 (as the verification returns it): the draft whose pages the
    prefix's drafts share from here on.  Requests that need more pages than they give back are served in their order while there are enough; one that is
    not served keeps what it has, and is given the same `chosen` again.  Tokens behind shared_len that stay are in the chosen draft's own page alone: append them again for
    every draft.  Returns (shared_len [prefixes], tokens in shared pages; served [prefixes]: 1, 0: too few pages, -1:
    longer than the table; workspace)."""
    lib = load_library()
    shape = (pool.prefixes,)
    _numbers("length", length, shape, pool._index)
    if chosen is not None:
        _numbers("chosen", chosen, shape, pool._index)
    shared_len = length.new_empty(shape) if shared_len is None else _numbers("shared_len", shared_len, shape, pool._index)
    served = length.new_empty(shape) if served is None else _numbers("served", served, shape, pool._index)
    if workspace is None:
        workspace = torch.empty(max(int(lib.specgbv_pages_workspace_bytes(pool._c)), 256), dtype=torch.uint8, device=pool.device)
    else:
        _scratch(workspace, pool.device)
    args = _ADVANCE.pack(length.data_ptr(), chosen.data_ptr() if chosen is not None else 0, shared_len.data_ptr(), served.data_ptr(), room, 0)
    _check(_on(pool._index, lib.specgbv_pages_advance, pool._c, args, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
               _stream(pool.device, stream)))
    return shared_len, served, workspace


def _rows(name, x, table, rows, length, dtype):
    """(x, entries between its rows): int [rows, length] beside a table, new where x is None."""
    if x is None:
        return table.new_empty((rows, length), dtype=dtype), length
    if x.shape != (rows, length) or x.dtype is not dtype or x.get_device() != table.get_device() or (length > 1 and x.stride(1) != 1):
        raise ValueError("%s must be %s [%d, %d] on the table's GPU, its rows dense" % (name, dtype, rows, length))
    return x, _between(x.stride(0), rows, length)


def specgbv_slot_map(table, start, count, tokens: int, *, page_size: int, pages: int, drafts: int = 1, right: bool = False, flat: bool = True,
                     positions=None, slots=None, stream: Optional[int] = None):
    """Enqueue where new tokens lie: each of a prefix's `drafts` sequences has count [prefixes] tokens (int32, at most `tokens`) from position
    start [prefixes] on.  Returns (positions [S, tokens] int32, -1 where there is no token, slots [S, tokens] int64: page * page_size + slot of the
    token's place, -1: none; None where `flat` is false).  right: the tokens stand in a row's last places instead of its first ones."""
    lib = load_library()
    if table.dim() != 2 or table.dtype is not torch.int32 or not table.is_cuda or (table.shape[1] > 1 and table.stride(1) != 1):
        raise ValueError("table must be int32 [sequences, width] on the GPU, its rows dense")
    S, index = table.shape[0], table.get_device()
    if drafts < 1 or S % drafts:
        raise ValueError("%d sequences are not prefixes of %d drafts" % (S, drafts))
    if tokens < 0:
        raise ValueError("tokens must be >= 0, got %d" % tokens)
    _numbers("start", start, (S // drafts,), index)
    _numbers("count", count, (S // drafts,), index)
    positions, positions_stride = _rows("positions", positions, table, S, tokens, torch.int32)
    slots, slots_stride = _rows("slots", slots, table, S, tokens, torch.int64) if flat else (None, tokens)
    args = _SLOTS.pack(table.data_ptr(), start.data_ptr(), count.data_ptr(), positions.data_ptr(), slots.data_ptr() if flat else 0,
                       _between(table.stride(0), S, table.shape[1]), positions_stride, slots_stride, S, drafts, table.shape[1], page_size, pages, tokens,
                       1 if right else 0, 0)
    _check(_on(index, lib.specgbv_slot_map, args, _stream(table.device, stream)))
    return positions, slots


def specgbv_filter_workspace_bytes(rows: int, V: int, dtype: int) -> int:
    return int(load_library().specgbv_filter_workspace_bytes(rows, V, dtype))


def _rows_of(name, x, V=None):
    """(rows, stride between rows) of x [..., V] whose leading dimensions step evenly."""
    if 0 in x.shape[:-1]:
        return 0, x.shape[-1]
    if x.dim() == 2:
        rows, stride = x.shape[0], x.stride(0)
    else:
        rows, stride = 1, x.shape[-1]
        for n, s in zip(reversed(x.shape[:-1]), reversed(x.stride()[:-1])):
            if n == 1:
                continue
            if rows == 1:
                stride = s
            elif s != rows * stride:
                raise ValueError("the rows of %s must step evenly" % name)
            rows *= n
    if x.shape[-1] > 1 and x.stride(-1) != 1:
        raise ValueError("the last dimension of %s must be dense" % name)
    return rows, max(stride, x.shape[-1]) if rows < 2 else stride


def specgbv_sample_filtered(logits, u=None, *, temperature=None, top_k=None, top_p=None, min_p=None, draw: bool = True,
                            keep: bool = False, out=None, kept=None, workspace=None, stream: Optional[int] = None):
    """Enqueue, per row of logits [rows, V] (or [..., V]), the truncation by top_k, min_p and top_p and (draw) the token that
    the uniform u [rows] selects from what is kept; the order of entries is by logit, the largest first, ties by the lowest index.  temperature,
    top_p, min_p and u are float32 [rows] tensors, top_k int32 [rows], each optional (1, off, off; 0: off).  Returns (tokens [rows] int32
    or None, kept or None, workspace); kept (keep): the logits with -inf where an entry is dropped, `kept` may be logits itself."""
    lib = load_library()
    if logits.dtype not in _DTYPES:
        raise TypeError("logits must be float32 or bfloat16, got %s" % logits.dtype)
    if not logits.is_cuda or logits.dim() < 2:
        raise ValueError("logits must be a GPU tensor [rows, V]")
    dev, V = logits.device, logits.shape[-1]
    rows, row_stride = _rows_of("logits", logits)
    if not draw and not keep:
        raise ValueError("nothing is asked for: draw and keep are both false")
    if draw and u is None:
        raise ValueError("a draw needs u")
    ptr = []
    for name, x, dtype in (("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32),
                           ("min_p", min_p, torch.float32), ("u", u if draw else None, torch.float32)):
        if x is None:
            ptr.append(None)
            continue
        if x.dtype is not dtype or x.numel() != rows or x.device != dev or not x.is_contiguous():
            raise ValueError("%s must be dense %s [%d] on the logits' GPU" % (name, dtype, rows))
        ptr.append(x.data_ptr())
    if not draw:
        out = None
    elif out is None:
        out = torch.empty(rows, dtype=torch.int32, device=dev)
    elif out.dtype is not torch.int32 or out.numel() != rows or out.device != dev or not out.is_contiguous():
        raise ValueError("out must be dense int32 [%d] on the logits' GPU" % rows)
    kept_stride = V
    if not keep:
        kept = None
    else:
        if kept is None:
            kept = torch.empty(logits.shape, dtype=logits.dtype, device=dev)
        elif kept.shape != logits.shape or kept.dtype is not logits.dtype or kept.device != dev:
            raise ValueError("kept must have the shape, dtype and GPU of logits")
        kept_stride = _rows_of("kept", kept)[1]
    dt = _DTYPES[logits.dtype]
    if workspace is None:
        workspace = torch.empty(max(int(lib.specgbv_filter_workspace_bytes(rows, V, dt)), 256), dtype=torch.uint8, device=dev)
    else:
        _scratch(workspace, dev)
    _check(lib.specgbv_sample_filtered(logits.data_ptr(), row_stride, rows, V, dt, ptr[0], ptr[1], ptr[2], ptr[3], ptr[4],
                                       out.data_ptr() if draw else None, kept.data_ptr() if keep else None, kept_stride,
                                       workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream(dev, stream)))
    return out, kept, workspace
