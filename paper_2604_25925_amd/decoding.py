"""Binding of the decoding step around the verification: a paged cache of keys and values, attention over it and draws
from truncated distributions.  Argument marshalling only, as in ``binding``.

The arguments of a call travel in one C structure (``specgbv_append_args``, ``specgbv_attend_args``), packed by the standard
library's ``struct`` with the C compiler's own alignment: for calls of a few microseconds of GPU time the two dozen conversions of a
long argument list would be most of the call.
"""
from __future__ import annotations

import struct
from typing import Optional

import torch

from .binding import BF16, F32, _check, _scratch, load_library

# specgbv_paged_cache, specgbv_append_args and specgbv_attend_args of the C header, field by field
_CACHE = struct.Struct("@PPP7q8i")
_APPEND = struct.Struct("@PPPPPPPP12qqd4i")
_ATTEND = struct.Struct("@PPPP6qq5if")

_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


# The handle of a device's current stream without a Stream object around it (1.8 us of a call's 9), where this torch has it.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(device, stream: Optional[int]) -> int:
    if stream is not None:
        return stream
    return _raw_stream(device.index) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


def _between(stride: int, rows: int, length: int) -> int:
    """Entries between rows of `length`: the tensor's own, which the library looks at, but of one row, whose stride is of no matter."""
    return stride if rows > 1 else max(stride, length)


class PagedCache:
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


def specgbv_cache_append(cache: PagedCache, q, k, v, positions, *, inv_freq=None, interleaved: bool = False, q_weight=None,
                         k_weight=None, eps: float = 1e-6, out=None, stream: Optional[int] = None):
    """Enqueue the append of new tokens: heads of q [S, T, heads, D] and k [S, T, kv_heads, D] are normalised (where q_weight /
    k_weight [D] are given) and rotated by positions [S, T] * inv_freq (float64, [pairs]; entries behind 2 * pairs stay); k and v
    go to the cache.  Positions below 0 are padding.  Returns the rotated queries (`out`; q itself may be given)."""
    lib = load_library()
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
    args = _APPEND.pack(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), positions.data_ptr(),
                        inv_freq.data_ptr() if pairs else 0, q_weight.data_ptr() if q_weight is not None else 0,
                        k_weight.data_ptr() if k_weight is not None else 0, qs[0], qs[1], qs[2], ks[0], ks[1], ks[2],
                        vs[0], vs[1], vs[2], os[0], os[1], os[2], ps, eps, T, H, pairs, 1 if interleaved else 0)
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
    T, H, qs = cache._heads("q", q)
    ps = cache._positions(positions, T)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    to, _, os = cache._heads("out", out, H)
    if to != T:
        raise ValueError("out must have the shape of q")
    args = _attend_args(cache, q, qs, T, H, out.data_ptr(), os, positions.data_ptr(), ps, window, shared_len, max_len, scale)
    if workspace is None:
        need = int(lib.specgbv_attend_workspace_bytes(cache._c, args))
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=cache.device)
    else:
        _scratch(workspace, cache.device)
    _check(lib.specgbv_attend_paged(cache._c, args, workspace.data_ptr(), workspace.numel() * workspace.element_size(),
                                    _stream(cache.device, stream)))
    return out, workspace


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
