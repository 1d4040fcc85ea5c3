"""Decoding with a paged key/value cache: the C entry points of include/mopar.h on torch tensors.

Row tensors are [tokens, heads, head_dim] views whose last dimension is contiguous (slices of fused
rows included); pools are [pages, kv_heads, page_tokens, head_dim], or with a leading [layers].  Device
integers are contiguous int32 tensors.  Every call runs on ``stream``, by default the current stream
of the tensors' device; on another stream than the one that allocated them, tensors (the workspace among
them) are the caller's to keep until the work is done.  Sizes that the library cannot see (one tensor
against another) are checked here and raise ``ValueError``; the library's own refusals raise ``MoparError``.
"""
from __future__ import annotations

import ctypes

import torch

from . import _lib as L
from ._lib import check, lib

_DTYPE = {torch.float32: L.MOPAR_F32, torch.bfloat16: L.MOPAR_BF16}


def _need(ok, what):
    if not ok:
        raise ValueError(what)


def _size(n, name):
    """n as the C int that it becomes (ctypes would drop the bits past 32)."""
    if not -2 ** 31 <= n < 2 ** 31:
        raise ValueError(f"{name}: {n} does not fit 32 bits")
    return n


# torch's own lookups, without a Stream object and without asking whether the GPU is up (the tensors are on it): a norm of
# five rows takes 5.5 us on the host with them, 3.4 of them its launch, and 5.9 without
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _call(fn, device, stream, *args):
    """The entry point with the stream's handle as its last argument, the tensors' device being the current one."""
    if device.type != "cuda":
        raise ValueError("the tensors must be on a GPU")
    now = _current_device()
    index = device.index
    if index is None:
        index = now
    if stream is not None:
        _need(stream.device.index == index, "the stream is on another device than the tensors")
        handle = stream.cuda_stream
    else:
        handle = _raw_stream(index)
    if index == now:
        status = fn(*args, handle)
    else:
        with torch.cuda.device(index):
            status = fn(*args, handle)
    if status:
        check(status)


def _dtype(t):
    dt = _DTYPE.get(t.dtype)
    if dt is None:
        raise ValueError("tensors must be float32 or bfloat16")
    return dt


def _rows(t, name, like, shape=None):
    """A mopar_rows of t; `like` is the tensor whose device and dtype it shares."""
    st = t.stride()
    if len(st) != 3 or (st[2] != 1 and t.shape[2] != 1):
        raise ValueError(f"{name}: [tokens, heads, head_dim] with contiguous dims")
    if t is not like and (t.dtype != like.dtype or t.device != like.device):
        raise ValueError(f"{name}: device or dtype differs")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name}: shape must be {tuple(shape)}")
    return L.Rows(t.data_ptr(), st[0], st[1])


def _ints(t, name, like, n, dtype=torch.int32):
    if t.dtype != dtype or not t.is_contiguous() or t.device != like.device:
        raise ValueError(f"{name}: a contiguous {dtype} tensor on the same device")
    if t.numel() != n:
        raise ValueError(f"{name}: {n} entries expected")
    return t.data_ptr()


class Rotary:
    """Rotary positions (mopar_rotary_create): the angles of a descriptor, made once."""

    def __init__(self, head_dim, **kw):
        """``kw``: rot_dim, layout, base, scaling, factor, context, beta_slow, beta_fast, mscale (mopar_rotary_desc)."""
        d = L.rotary_desc(head_dim, **kw)
        h = ctypes.c_void_p()
        check(lib().mopar_rotary_create(ctypes.byref(d), ctypes.byref(h)))
        self.handle, self.head_dim = h, head_dim

    def __del__(self):
        h = getattr(self, "handle", None)
        if h is not None and h.value and L is not None and L._lib is not None:
            L._lib.mopar_rotary_destroy(h)
            self.handle = None


class PagedCache:
    """A paged cache's pools and page table (mopar_cache).  ``table`` [sequences, max_pages] int32 may be
    changed in place between calls; its entries outside the pool stand for absent pages."""

    def __init__(self, k, v, table):
        _need(k.dim() in (4, 5) and k.shape == v.shape and k.dtype == v.dtype and k.device == v.device,
              "k and v: [pages, kv_heads, page_tokens, head_dim], with a leading [layers] or not, of one shape, dtype and device")
        layer = k[0] if k.dim() == 5 else k
        _need((layer.is_contiguous() and (v[0] if v.dim() == 5 else v).is_contiguous()) and k.stride() == v.stride(),
              "k and v: a layer's pages must be contiguous")
        _need(table.dim() == 2 and table.dtype == torch.int32 and table.device == k.device and
              (table.stride(1) == 1 or table.shape[1] == 1), "table: int32 [sequences, max_pages] on the pools' device")
        _need(table.shape[0] <= 1 or table.stride(0) >= table.shape[1], "table: the rows of two sequences overlap")
        self.k, self.v, self.table = k, v, table
        self.layers = k.shape[0] if k.dim() == 5 else 1
        self.layer_stride = k.stride(0) if k.dim() == 5 else 0
        pages, heads, page, d = layer.shape
        for n, name in ((heads, "kv_heads"), (page, "page_tokens"), (d, "head_dim"), (table.shape[0], "sequences"), (table.shape[1], "max_pages")):
            _size(n, name)
        self.raw = L.Cache(_dtype(k), heads, d, page, pages, k.data_ptr(), v.data_ptr(), table.data_ptr(),
                           max(table.stride(0), table.shape[1]), table.shape[1], table.shape[0])

    def layer(self, i):
        """The cache of layer i."""
        _need(self.k.dim() == 5, "the cache has no layers")
        return PagedCache(self.k[i], self.v[i], self.table)


def _single(cache):
    _need(cache.k.dim() == 4, "one layer's cache is needed: cache.layer(i)")
    return cache


def mopar_rotary_apply(rotary, x, y, pos, stream=None):
    """y = x with every head turned to its row's position."""
    rx, ry = _rows(x, "x", x), _rows(y, "y", x, x.shape)
    t, heads, d = x.shape
    _need(d == rotary.head_dim, "x: head_dim is not the rotary's")
    p = _ints(pos, "pos", x, t)
    _call(lib().mopar_rotary_apply, x.device, stream, rotary.handle, _dtype(x), t, _size(heads, "heads"), p, rx, ry)
    return y


def mopar_cache_append(cache, k, v, seq, slot, rotary=None, pos=None, q=None, q_out=None, stream=None):
    """Key and value rows to slot slot[t] of sequence seq[t]; with a rotary, keys turned, and q to q_out."""
    c = _single(cache).raw
    t = k.shape[0]
    shape = (t, c.kv_heads, c.head_dim)
    rk, rv = _rows(k, "k", cache.k, shape), _rows(v, "v", cache.k, shape)
    rq = ro = None
    heads = 0
    if rotary is not None:
        _need(pos is not None, "pos: needed with a rotary")
        _need((q is None) == (q_out is None), "q and q_out come together")
        if q is not None:
            heads = _size(q.shape[1], "heads")
            rq, ro = _rows(q, "q", cache.k, (t, heads, c.head_dim)), _rows(q_out, "q_out", cache.k, (t, heads, c.head_dim))
    else:
        _need(pos is None and q is None and q_out is None, "pos, q and q_out go with a rotary")
    ps = None if pos is None else _ints(pos, "pos", cache.k, t)
    sq, sl = _ints(seq, "seq", cache.k, t), _ints(slot, "slot", cache.k, t)
    _call(lib().mopar_cache_append, cache.k.device, stream, c, None if rotary is None else rotary.handle, t, heads, ps, sq, sl, rq, ro,
          rk, rv)


def mopar_cache_keep(cache, lens, path_offsets, path, max_path, stream=None):
    """The accepted drafted tokens of every sequence moved to where it goes on, in every layer."""
    c = cache.raw
    ln, po = _ints(lens, "lens", cache.k, c.n_seq), _ints(path_offsets, "path_offsets", cache.k, c.n_seq + 1)
    pa = _ints(path, "path", cache.k, path.numel())
    _call(lib().mopar_cache_keep, cache.k.device, stream, c, cache.layers, cache.layer_stride, ln, po, path.numel(), pa,
          _size(max_path, "max_path"))


def _attention(q, kv_heads, scale):
    d = q.shape[2]
    return L.Attention(_dtype(q), _size(q.shape[1], "heads"), _size(kv_heads, "kv_heads"), _size(d, "head_dim"), d ** -0.5 if scale is None else scale, 0)


def mopar_attention_prompt(q, k, v, out, offsets, max_len, scale=None, stream=None):
    """Causal attention over packed prompts; sequence s is rows offsets[s] .. offsets[s + 1] - 1."""
    _need(q.dim() == 3 and k.dim() == 3, "q, k: [tokens, heads, head_dim]")
    t, d = q.shape[0], q.shape[2]
    rq, ro = _rows(q, "q", q), _rows(out, "out", q, q.shape)
    rk, rv = _rows(k, "k", q, (t, k.shape[1], d)), _rows(v, "v", q, (t, k.shape[1], d))
    off = _ints(offsets, "offsets", q, offsets.numel())
    _need(offsets.numel() >= 1, "offsets: one more than sequences")
    a = _attention(q, k.shape[1], scale)
    _call(lib().mopar_attention_prompt, q.device, stream, a, t, _size(offsets.numel() - 1, "sequences"), off, _size(max_len, "max_len"),
          rq, rk, rv, ro)
    return out


def mopar_attention_cache_workspace_bytes(q, cache, max_q, max_len):
    c = _single(cache).raw
    n = ctypes.c_size_t()
    a = _attention(q, c.kv_heads, None)
    check(lib().mopar_attention_cache_workspace_bytes(ctypes.byref(a), ctypes.byref(c), q.shape[0], _size(max_q, "max_q"),
                                                        _size(max_len, "max_len"), ctypes.byref(n)))
    return n.value


def alloc_attention_workspace(q, cache, max_q, max_len):
    """A workspace for mopar_attention_cache calls with as many rows, max_q and max_len as these, or fewer."""
    n = mopar_attention_cache_workspace_bytes(q, cache, max_q, max_len)
    return torch.empty(max(n, 16), dtype=torch.uint8, device=q.device)


def mopar_attention_cache(q, out, cache, offsets, max_q, lens, max_len, mask=None, scale=None, ws=None, stream=None):
    """Attention of drafted tokens over the cache: of a tree (``mask`` int64 [tokens, words], bit j of a row:
    it sees drafted token j) or, without a mask, of one new token or a chain of them."""
    c = _single(cache).raw
    _need(q.dim() == 3, "q: [tokens, heads, head_dim]")
    rq, ro = _rows(q, "q", cache.k), _rows(out, "out", cache.k, q.shape)
    off, ln = _ints(offsets, "offsets", cache.k, c.n_seq + 1), _ints(lens, "lens", cache.k, c.n_seq)
    words, mk = 0, None
    if mask is not None:
        _need(mask.dim() == 2, "mask: int64 [tokens, words]")
        words = mask.shape[1]
        mk = _ints(mask, "mask", cache.k, q.shape[0] * words, torch.int64)
    a = _attention(q, c.kv_heads, scale)
    if ws is not None:
        _need(ws.device == q.device and ws.is_contiguous(), "ws: a contiguous tensor on the same device")
    _call(lib().mopar_attention_cache, q.device, stream, a, c, q.shape[0], off, _size(max_q, "max_q"), ln, _size(max_len, "max_len"),
          mk, _size(words, "words"), rq, ro, None if ws is None else ws.data_ptr(), 0 if ws is None else ws.nbytes)
    return out
