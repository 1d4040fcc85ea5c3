"""A decoder's steps in 8 bits: the C entry points of include/mopar.h on torch tensors.

Rows are [tokens, width] views, float32 or bfloat16, whose last dimension is contiguous (slices of fused rows
included).  8-bit rows are a ``Rows8``.  As in ``serving``, every call runs on ``stream``, by default the
current stream of the tensors' device; sizes that the library cannot see (one tensor against another) are checked here and
raise ``ValueError``; the library's own refusals raise ``MoparError``.
"""
from __future__ import annotations

import ctypes

import torch

from . import _lib as L
from ._lib import check, lib
from .serving import _call, _dtype, _ints, _need, _size


def _matrix(t, name, like, shape=None):
    """A mopar_matrix of t; `like` is the tensor whose device and dtype it shares."""
    st = t.stride()
    if len(st) != 2 or (st[1] != 1 and t.shape[1] != 1):
        raise ValueError(f"{name}: [rows, width] with contiguous rows")
    if t is not like:
        if t.dtype != like.dtype or t.device != like.device:
            raise ValueError(f"{name}: device or dtype differs")
        if shape is not None and t.shape != shape:
            raise ValueError(f"{name}: shape must be {tuple(shape)}")
    return L.Matrix(t.data_ptr(), st[0])


def _vector(t, name, like, n, dtype=None):
    """The address of a contiguous tensor of n entries on the device of `like` (None: no tensor)."""
    if t is None:
        return None
    return _ints(t, name, like, n, like.dtype if dtype is None else dtype)


class Rows8:
    """Rows in 8 bits (mopar_rows8): ``values`` int8 [rows, width], each row at a multiple of 16 bytes and followed by
    what fills its last 16, and ``scales`` float32 [rows]."""

    def __init__(self, values, scales):
        _need(values.dim() == 2 and values.dtype == torch.int8 and (values.stride(1) == 1 or values.shape[1] == 1),
              "values: int8 [rows, width] with contiguous rows")
        rows, width = values.shape
        stride = values.stride(0)
        if rows <= 1 and stride % 16:
            stride = (width + 15) // 16 * 16
        _need(stride % 16 == 0 and values.data_ptr() % 16 == 0, "values: rows must start at multiples of 16 bytes (alloc_rows8)")
        end = values.storage_offset() + max(rows - 1, 0) * stride + (width + 15) // 16 * 16
        _need(rows == 0 or end <= values.untyped_storage().nbytes(), "values: the last row's 16 bytes are not all there (alloc_rows8)")
        _need(scales.dtype == torch.float32 and scales.is_contiguous() and scales.numel() == rows and scales.device == values.device,
              "scales: contiguous float32 [rows] on the values' device")
        self.values, self.scales = values, scales
        self.rows, self.width, self.device = rows, width, values.device
        self.raw = L.Rows8(values.data_ptr(), stride, scales.data_ptr())

    def dequantized(self):
        """What the rows stand for, float32."""
        return self.values * self.scales[:, None]


def alloc_rows8(rows, width, device):
    """8-bit rows to be written, laid out as the kernels read them: from 512 on, rows start with a cache line (products
    whose rows do not take up to 45 % longer)."""
    unit = 128 if width >= 512 else 16
    q = torch.empty(rows, (width + unit - 1) // unit * unit, dtype=torch.int8, device=device)
    return Rows8(q[:, :width], torch.empty(rows, dtype=torch.float32, device=device))


def _rows8(r, name, device, rows, width):
    if not isinstance(r, Rows8):
        raise ValueError(f"{name}: a Rows8")
    if r.device is not device and r.device != device:
        raise ValueError(f"{name}: another device")
    if r.rows != rows or r.width != width:
        raise ValueError(f"{name}: {rows} rows of {width} expected")
    return r.raw


def mopar_rms_norm(x, weight, eps=1e-6, residual=None, total=None, out=None, out8=None, stream=None):
    """Root mean square norm of x (+ residual, the sum going to total): to out, to 8-bit rows out8, or both."""
    if x.dim() != 2:
        raise ValueError("x: [tokens, width]")
    (t, w), device = x.shape, x.device
    dt = _dtype(x)
    rx = _matrix(x, "x", x)
    rr = None if residual is None else _matrix(residual, "residual", x, x.shape)
    rt = None if total is None else _matrix(total, "total", x, x.shape)
    ro = None if out is None else _matrix(out, "out", x, x.shape)
    r8 = None if out8 is None else _rows8(out8, "out8", device, t, w)
    wt = _vector(weight, "weight", x, w)
    _call(lib().mopar_rms_norm, device, stream, dt, t, _size(w, "width"), rx, rr, rt, wt, eps, ro, r8)


def mopar_quantize_rows(x, out8, gate=None, act=None, stream=None):
    """x, or with a gate act(gate) x ("silu", which is also without act, or "gelu"), as 8-bit rows out8."""
    if x.dim() != 2:
        raise ValueError("x: [tokens, width]")
    if act is None:
        act = "none" if gate is None else "silu"
    if act not in L.GATE or (gate is None) != (act == "none"):
        raise ValueError("act: silu or gelu with a gate, none without")
    (t, w), device = x.shape, x.device
    dt = _dtype(x)
    rx = _matrix(x, "x", x)
    rg = None if gate is None else _matrix(gate, "gate", x, x.shape)
    r8 = _rows8(out8, "out8", device, t, w)
    _call(lib().mopar_quantize_rows, device, stream, dt, t, _size(w, "width"), rx, rg, L.GATE[act], r8)
    return out8


def mopar_linear8_workspace_bytes(tokens, n_out, width):
    n = ctypes.c_size_t()
    check(lib().mopar_linear8_workspace_bytes(tokens, n_out, _size(width, "width"), ctypes.byref(n)))
    return n.value


def alloc_linear8_workspace(x, w, out):
    """A workspace for products of so many rows x and w of such a width, or smaller ones."""
    return torch.empty(max(mopar_linear8_workspace_bytes(x.rows, w.rows, w.width), 16), dtype=torch.uint8, device=out.device)


def _workspace(ws, device):
    if ws is None:
        return None, 0
    if ws.device != device or not ws.is_contiguous():
        raise ValueError("ws: a contiguous tensor on the same device")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def mopar_linear8(x, w, out, bias=None, ws=None, stream=None):
    """out = x w^T (+ bias) of 8-bit rows x [tokens, width] and w [n_out, width]."""
    if out.dim() != 2:
        raise ValueError("out: [tokens, n_out]")
    if not isinstance(w, Rows8):
        raise ValueError("w: a Rows8")
    dt, device, width = _dtype(out), out.device, w.width
    t, n_out = out.shape
    rx, rw = _rows8(x, "x", device, t, width), _rows8(w, "w", device, n_out, width)
    ro = _matrix(out, "out", out)
    b = None if bias is None else _vector(bias, "bias", out, n_out)
    p, n = _workspace(ws, device)
    _call(lib().mopar_linear8, device, stream, dt, t, n_out, _size(width, "width"), rx, rw, b, ro, p, n)
    return out


def mopar_token_logprobs_workspace_bytes(rows, vocab, top):
    n = ctypes.c_size_t()
    check(lib().mopar_token_logprobs_workspace_bytes(rows, _size(vocab, "vocab"), _size(top, "top"), ctypes.byref(n)))
    return n.value


def alloc_token_logprobs_workspace(logits, top=0):
    """A workspace for calls of as many rows, so large a vocabulary and so many alternatives, or fewer."""
    n = mopar_token_logprobs_workspace_bytes(logits.shape[0], logits.shape[1], top)
    return torch.empty(max(n, 16), dtype=torch.uint8, device=logits.device)


def mopar_token_logprobs(logits, tokens, logprob, entropy=None, rank=None, top_logprob=None, top_id=None, scale=1.0, ws=None, stream=None):
    """Log probabilities of ``tokens`` (int32 [rows]) under logits [rows, vocab] times ``scale``, float32; their ranks (int32), the
    entropy, and the largest alternatives in top_id (int32) and top_logprob, both [rows, top]."""
    _need(logits.dim() == 2, "logits: [rows, vocab]")
    t, v = logits.shape
    dt = _dtype(logits)
    f32, i32 = torch.float32, torch.int32
    rl = _matrix(logits, "logits", logits)
    tok = _vector(tokens, "tokens", logits, t, i32)
    lp, en = _vector(logprob, "logprob", logits, t, f32), _vector(entropy, "entropy", logits, t, f32)
    rk = _vector(rank, "rank", logits, t, i32)
    _need((top_logprob is None) == (top_id is None), "top_logprob and top_id come together")
    top = 0
    if top_id is not None:
        _need(top_id.dim() == 2 and top_id.shape[0] == t, "top_id: [rows, top]")
        _need(top_logprob.shape == top_id.shape, "top_logprob: [rows, top], as top_id")
        top = top_id.shape[1]
    tl, ti = _vector(top_logprob, "top_logprob", logits, t * top, f32), _vector(top_id, "top_id", logits, t * top, i32)
    p, n = _workspace(ws, logits.device)
    _call(lib().mopar_token_logprobs, logits.device, stream, dt, t, _size(v, "vocab"), rl, scale, tok, _size(top, "top"), lp, en, rk, tl, ti, p, n)
    return logprob
