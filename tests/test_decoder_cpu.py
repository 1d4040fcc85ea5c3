"""Host checks of a decoder's steps in 8 bits: what is refused (before any device call), and workspace sizes."""
import ctypes
import os

import pytest
import torch

import paper_2404_02445_amd as P
from paper_2404_02445_amd import _lib as L
from tests import test_inline_reads as inline

A = 0x10000          # an aligned address that no accepted call ever sees
E, U, D, W = L.MOPAR_E_ARG, L.MOPAR_E_UNSUPPORTED, L.MOPAR_E_DTYPE, L.MOPAR_E_WORKSPACE


def status(fn, *args):
    st = getattr(P.lib(), fn)(*args)
    if st != 0:
        assert P.lib().mopar_last_error()
    return st


def mat(data=A, stride=512):
    return L.Matrix(data, stride)


def rows8(q=A, stride=512, scale=A):
    return L.Rows8(q, stride, scale)


def ref(x):
    return None if x is None else ctypes.byref(x)


def norm_status(dtype=L.MOPAR_BF16, tokens=4, width=500, x=mat(), residual=None, total=None, weight=A, eps=1e-5, out=mat(), out8=None):
    return status("mopar_rms_norm", dtype, tokens, width, ref(x), ref(residual), ref(total), weight, eps, ref(out), ref(out8), None)


def test_norm_refusals():
    assert norm_status(tokens=0) == 0 and norm_status(tokens=0, x=None, weight=None) == 0
    assert norm_status(dtype=L.MOPAR_I32) == D
    r = mat()
    for kw in (dict(tokens=-1), dict(width=0), dict(width=-1), dict(width=(1 << 24) + 1), dict(x=None), dict(x=mat(None)), dict(x=mat(A + 1)),
               dict(x=mat(A, -1)), dict(weight=None), dict(weight=A + 1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
               dict(out=None), dict(out=mat(A, 499)), dict(out=mat(A + 1)), dict(total=mat(A + 2)), dict(residual=mat(A + 1)),
               dict(residual=r, total=mat(A + 2, 499)), dict(residual=r, total=mat()), dict(out8=rows8(None)), dict(out8=rows8(A + 8)),
               dict(out8=rows8(A, 504)), dict(out8=rows8(A, -16)), dict(out8=rows8(A, 496)), dict(out8=rows8(scale=None)), dict(out8=rows8(scale=A + 2)),
               dict(dtype=L.MOPAR_F32, x=mat(A + 2))):
        assert norm_status(**kw) == E, kw
    for kw in (dict(tokens=1 << 31), dict(x=mat(A, 1 << 45)), dict(out=mat(A, 1 << 45)), dict(out8=rows8(A, 1 << 23))):
        assert norm_status(**kw) == U, kw


def quant_status(dtype=L.MOPAR_BF16, tokens=4, width=500, x=mat(), gate=None, act=0, out8=rows8()):
    return status("mopar_quantize_rows", dtype, tokens, width, ref(x), ref(gate), act, ref(out8), None)


def test_quantize_refusals():
    assert quant_status(tokens=0) == 0 and quant_status(dtype=5) == D
    for kw in (dict(tokens=-1), dict(width=0), dict(x=None), dict(x=mat(A + 1)), dict(act=1), dict(act=-1, gate=mat()), dict(act=3, gate=mat()), dict(gate=mat()),
               dict(act=1, gate=mat(A + 1)), dict(act=2, gate=mat(None)), dict(out8=None), dict(out8=rows8(A, 496)), dict(out8=rows8(scale=None))):
        assert quant_status(**kw) == E, kw
    assert quant_status(tokens=1 << 31) == U and quant_status(gate=mat(A, 1 << 45), act=1) == U


def linear_status(dtype=L.MOPAR_BF16, tokens=4, n=300, width=500, x=rows8(), w=rows8(), bias=None, out=mat(), ws=None, ws_n=0):
    return status("mopar_linear8", dtype, tokens, n, width, ref(x), ref(w), bias, ref(out), ws, ws_n, None)


def linear_ws(tokens, n, width):
    b = ctypes.c_size_t()
    return status("mopar_linear8_workspace_bytes", tokens, n, width, ctypes.byref(b)), b.value


def test_linear_refusals():
    assert linear_status(tokens=0) == 0 and linear_status(n=0) == 0 and linear_status(dtype=2) == D
    for kw in (dict(tokens=-1), dict(n=-1), dict(width=0), dict(x=None), dict(w=None), dict(out=None), dict(x=rows8(A + 8)), dict(w=rows8(A, 500)),
               dict(x=rows8(scale=None)), dict(w=rows8(scale=A + 1)), dict(bias=A + 1), dict(out=mat(A, 299)), dict(out=mat(None)), dict(ws=A + 8, ws_n=1 << 30)):
        assert linear_status(**kw) == E, kw
    for kw in (dict(width=1 << 17), dict(tokens=1 << 31), dict(n=1 << 31), dict(tokens=1 << 18, n=1 << 18), dict(x=rows8(A, 1 << 23)), dict(out=mat(A, 1 << 45))):
        assert linear_status(**kw) == U, kw
    st, need = linear_ws(64, 4096, 14336)
    assert st == 0 and need > 0 and linear_status(tokens=64, n=4096, width=14336, out=mat(A, 4096), ws=A, ws_n=need - 1) == W
    assert linear_ws(64, 4096, 128) == (0, 0) and linear_ws(0, 5, 999) == (0, 0)
    assert status("mopar_linear8_workspace_bytes", 1, 1, 1, None) == E


def test_a_linear_workspace_holds_smaller_calls():
    ms, ns, ks = (1, 16, 17, 64, 65, 300, 5000), (1, 31, 64, 500, 4096, 30000), (1, 128, 129, 1000, 5000, 131071)
    size = {(i, j, l): linear_ws(m, n, k)[1] for i, m in enumerate(ms) for j, n in enumerate(ns) for l, k in enumerate(ks)}
    for (i, j, l), v in size.items():
        for up in ((i + 1, j, l), (i, j + 1, l), (i, j, l + 1)):
            assert v <= size.get(up, v)


def lp_status(dtype=L.MOPAR_BF16, rows=4, vocab=500, logits=mat(), scale=1.0, token=A, top=0, lp=A, en=A, rank=A, tl=None, ti=None, ws=None, n=0):
    return status("mopar_token_logprobs", dtype, rows, vocab, ref(logits), scale, token, top, lp, en, rank, tl, ti, ws, n, None)


def lp_ws(rows, vocab, top):
    b = ctypes.c_size_t()
    return status("mopar_token_logprobs_workspace_bytes", rows, vocab, top, ctypes.byref(b)), b.value


def test_logprobs_refusals():
    assert lp_status(rows=0) == 0 and lp_status(dtype=2) == D
    for kw in (dict(rows=-1), dict(vocab=0), dict(top=-1), dict(top=65, tl=A, ti=A), dict(vocab=9, top=10, tl=A, ti=A), dict(logits=None), dict(logits=mat(A + 1)),
               dict(logits=mat(A, -5)), dict(token=None), dict(token=A + 2), dict(lp=None), dict(en=A + 1), dict(rank=A + 2), dict(top=3), dict(top=3, tl=A),
               dict(top=3, ti=A), dict(top=3, tl=A + 1, ti=A), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(scale=3e38), dict(ws=A + 4, n=1 << 30)):
        assert lp_status(**kw) == E, kw
    for kw in (dict(rows=1 << 24), dict(vocab=1 << 28), dict(logits=mat(A, 1 << 45))):
        assert lp_status(**kw) == U, kw
    st, need = lp_ws(4, 128000, 20)
    assert st == 0 and need > 0 and lp_status(vocab=128000, top=20, tl=A, ti=A, ws=A, n=need - 1) == W
    assert status("mopar_token_logprobs_workspace_bytes", 1, 1, 1, None) == E


def test_a_logprobs_workspace_holds_smaller_calls():
    rs, vs, ts = (1, 3, 31, 32, 33, 500, 1024, 5000), (64, 4096, 8192, 50000, 128000, 1 << 20), (0, 1, 20, 64)
    size = {(i, j, l): lp_ws(r, v, t)[1] for i, r in enumerate(rs) for j, v in enumerate(vs) for l, t in enumerate(ts)}
    for (i, j, l), v in size.items():
        for up in ((i + 1, j, l), (i, j + 1, l), (i, j, l + 1)):
            assert v <= size.get(up, v)


def test_binding_refuses_mismatched_tensors():
    bf = torch.bfloat16
    x, w = torch.zeros(3, 40, dtype=bf), torch.zeros(40, dtype=bf)
    q = P.alloc_rows8(3, 40, "cpu")
    i3, f3 = torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    bad = [lambda: P.mopar_rms_norm(x, w, out=x),                                                                  # on the CPU
           lambda: P.mopar_rms_norm(x, w[:39], out=x), lambda: P.mopar_rms_norm(x, w.float(), out=x), lambda: P.mopar_rms_norm(x.half(), w.half(), out=x.half()),
           lambda: P.mopar_rms_norm(x, w, out=x[:2]), lambda: P.mopar_rms_norm(x, w, out=x.float()), lambda: P.mopar_rms_norm(x.t(), w[:3], out=x.t()),
           lambda: P.mopar_rms_norm(x, w, residual=x[:, :39], out=x), lambda: P.mopar_rms_norm(x, w, out8=P.alloc_rows8(3, 41, "cpu")),
           lambda: P.mopar_rms_norm(x, w, out8=x), lambda: P.mopar_rms_norm(x[0], w, out=x[0]),
           lambda: P.mopar_quantize_rows(x, q, gate=x[:2]), lambda: P.mopar_quantize_rows(x, q, gate=x, act="none"), lambda: P.mopar_quantize_rows(x, q, gate=x, act="relu"),
           lambda: P.mopar_quantize_rows(x, P.alloc_rows8(2, 40, "cpu")),
           lambda: P.mopar_linear8(q, P.alloc_rows8(5, 41, "cpu"), torch.zeros(3, 5)), lambda: P.mopar_linear8(q, q, torch.zeros(3, 5)),
           lambda: P.mopar_linear8(q, q, torch.zeros(2, 3)), lambda: P.mopar_linear8(q, q, torch.zeros(3, 3).half()), lambda: P.mopar_linear8(x, q, torch.zeros(3, 3)),
           lambda: P.mopar_linear8(q, q, torch.zeros(3, 3), bias=torch.zeros(3, dtype=bf)), lambda: P.mopar_linear8(q, q, torch.zeros(3, 6)[:, ::2]),
           lambda: P.mopar_token_logprobs(x, i3[:2], f3), lambda: P.mopar_token_logprobs(x, i3.long(), f3), lambda: P.mopar_token_logprobs(x, i3, f3.double()),
           lambda: P.mopar_token_logprobs(x, i3, f3, top_id=torch.zeros(3, 2, dtype=torch.int32)), lambda: P.mopar_token_logprobs(x, i3, f3, rank=f3),
           lambda: P.mopar_token_logprobs(x, i3, f3, top_id=torch.zeros(2, 2, dtype=torch.int32), top_logprob=torch.zeros(2, 2)),
           lambda: P.Rows8(torch.zeros(3, 40, dtype=torch.int8), f3), lambda: P.Rows8(torch.zeros(3, 48), f3), lambda: P.Rows8(q.values, f3[:2]),
           lambda: P.Rows8(q.values, f3.double()), lambda: P.Rows8(torch.zeros(3, 48, dtype=torch.int8)[:, 1:41], f3),
           lambda: P.Rows8(torch.zeros(2 * 48 + 40, dtype=torch.int8).as_strided((3, 40), (48, 1)), f3)]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print("accepted:", i)


def test_binding_refuses_sizes_past_32_bits():
    for n in (1 << 31, 1 << 32, (1 << 32) + 5, -(1 << 32)):
        for f in (lambda: P.mopar_linear8_workspace_bytes(1, 1, n), lambda: P.mopar_token_logprobs_workspace_bytes(1, n, 0),
                  lambda: P.mopar_token_logprobs_workspace_bytes(1, 100, n)):
            with pytest.raises(ValueError):
                f()


def test_rows8_layout():
    q = P.alloc_rows8(5, 33, "cpu")
    assert q.values.shape == (5, 33) and q.values.stride() == (48, 1) and q.raw.stride == 48 and q.scales.shape == (5,)
    one = P.Rows8(torch.zeros(16, dtype=torch.int8)[None, :9], torch.zeros(1))
    assert one.raw.stride == 16 and P.alloc_rows8(0, 7, "cpu").rows == 0


@pytest.mark.parametrize("name", ["rows8.hip", "linear8.hip", "logprobs.hip"])
def test_no_read_outlives_its_asm(name):
    with open(os.path.join(inline.CSRC, name)) as f:
        assert inline.faults(f.read()) == []
