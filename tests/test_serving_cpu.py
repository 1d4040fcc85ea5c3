"""Host checks of decoding with a paged cache: what is refused (before any device call), workspace sizes, and the
rotary's angles."""
import ctypes
import math
import os
import re
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2404_02445_amd as P
from tests.helpers import host_rule
from paper_2404_02445_amd import _lib as L

A = 0x10000          # an aligned address that no accepted call ever sees


def status(fn, *args):
    st = getattr(P.lib(), fn)(*args)
    if st != 0:
        assert P.lib().mopar_last_error()
    return st


def rows(data=A, ts=1024, hs=128):
    return L.Rows(data, ts, hs)


def cache(**kw):
    c = L.Cache(L.MOPAR_BF16, 2, 128, 16, 100, A, A, A, 8, 8, 3)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def attention(**kw):
    a = L.Attention(L.MOPAR_BF16, 8, 2, 128, 0.1, 0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def rotary(**kw):
    d = dict(head_dim=128)
    d.update(kw)
    return P.Rotary(**d)


@pytest.mark.parametrize("kw", [dict(head_dim=0), dict(head_dim=258), dict(rot_dim=3), dict(rot_dim=0), dict(rot_dim=130),
                                dict(base=0.5), dict(base=float("nan")), dict(base=float("inf")), dict(scaling="linear", factor=0.5),
                                dict(scaling="ntk", factor=float("nan")), dict(scaling="ntk", rot_dim=2, factor=2.0),
                                dict(scaling="yarn", factor=2.0), dict(scaling="yarn", factor=2.0, context=-1.0), dict(mscale=-1.0),
                                dict(scaling="yarn", factor=2.0, context=100.0, beta_slow=3.0, beta_fast=2.0)])
def test_rotary_refusals(kw):
    with pytest.raises(P.MoparError) as e:
        rotary(**kw)
    assert e.value.status == L.MOPAR_E_ARG


def test_rotary_create_null():
    h = ctypes.c_void_p(1)
    assert status("mopar_rotary_create", None, ctypes.byref(h)) == L.MOPAR_E_ARG and not h.value
    d = L.RotaryDesc(0, 9, 64, 64, 1e4, 1, 0, 0, 0, 0)
    assert status("mopar_rotary_create", ctypes.byref(d), ctypes.byref(h)) == L.MOPAR_E_ARG
    assert status("mopar_rotary_create", ctypes.byref(d), None) == L.MOPAR_E_ARG


class Table(ctypes.Structure):
    _fields_ = [("w", ctypes.c_uint64 * 128), ("m", ctypes.c_float), ("d", ctypes.c_int), ("rot", ctypes.c_int), ("inter", ctypes.c_int)]


@pytest.mark.parametrize("scaling,kw", [(0, {}), (1, dict(factor=3.0)), (2, dict(factor=8.0)), (3, dict(factor=16.0, context=4096.0)),
                                        (3, dict(factor=4.0, context=2048.0, beta_slow=2.0, beta_fast=20.0, mscale=1.5))])
@pytest.mark.parametrize("r", [2, 64, 250])
def test_rotary_angles(scaling, kw, r):
    """The 64-bit fractions of a turn against the formulas in extended precision."""
    if scaling == 2 and r == 2:
        pytest.skip("NTK scaling needs a rot_dim above 2")
    d = L.RotaryDesc(0, scaling, 256, r, 500000.0, kw.get("factor", 1.0), kw.get("context", 0.0), kw.get("beta_slow", 0.0),
                     kw.get("beta_fast", 0.0), kw.get("mscale", 0.0))
    t = Table()
    fn = host_rule("_ZN5mopar12rotary_tableERK17mopar_rotary_descPNS_11RotaryTableE", ctypes.c_void_p, ctypes.c_void_p)
    assert fn(ctypes.addressof(d), ctypes.addressof(t)) == 0
    f, ld = np.longdouble(kw.get("factor", 1.0)), np.longdouble
    pi = ld("3.14159265358979323846264338327950288")
    base = ld(500000.0) * (f ** (ld(r) / (r - 2)) if scaling == 2 else 1)
    for j in range(r // 2):
        w = base ** (ld(-2 * j) / r)
        if scaling == 1:
            w = w / f
        if scaling == 3:
            slow, fast = (kw.get("beta_slow", 1.0), kw.get("beta_fast", 32.0))
            g = min(max((ld(kw["context"]) * w / (2 * pi) - slow) / (fast - slow), ld(0)), ld(1))
            w = w * (g + (1 - g) / f)
        want = Fraction(*(w / (2 * pi)).as_integer_ratio()) * 2 ** 64
        assert abs(t.w[j] - want) <= max(Fraction(1), want * Fraction(1, 2 ** 58))
    m = kw.get("mscale") or (0.1 * math.log(float(f)) + 1 if scaling == 3 else 1.0)
    assert t.m == np.float32(m) and (t.d, t.rot, t.inter) == (256, r, 0)


def apply_status(dtype=L.MOPAR_BF16, tokens=4, heads=2, pos=A, x=None, y=None, rot=None):
    rot = rot or rotary()
    return status("mopar_rotary_apply", rot.handle, dtype, tokens, heads, pos, ctypes.byref(x or rows()), ctypes.byref(y or rows()), None)


def test_rotary_apply_refusals():
    E = L.MOPAR_E_ARG
    assert apply_status(tokens=0) == 0 and apply_status(heads=0) == 0
    assert apply_status(tokens=-1) == E and apply_status(heads=-1) == E and apply_status(pos=None) == E
    assert apply_status(dtype=L.MOPAR_I32) == L.MOPAR_E_DTYPE
    assert apply_status(tokens=1 << 30, heads=2) == L.MOPAR_E_UNSUPPORTED
    assert apply_status(rot=rotary(head_dim=100)) == L.MOPAR_E_UNSUPPORTED
    for bad in (rows(None), rows(A + 2), rows(A, 1020), rows(A, 1024, 4), rows(A, -1024), rows(A, 1024, -128)):
        assert apply_status(x=bad) == E and apply_status(y=bad) == E
    assert apply_status(x=rows(A, 1 << 26)) == L.MOPAR_E_UNSUPPORTED
    assert apply_status(y=rows(A, 128, 128)) == E and apply_status(y=rows(A, 1024, 64)) == E      # rows overlap
    r = rotary()
    assert status("mopar_rotary_apply", None, L.MOPAR_BF16, 4, 2, A, ctypes.byref(rows()), ctypes.byref(rows()), None) == E
    assert status("mopar_rotary_apply", r.handle, L.MOPAR_BF16, 4, 2, A, None, ctypes.byref(rows()), None) == E


BAD_CACHES = [(dict(dtype=2), L.MOPAR_E_DTYPE), (dict(kv_heads=0), 1), (dict(head_dim=20), 4), (dict(head_dim=264), 4),
              (dict(head_dim=0), 4), (dict(page_tokens=24), 1), (dict(page_tokens=0), 1), (dict(page_tokens=8192), 1),
              (dict(pages=0), 1), (dict(pages=1 << 31), 1), (dict(n_seq=-1), 1), (dict(max_pages=0), 1), (dict(table_stride=7), 1),
              (dict(max_pages=1 << 28, table_stride=1 << 28), 1), (dict(k=None), 1), (dict(v=A + 8), 1), (dict(table_dev=None), 1)]


def append_status(c=None, rot=None, tokens=5, heads=8, pos=A, seq=A, slot=A, q=None, q_out=None, k=None, v=None):
    h = rot.handle if rot else None
    return status("mopar_cache_append", ctypes.byref(c or cache()), h, tokens, heads, pos, seq, slot, ctypes.byref(q or rows()),
                  ctypes.byref(q_out or rows()), ctypes.byref(k or rows()), ctypes.byref(v or rows()), None)


def test_append_refusals():
    E = L.MOPAR_E_ARG
    for kw, want in BAD_CACHES:
        assert append_status(cache(**kw)) == want, kw
    assert append_status(tokens=0) == 0 and append_status(tokens=-1) == E and append_status(heads=-1) == E
    r = rotary()
    for kw in (dict(seq=None), dict(slot=None), dict(pos=None, rot=r), dict(rot=rotary(head_dim=64)), dict(rot=r, q=rows(A + 4)),
               dict(rot=r, q_out=rows(A, 128)), dict(k=rows(None)), dict(v=rows(A, 1025))):
        assert append_status(**kw) == E, kw
    assert append_status(tokens=1 << 30) == L.MOPAR_E_UNSUPPORTED
    assert status("mopar_cache_append", None, None, 1, 0, A, A, A, None, None, ctypes.byref(rows()), ctypes.byref(rows()), None) == E


def keep_status(c=None, layers=1, stride=0, ln=A, off=A, entries=4, path=A, max_path=4):
    return status("mopar_cache_keep", ctypes.byref(c or cache()), layers, stride, ln, off, entries, path, max_path, None)


def test_keep_refusals():
    E = L.MOPAR_E_ARG
    for kw, want in BAD_CACHES:
        assert keep_status(cache(**kw)) == want, kw
    for kw in (dict(layers=0), dict(entries=0), dict(max_path=0), dict(c=cache(n_seq=0))):
        assert keep_status(**kw) == 0
    one = 100 * 2 * 16 * 128
    for kw in (dict(layers=-1), dict(entries=-1), dict(max_path=-1), dict(ln=None), dict(off=None), dict(path=None),
               dict(layers=2, stride=one - 8), dict(layers=2, stride=one + 4)):
        assert keep_status(**kw) == E, kw
    assert keep_status(layers=1 << 30, stride=one, c=cache(n_seq=2)) == L.MOPAR_E_UNSUPPORTED


BAD_ATTENTION = [(dict(dtype=2), L.MOPAR_E_DTYPE), (dict(heads=0), 1), (dict(kv_heads=0), 1), (dict(heads=7), 1), (dict(head_dim=80), 4),
                 (dict(head_dim=256), 4), (dict(scale=0.0), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1)]


def prompt_status(a=None, tokens=10, n_seq=2, off=A, max_len=5, q=None, k=None, v=None, out=None):
    r = rows
    return status("mopar_attention_prompt", ctypes.byref(a or attention()), tokens, n_seq, off, max_len, ctypes.byref(q or r()),
                  ctypes.byref(k or r()), ctypes.byref(v or r()), ctypes.byref(out or r()), None)


def test_prompt_refusals():
    E = L.MOPAR_E_ARG
    for kw, want in BAD_ATTENTION:
        assert prompt_status(attention(**kw)) == want, kw
    for kw in (dict(tokens=0), dict(n_seq=0), dict(max_len=0)):
        assert prompt_status(**kw) == 0
    for kw in (dict(tokens=-1), dict(tokens=1 << 31), dict(n_seq=-1), dict(max_len=-1), dict(off=None), dict(q=rows(None)), dict(k=rows(A + 8)),
               dict(v=rows(A, 1028)), dict(out=rows(A, 512)), dict(out=rows(A, 1024, 120))):
        assert prompt_status(**kw) == E, kw
    assert prompt_status(attention(heads=65536), n_seq=1 << 20, tokens=10) == L.MOPAR_E_UNSUPPORTED
    assert prompt_status(k=rows(A, 1 << 26)) == L.MOPAR_E_UNSUPPORTED


def ws_bytes(a=None, c=None, tokens=10, max_q=4, max_len=100):
    n = ctypes.c_size_t()
    st = status("mopar_attention_cache_workspace_bytes", ctypes.byref(a or attention()), ctypes.byref(c or cache()), tokens, max_q, max_len,
                ctypes.byref(n))
    return st, n.value


def cache_status(a=None, c=None, tokens=10, off=A, max_q=4, ln=A, max_len=100, mask=None, words=0, q=None, out=None, ws=A, ws_n=1 << 40):
    return status("mopar_attention_cache", ctypes.byref(a or attention()), ctypes.byref(c or cache()), tokens, off, max_q, ln, max_len, mask, words,
                  ctypes.byref(q or rows()), ctypes.byref(out or rows()), ws, ws_n, None)


def test_cache_attention_refusals():
    E = L.MOPAR_E_ARG
    for kw, want in BAD_ATTENTION:
        assert cache_status(attention(**kw)) == want and ws_bytes(attention(**kw))[0] == want, kw
    for kw, want in BAD_CACHES:
        assert cache_status(c=cache(**kw)) == want, kw
    for kw in (dict(tokens=0), dict(max_q=0), dict(c=cache(n_seq=0))):
        assert cache_status(**kw) == 0
    for kw in (dict(a=attention(kv_heads=4)), dict(a=attention(head_dim=64)), dict(a=attention(dtype=0)), dict(tokens=-1), dict(max_q=-1),
               dict(max_len=0), dict(off=None), dict(ln=None), dict(mask=A, words=0), dict(mask=A, words=1, max_q=65), dict(mask=A + 4, words=1),
               dict(q=rows(None)), dict(out=rows(A, 1024, 64)), dict(max_len=100000, ws=None), dict(max_len=100000, ws=A + 8)):
        assert cache_status(**kw) == E, kw
    assert cache_status(max_q=1 << 18) == L.MOPAR_E_UNSUPPORTED
    assert cache_status(c=cache(n_seq=1 << 30), max_len=1 << 20) == L.MOPAR_E_UNSUPPORTED
    st, need = ws_bytes(max_len=100000)
    assert st == 0 and need > 0
    assert cache_status(max_len=100000, ws_n=need - 1) == L.MOPAR_E_WORKSPACE
    assert ws_bytes(max_len=1) == (0, 0)


def test_sizes_that_no_grid_or_offset_holds():
    """Sizes at which an index, a byte offset or a grid would not fit are refused, and the last that fit are not."""
    E, U = L.MOPAR_E_ARG, L.MOPAR_E_UNSUPPORTED
    assert apply_status(heads=65537) == E and apply_status(x=rows(A, 1024, 1 << 44)) == E
    # one pair of dims a thread: 2^30 rows of 31 units
    assert apply_status(rot=rotary(head_dim=32, rot_dim=2), tokens=1 << 30, heads=1) == U
    with pytest.raises(P.MoparError):
        rotary(mscale=1e39)
    big = cache(kv_heads=65536, page_tokens=4096, head_dim=256, pages=1 << 11)
    assert append_status(big, k=rows(None)) == E and b"elements" in P.lib().mopar_last_error()
    assert prompt_status(attention(scale=3e38)) == E
    assert prompt_status(tokens=1 << 30) == U
    assert prompt_status(attention(heads=64), n_seq=1 << 18, tokens=1 << 20) == U
    wide = cache(page_tokens=4096, max_pages=1 << 18, table_stride=1 << 18)
    wider = cache(page_tokens=4096, max_pages=(1 << 18) + 1, table_stride=(1 << 18) + 1)
    assert ws_bytes(c=wide, max_len=2 ** 31 - 1)[0] == 0 and ws_bytes(c=wider, max_len=1 << 30)[0] == 0
    assert ws_bytes(c=wider, max_len=(1 << 30) + 1)[0] == U
    assert ws_bytes(max_len=2 ** 31 - 1)[0] == 0
    assert ws_bytes(c=cache(n_seq=(1 << 21) - 1), max_len=1)[0] == 0 and ws_bytes(c=cache(n_seq=1 << 21), max_len=1)[0] == U
    assert keep_status(layers=1 << 12, stride=1 << 20, c=cache(n_seq=1 << 12)) == U


def test_layers_whose_offsets_no_word_holds():
    """Byte offsets of the layers stay within 2^60; the stride of a single layer is not read."""
    far = 1 << 61
    assert keep_status(layers=2, stride=far) == L.MOPAR_E_ARG and b"2^58 elements" in P.lib().mopar_last_error()
    assert keep_status(layers=2, stride=1 << 57, ln=None) == L.MOPAR_E_ARG and b"null" in P.lib().mopar_last_error()
    assert keep_status(layers=1, stride=far, ln=None) == L.MOPAR_E_ARG and b"null" in P.lib().mopar_last_error()


def test_a_cache_of_no_sequences_needs_no_table():
    none = cache(n_seq=0, table_dev=None)
    assert keep_status(none) == 0 and cache_status(c=none) == 0
    assert append_status(none, tokens=0) == 0


@pytest.mark.parametrize("dtype,dims", [(L.MOPAR_BF16, (32, 64, 96, 128)), (L.MOPAR_F32, (32, 64, 96, 128))])
def test_a_workspace_holds_smaller_calls(dtype, dims):
    """The size does not fall as sequences, drafted tokens or the limit grow."""
    steps = dict(n_seq=(1, 3, 40, 700, 20000), max_q=(1, 5, 8, 9, 16, 17, 64, 65, 300), max_len=(1, 33, 129, 160, 289, 321, 700, 5000, 100000))
    for d in dims:
        def need(n_seq, max_q, max_len):
            st, n = ws_bytes(attention(dtype=dtype, head_dim=d), cache(dtype=dtype, head_dim=d, n_seq=n_seq), 10, max_q, max_len)
            return n if st == 0 else None
        size = {(i, j, k): need(a, b, c) for i, a in enumerate(steps["n_seq"]) for j, b in enumerate(steps["max_q"])
                for k, c in enumerate(steps["max_len"])}
        for (i, j, k), n in size.items():
            for up in ((i + 1, j, k), (i, j + 1, k), (i, j, k + 1)):
                if size.get(up) is not None:
                    assert n <= size[up], (d, (i, j, k), up)


def test_binding_refuses_mismatched_tensors():
    bf = torch.bfloat16
    k = torch.zeros(4, 2, 16, 64, dtype=bf)
    table = torch.zeros(2, 2, dtype=torch.int32)
    c = P.PagedCache(k, k.clone(), table)
    x = torch.zeros(3, 2, 64, dtype=bf)
    i3, i2 = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    rot = rotary(head_dim=64)
    bad = [lambda: P.mopar_rotary_apply(rot, x, x[:2], i3), lambda: P.mopar_rotary_apply(rot, x, x, i2),
           lambda: P.mopar_rotary_apply(rot, x, x, i3.long()), lambda: P.mopar_rotary_apply(rotary(), x, x, i3),
           lambda: P.mopar_rotary_apply(rot, x.float(), x, i3), lambda: P.mopar_rotary_apply(rot, x, x, i3),    # on the CPU
           lambda: P.mopar_rotary_apply(rot, x.half(), x.half(), i3),
           lambda: P.PagedCache(k, k[:3], table), lambda: P.PagedCache(k, k.float(), table), lambda: P.PagedCache(k.transpose(1, 2), k.transpose(1, 2), table),
           lambda: P.PagedCache(k, k, table.long()), lambda: P.PagedCache(k, k, table[0]), lambda: c.layer(0),
           lambda: P.mopar_cache_append(c, x, x[:2], i3, i3), lambda: P.mopar_cache_append(c, x, x, i3, i2),
           lambda: P.mopar_cache_append(c, x, x, i3, i3, rotary=rot), lambda: P.mopar_cache_append(c, x, x, i3, i3, pos=i3),
           lambda: P.mopar_cache_append(c, x, x, i3, i3, rotary=rot, pos=i3, q=x),
           lambda: P.mopar_cache_append(P.PagedCache(k[None], k[None], table), x, x, i3, i3),
           lambda: P.mopar_cache_keep(c, i3, i3, i3, 1), lambda: P.mopar_cache_keep(c, i2, i2, i3, 1),
           lambda: P.mopar_attention_prompt(x, x, x[:, :1], x, i2, 3), lambda: P.mopar_attention_prompt(x, x, x, x[:2], i2, 3),
           lambda: P.mopar_attention_prompt(x, x, x, x, i2.long(), 3), lambda: P.mopar_attention_prompt(x, x, x, x, i2[:0], 3),
           lambda: P.mopar_attention_cache(x, x, c, i2, 1, i2, 3), lambda: P.mopar_attention_cache(x, x, c, i3, 1, i3, 3),
           lambda: P.mopar_attention_cache(x, x, c, i3, 1, i2, 3, mask=torch.zeros(2, 1, dtype=torch.int64))]
    for f in bad:
        with pytest.raises(ValueError):
            f()


def test_binding_refuses_sizes_past_32_bits():
    """They are not answered as what their lower 32 bits say."""
    bf, past = torch.bfloat16, 1 << 32
    k = torch.zeros(4, 2, 16, 64, dtype=bf)
    c = P.PagedCache(k, k.clone(), torch.zeros(2, 2, dtype=torch.int32))
    x = torch.zeros(3, 2, 64, dtype=bf)
    i3, i2 = torch.zeros(3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for what, f in [("max_len", lambda n: P.mopar_attention_prompt(x, x, x, x, i2, n)),
                    ("max_len", lambda n: P.mopar_attention_cache(x, x, c, i3, 1, i2, n)), ("max_q", lambda n: P.mopar_attention_cache(x, x, c, i3, n, i2, 8)),
                    ("max_len", lambda n: P.mopar_attention_cache_workspace_bytes(x, c, 1, n)),
                    ("max_q", lambda n: P.alloc_attention_workspace(x, c, n, 8)), ("max_path", lambda n: P.mopar_cache_keep(c, i2, i3, i3, n)),
                    ("rot_dim", lambda n: P.Rotary(64, rot_dim=n)), ("head_dim", lambda n: P.Rotary(n, rot_dim=32))]:
        for n in (past + 32, 1 << 31, -past):
            with pytest.raises(ValueError, match=what):
                f(n)


def test_the_version_tells_the_layout_of_the_structs():
    """mopar_op of version 0.1 had no rotary descriptor and ended at w5."""
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "mopar.h")) as f:
        version = re.search(r'#define MOPAR_VERSION "([0-9.]+)"', f.read())[1]
    assert P.lib().mopar_version().decode() == f"mopar-mi355x {version} (gfx950)"
    assert version != "0.1" and ctypes.sizeof(L.Op) == L.Op.w5.offset + 8 + 8 + ctypes.sizeof(L.RotaryDesc)


def test_binding_refuses_tables_whose_rows_overlap():
    """A table of one row expanded over the sequences has no row behind the first: it is not read as if it had."""
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    row = torch.zeros(1, 3, dtype=torch.int32)
    for table in (row.expand(5, 3), row[:, :1].expand(5, 1), torch.zeros(9, dtype=torch.int32).as_strided((3, 3), (2, 1))):
        with pytest.raises(ValueError, match="table"):
            P.PagedCache(k, k.clone(), table)
    wide = torch.zeros(4, 8, dtype=torch.int32)
    assert P.PagedCache(k, k.clone(), wide[:, 2:5]).raw.table_stride == 8
    assert P.PagedCache(k, k.clone(), row.expand(1, 3)).raw.table_stride == 3
    assert P.PagedCache(k, k.clone(), wide[:, :1]).raw.table_stride == 8
