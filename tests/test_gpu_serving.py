"""Decoding with a paged cache on the GPU against plain float64 forms: rotary positions, cache writes, prompt
attention, attention over the cache, kept paths, and a run of them together."""
import pytest
import torch

import paper_2404_02445_amd as P
from tests.serving_ref import (attend, cache_rows, check, pack_mask, page_table, rotate, rotate_tol, tree_mask)

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, dt="bf16"):
    return torch.randn(shape, generator=g).to(DT[dt]).cuda()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# --- rotary positions --------------------------------------------------------------------------

@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("tokens,heads,d,rot", [(1, 1, 64, 64), (7, 5, 64, 32), (301, 3, 128, 128), (5, 40, 96, 96), (33, 2, 64, 20),
                                                (3, 4, 256, 256), (9, 2, 16, 2), (130, 6, 128, 94)])
def test_rotary(dt, layout, tokens, heads, d, rot):
    g = gen(tokens + d + rot)
    rows = randn(g, tokens, heads + 2, d, dt=dt)
    x = rows[:, 1:heads + 1]
    pos = torch.randint(0, 5000, (tokens,), generator=g, dtype=torch.int32).cuda()
    y = torch.full((tokens, heads, d), 7.0, device="cuda", dtype=DT[dt])
    P.mopar_rotary_apply(P.Rotary(d, rot_dim=rot, layout=layout), x, y, pos)
    ref, mag = rotate(x, pos, rot, layout)
    check(y, ref, rotate_tol(ref, mag, DT[dt]))
    assert torch.equal(y[..., rot:], x[..., rot:])
    before = rows.clone()
    P.mopar_rotary_apply(P.Rotary(d, rot_dim=rot, layout=layout), x, x, pos)          # in place, the rows around untouched
    assert torch.equal(x, y)
    assert torch.equal(rows[:, 0], before[:, 0]) and torch.equal(rows[:, -1], before[:, -1])


@pytest.mark.parametrize("scaling,kw,m", [("linear", dict(factor=4.0), 1.0), ("ntk", dict(factor=8.0), 1.0),
                                          ("yarn", dict(factor=16.0, context=4096), 0.1 * torch.log(torch.tensor(16.0, dtype=torch.float64)).item() + 1),
                                          ("none", dict(), 1.0)])
def test_rotary_scaled_and_far(scaling, kw, m):
    g = gen(3)
    x = randn(g, 6, 3, 128, dt="f32")
    pos = ints([0, 1, 131071, 2 ** 31 - 1, -5, -2 ** 31])
    y = torch.empty_like(x)
    P.mopar_rotary_apply(P.Rotary(128, base=500000.0, scaling=scaling, **kw), x, y, pos)
    ref, mag = rotate(x, pos, 128, m=m, base=500000.0, scaling=scaling, **kw)
    check(y, ref, rotate_tol(ref, mag, torch.float32, far=2 ** 31))


def test_rotary_heads_outside_tokens_and_mscale():
    g = gen(4)
    x = randn(g, 3, 50, 64).transpose(0, 1)                 # [tokens, heads, d] inside [heads, tokens, d]
    y = torch.empty(3, 50, 64, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    P.mopar_rotary_apply(P.Rotary(64, mscale=0.5), x, y, pos)
    ref, mag = rotate(x, pos, 64, m=0.5)
    check(y, ref, rotate_tol(ref, mag, torch.bfloat16))


def test_rotary_passes_nan_beside_what_turns():
    x = torch.zeros(2, 1, 64, device="cuda", dtype=torch.float32)
    x[:, :, 10:] = float("nan")
    y = torch.empty_like(x)
    P.mopar_rotary_apply(P.Rotary(64, rot_dim=10, layout="interleaved"), x, y, ints([3, 4]))
    assert bool((y[:, :, :10] == 0).all()) and bool(y[:, :, 10:].isnan().all())


# --- cache writes --------------------------------------------------------------------------------

@pytest.mark.parametrize("dt,kv,heads,d,page,rot,layout", [("bf16", 2, 6, 128, 16, 128, "half"), ("f32", 3, 3, 64, 1, 32, "interleaved"),
                                                           ("bf16", 1, 8, 96, 64, 30, "half"), ("f32", 2, 2, 32, 256, 32, "half"),
                                                           ("bf16", 5, 5, 16, 8, 0, "half")])
def test_append(dt, kv, heads, d, page, rot, layout):
    g = gen(d + page)
    past, new = [5, 0, 300, 17], [3, 70, 1, 0]
    table, pages = page_table([a + b for a, b in zip(past, new)], page, g)
    table = table.cuda()
    kc, vc = (randn(g, pages, kv, page, d, dt=dt) for _ in range(2))
    seq = [s for s, n in enumerate(new) for _ in range(n)] + [-1, 4, 0, 0]          # padding, no such sequence, slots out of range
    slot = [past[s] + i for s, n in enumerate(new) for i in range(n)] + [0, 0, -1, table.shape[1] * page]
    t = len(seq)
    rows = randn(g, t, heads + 2 * kv, d, dt=dt)
    q, k, v = rows[:, :heads], rows[:, heads:heads + kv], rows[:, heads + kv:]
    pos = torch.randint(0, 3000, (t,), generator=g, dtype=torch.int32).cuda()
    want_k, want_v = kc.clone(), vc.clone()
    q_out = torch.full((t, heads, d), 7.0, device="cuda", dtype=DT[dt])
    cache = P.PagedCache(kc, vc, table)
    turned = k
    if rot:
        r = P.Rotary(d, rot_dim=rot, layout=layout)
        P.mopar_cache_append(cache, k, v, ints(seq), ints(slot), rotary=r, pos=pos, q=q, q_out=q_out)
        turned = torch.empty(t, kv, d, device="cuda", dtype=DT[dt])
        P.mopar_rotary_apply(r, k, turned, pos)
        ref, mag = rotate(q, pos, rot, layout)
        check(q_out, ref, rotate_tol(ref, mag, DT[dt]))
    else:
        P.mopar_cache_append(cache, k, v, ints(seq), ints(slot))
    for i in range(sum(new)):
        p, at = int(table[seq[i], slot[i] // page]), slot[i] % page
        want_k[p, :, at], want_v[p, :, at] = turned[i], v[i]
    assert torch.equal(kc, want_k) and torch.equal(vc, want_v)


def test_append_keeps_off_absent_pages():
    g = gen(9)
    kc, vc = (randn(g, 4, 2, 16, 64) for _ in range(2))
    before = kc.clone(), vc.clone()
    k, v = randn(g, 3, 2, 64), randn(g, 3, 2, 64)
    table = ints([[-1, 4, 2 ** 31 - 1]])
    P.mopar_cache_append(P.PagedCache(kc, vc, table), k, v, ints([0, 0, 0]), ints([3, 20, 40]))
    assert torch.equal(kc, before[0]) and torch.equal(vc, before[1])


@pytest.mark.parametrize("dt,kv,d,page,layers", [("bf16", 8, 128, 16, 3), ("f32", 1, 32, 1, 1), ("bf16", 3, 96, 64, 2)])
def test_keep(dt, kv, d, page, layers):
    g = gen(page)
    past, drafts = [5, 31, 0, 100, 12], 30
    paths = [[0, 3, 7, 8, 20], [29], [], [0, 1, 2], [1, 4, 5, 6, 10, 11, 12, 13, 21, 22, 23, 29]]
    table, pages = page_table([p + drafts for p in past], page, g)
    kc, vc = (randn(g, layers, pages, kv, page, d, dt=dt) for _ in range(2))
    want = [kc.clone(), vc.clone()]
    for pool in want:
        old = pool.clone()
        for s, path in enumerate(paths):
            for i, j in enumerate(path):
                a, b = past[s] + i, past[s] + j
                pool[:, table[s, a // page], :, a % page] = old[:, table[s, b // page], :, b % page]
    if layers == 1:
        kc, vc, want = kc[0], vc[0], [w[0] for w in want]
    off = [0]
    for p in paths:
        off.append(off[-1] + len(p))
    P.mopar_cache_keep(P.PagedCache(kc, vc, table.cuda()), ints(past), ints(off), ints([i for p in paths for i in p]), 12)
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])


def test_keep_bounds():
    """Indices below their place, negative ones, absent pages and entries past max_path move nothing."""
    g = gen(2)
    kc, vc = (randn(g, 6, 2, 8, 64) for _ in range(2))
    want = kc.clone(), vc.clone()
    table = ints([[0, 1, -1], [2, 9, 3], [4, 5, 1]])
    # sequence 0: [5] moves, then 0 < 1 and -3 do not, then slot 16 (absent) does not; 1: to and from page 9; 2: cut after four
    paths, off = [5, 0, -3, 14, 3, 9, 2, 3, 4, 5, 6], [0, 4, 6, 11]
    P.mopar_cache_keep(P.PagedCache(kc, vc, table), ints([2, 7, 0]), ints(off), ints(paths), 4)
    for w in want:
        old = w.clone()
        w[0, :, 2] = old[0, :, 7]                       # slot 7 -> 2 of sequence 0
        for i, j in enumerate([2, 3, 4, 5]):
            w[4, :, i] = old[4, :, j]
    # sequence 1: slot 10 (page 9: absent) -> 7 and slot 16 -> 8 (absent): nothing
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])


# --- prompt attention ----------------------------------------------------------------------------

def prompt(q, k, v, lens, offsets=None, max_len=None, out=None):
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    out = torch.full((q.shape[0], q.shape[1], q.shape[2]), 7.0, device="cuda", dtype=q.dtype) if out is None else out
    return P.mopar_attention_prompt(q, k, v, out, ints(off if offsets is None else offsets), max_len or max(lens))


def causal(n):
    return torch.ones(n, n, dtype=torch.bool).tril()


def check_prompt(out, q, k, v, lens, scale=None):
    at = 0
    for n in lens:
        ref, tol = attend(q[at:at + n], k[at:at + n], v[at:at + n], causal(n), q.shape[2] ** -0.5 if scale is None else scale)
        check(out[at:at + n], ref, tol, f"rows {at} to {at + n}")
        at += n
    assert bool((out[at:] == 7.0).all()), "rows behind the last sequence"


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("lens", [[1], [2, 1, 0, 33], [31, 32, 127], [128, 129, 257], [300, 0, 65]])
def test_prompt(dt, d, lens):
    g = gen(d + sum(lens))
    heads, kv, t = 6, 2, sum(lens) + 3
    rows = randn(g, t, heads + 2 * kv, d, dt=dt)
    rows[:, :heads] *= 2
    q, k, v = rows[:, :heads], rows[:, heads:heads + kv], rows[:, heads + kv:]
    check_prompt(prompt(q, k, v, lens), q, k, v, lens)


@pytest.mark.parametrize("dt,heads,kv", [("bf16", 1, 1), ("bf16", 5, 5), ("bf16", 8, 1), ("f32", 7, 7), ("f32", 14, 2)])
def test_prompt_heads(dt, heads, kv):
    g = gen(heads)
    lens = [70, 200]
    q, k, v = randn(g, 270, heads, 64, dt=dt), randn(g, 270, kv, 64, dt=dt), randn(g, 270, kv, 64, dt=dt)
    check_prompt(prompt(q, k, v, lens), q, k, v, lens)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv,d", [(4, 2, 64), (8, 2, 128), (12, 2, 32), (24, 3, 96)])
def test_prompt_groups_of_two_and_four_heads(dt, heads, kv, d):
    """Tiles of two or four heads of a key head, and lengths round their 64 and 32 tokens."""
    g = gen(heads + d)
    lens = [33, 0, 129, 1, 64, 31, 96]
    t = sum(lens) + 2
    q, k, v = randn(g, t, heads, d, dt=dt), randn(g, t, kv, d, dt=dt), randn(g, t, kv, d, dt=dt)
    check_prompt(prompt(q, k, v, lens), q, k, v, lens)


def test_prompt_long():
    g = gen(5)
    n = 4500
    q, k, v = randn(g, n, 2, 128), randn(g, n, 1, 128), randn(g, n, 1, 128)
    check_prompt(prompt(q, k, v, [n]), q, k, v, [n])


def test_prompt_many_sequences():
    g = gen(6)
    lens = [(7 * i) % 23 for i in range(300)]
    t = sum(lens)
    q, k, v = randn(g, t, 2, 64), randn(g, t, 2, 64), randn(g, t, 2, 64)
    check_prompt(prompt(q, k, v, lens), q, k, v, lens)


def test_prompt_strides_and_order():
    g = gen(7)
    q = randn(g, 4, 100, 64).transpose(0, 1)                # heads outside tokens
    k, v = randn(g, 100, 1, 200)[..., 8:72], randn(g, 100, 1, 64)
    out = torch.full((4, 100, 64), 7.0, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    check_prompt(prompt(q, k, v, [40, 60], out=out), q, k, v, [40, 60])


def test_prompt_large_scores():
    """Maxima that rise from tile to tile, and scores far past exp's range."""
    g = gen(8)
    n = 200
    q, k, v = randn(g, n, 1, 64, dt="f32") * 8, randn(g, n, 1, 64, dt="f32"), randn(g, n, 1, 64, dt="f32")
    k *= torch.linspace(0.1, 30, n, device="cuda")[:, None, None]
    check_prompt(prompt(q, k, v, [n]), q, k, v, [n])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_prompt_hidden_values_do_not_reach_a_row(dt):
    g = gen(9)
    lens = [140, 50]
    q, k, v = (randn(g, 192, 2, 64, dt=dt) for _ in range(3))
    v[70, 0, 3], v[71, 1, 5], v[72, 0, 63] = float("inf"), float("-inf"), float("nan")
    k[100, 0, 7] = float("nan")
    v[139, 1], k[139, 1] = float("nan"), float("inf")
    v[190:], k[190:] = float("nan"), float("nan")           # rows of no sequence
    out = prompt(q, k, v, lens)
    o = out.double().cpu()
    assert bool(torch.isfinite(o[:70]).all()) and bool(torch.isfinite(o[140:190]).all())
    assert bool((o[70:100, 0, 3] == float("inf")).all()) and bool((o[71:139, 1, 5] == float("-inf")).all())
    assert bool(o[72:140, 0, 63].isnan().all()) and bool(o[100:140, 0].isnan().all()) and bool(o[139, 1].isnan().all())
    rest = o[70:100, 0].clone()
    rest[:, 3] = 0
    rest[2:, 63] = 0
    assert bool(torch.isfinite(rest).all())
    check_prompt(torch.cat([out[140:190], out[190:]]), q[140:], k[140:], v[140:], [50])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_prompt_hidden_values_in_grouped_heads(dt):
    """Infinities and NaN reach the same dims of the same rows whether a key head is shared or given once a head."""
    g = gen(10)
    q, k, v = randn(g, 150, 4, 64, dt=dt), randn(g, 150, 1, 64, dt=dt), randn(g, 150, 1, 64, dt=dt)
    v[33, 0, 3], v[70, 0, 5], v[149, 0, 1] = float("inf"), float("nan"), float("-inf")
    k[95, 0, 7] = float("nan")
    k4, v4 = k.expand(150, 4, 64).contiguous(), v.expand(150, 4, 64).contiguous()
    for n in (2, 4):
        out, each = prompt(q[:, :n], k, v, [150]), prompt(q[:, :n], k4[:, :n], v4[:, :n], [150])
        for kind in (torch.isnan, torch.isposinf, torch.isneginf):
            assert torch.equal(kind(out), kind(each))
        assert bool(torch.isfinite(out[:33]).all()) and bool((out[33:95, :, 3] == float("inf")).all())


def test_prompt_offsets_out_of_bounds_are_cut():
    g = gen(10)
    q, k, v = (randn(g, 50, 2, 64) for _ in range(3))
    out = torch.full_like(q, 7.0)
    P.mopar_attention_prompt(q, k, v, out, ints([-7, 20, 10, 30, 10 ** 9]), 25)
    ref = torch.full_like(q, 7.0)
    P.mopar_attention_prompt(q, k, v, ref, ints([0, 20]), 25)
    assert torch.equal(out[:10], ref[:10])


# --- attention over the cache ------------------------------------------------------------------

def over_cache(g, dt, heads, kv, d, page, lens, new, mask, spare=0, max_len=None, absent=None, poison=True):
    t, top = sum(new) + spare, max(max(new), 1)
    table, pages = page_table([a + b for a, b in zip(lens, new)], page, g)
    kc, vc = (randn(g, pages, kv, page, d, dt=dt) for _ in range(2))
    q = randn(g, t, heads, d, dt=dt) * 2
    if absent is not None:
        table[absent[0], absent[1]] = absent[2]
    if poison:                                              # what no sequence holds is NaN
        held = torch.zeros(pages, page, dtype=torch.bool)
        for s, (a, b) in enumerate(zip(lens, new)):
            for i in range(a + b):
                p = int(table[s, i // page])
                if 0 <= p < pages:
                    held[p, i % page] = True
        for pool in (kc, vc):
            pool.masked_fill_(~held[:, None, :, None].cuda(), float("nan"))
    words = (top + 63) // 64
    seen, bits = [], []
    for n in new:
        a = mask(n) if mask else causal(n)
        seen.append(a)
        bits.append(pack_mask(a, words))
    bits.append(torch.full((spare, words), -1))
    off = [0]
    for n in new:
        off.append(off[-1] + n)
    out = torch.full((t, heads, d), 7.0, device="cuda", dtype=DT[dt])
    cache = P.PagedCache(kc, vc, table.cuda())
    longest = max_len or max(a + b for a, b in zip(lens, new))
    ws = P.alloc_attention_workspace(q, cache, top, max(longest, 1))
    ws.fill_(0xFF)
    args = (q, out, cache, ints(off), top, ints(lens), max(longest, 1))
    m = torch.cat(bits).cuda() if mask else None
    P.mopar_attention_cache(*args, mask=m, ws=ws)
    kcp, vcp = kc.cpu(), vc.cpu()
    for s, n in enumerate(new):
        total = lens[s] + n
        vis = torch.cat([torch.ones(n, lens[s], dtype=torch.bool), seen[s]], 1)[:, :min(total, longest)]
        for i in range(vis.shape[1]):
            p = int(table[s, i // page])
            if not 0 <= p < pages:
                vis[:, i] = False
        k, v = (cache_rows(x, table, s, vis.shape[1]) for x in (kcp, vcp))
        ref, tol = attend(q[off[s]:off[s + 1]], k, v, vis, d ** -0.5)
        check(out[off[s]:off[s + 1]], ref, tol, f"sequence {s}")
    assert bool((out[off[-1]:] == 7.0).all()), "rows behind the last sequence"
    return args, m, ws


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 96, 128])
@pytest.mark.parametrize("heads,kv", [(8, 2), (3, 3)])
def test_single_tokens(dt, d, heads, kv):
    over_cache(gen(d), dt, heads, kv, d, 16, [0, 1, 31, 128, 700, 255], [1, 1, 1, 1, 1, 0], None, spare=2)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(32, 64), (64, 1), (96, 8), (128, 32), (128, 256)])
@pytest.mark.parametrize("new", [[5, 1, 0, 8], [40, 64, 17, 3], [130, 2, 70, 65]])
def test_trees(dt, d, page, new):
    g = gen(d + page)
    over_cache(g, dt, 4, 2, d, page, [60, 0, 333, 1000], new, lambda n: tree_mask(n, g)[0] if n else causal(0), spare=1)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_chains_without_a_mask(dt):
    over_cache(gen(1), dt, 4, 4, 64, 16, [100, 0, 31], [33, 65, 1], None)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_rows_that_see_nothing(dt):
    def mask(n):
        a = causal(n)
        a[1::3] = False
        return a
    over_cache(gen(2), dt, 4, 1, 64, 8, [0, 0, 40], [7, 40, 30], mask)


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("f32", 64), ("bf16", 64)])
def test_cache_split_over_a_long_axis(dt, d):
    over_cache(gen(3), dt, 4, 2, d, 64, [5000, 300, 2047], [1, 1, 1], None)
    g = gen(4)
    over_cache(g, dt, 4, 2, d, 16, [3000, 3, 513], [9, 20, 12], lambda n: tree_mask(n, g)[0])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("new", [[1, 1, 0, 1, 1], [16, 3, 0, 9, 1], [40, 2, 0, 64, 17]])
def test_short_sequences_under_a_far_limit(dt, new):
    """A limit that lets the blocks share the work, on sequences that fill a few of the shares."""
    over_cache(gen(14), dt, 8, 2, 64, 16, [70, 0, 33, 1, 300], new, lambda n: tree_mask(n, gen(n))[0] if n else causal(0), spare=3, max_len=200000)


def shares(dt, d, heads, kv, seqs, top, limit):
    """Blocks that share a call's key stages, keys of a stage, rows of a tile: the rule, its workspace checked against the library's."""
    def plan(rows):
        bm = 32 if rows <= 32 else 64 if rows <= 64 else 256
        es = 2 if dt == "bf16" else 4
        kt = 64 if es == 2 and bm == 256 else 32
        stage = 2 * kt * (128 if d > 64 else d) * es
        ring = 4 if bm == 64 and stage == 16384 else 2
        slots = 256 * min(256 // bm, 160 * 1024 // (ring * stage + bm // 32 * 1024))
        units, nt = seqs * kv * -(-rows // bm), -(-limit // kt)
        blocks = min(slots, units * nt)
        saved = nt * -(-units // slots) - -(-nt * units // slots)
        return blocks * (2 * bm * (d + 2) * 4 + 32), blocks if saved > (9 if es == 2 else 4) else 0, kt, bm
    rows = top * heads // kv
    pool = torch.empty(1, kv, 16, d, dtype=DT[dt])
    cache = P.PagedCache(pool, pool, torch.zeros(seqs, 1, dtype=torch.int32))
    need = P.mopar_attention_cache_workspace_bytes(torch.empty(1, heads, d, dtype=DT[dt]), cache, top, limit)
    assert need == max(plan(r)[0] for r in (rows, min(rows, 32), min(rows, 64)))
    return plan(rows)[1:]


@pytest.mark.parametrize("dt,d,page", [("bf16", 128, 16), ("bf16", 64, 1), ("bf16", 96, 64), ("bf16", 32, 8), ("f32", 64, 16), ("f32", 128, 32),
                                       ("f32", 96, 1), ("f32", 32, 128)])
@pytest.mark.parametrize("seqs,top,tile", [(40, 1, 32), (40, 16, 64), (24, 40, 256)])
def test_shares_of_several_units(dt, d, page, seqs, top, tile):
    """Ragged sequences of which a block's share holds many stages: whole units, the end of one and the start of the next."""
    g = gen(seqs + d + page)
    kv = 8 if tile == 32 else 4
    heads = 4 * kv
    lens = [int(x) for x in torch.randint(1, 1500, (seqs,), generator=g)]
    new = [int(x) for x in torch.randint(1, top + 1, (seqs,), generator=g)]
    lens[0], lens[3], lens[4], lens[5], new[0], new[7] = 1500, 0, 1, 31, top, 0
    limit = 1500 + top
    blocks, kt, bm = shares(dt, d, heads, kv, seqs, top, limit)
    nt = [-(-(a + b) // kt) for a, b in zip(lens, new)]
    units = [kv * -(-n * 4 // bm) for n in new]
    per = -(-sum(a * b for a, b in zip(nt, units)) // blocks)
    assert bm == tile and blocks > 0 and per > 2 and per > 2 * min(n for n, u in zip(nt, units) if u)
    over_cache(g, dt, heads, kv, d, page, lens, new, (lambda n: tree_mask(n, g)[0] if n else causal(0)) if top > 1 else None, spare=2,
               absent=(0, 700 // page, -1), max_len=limit)


def test_one_workspace_for_every_size():
    """The largest call's workspace, full of NaN, under calls of fewer sequences and drafted tokens that share where it does not."""
    g = gen(15)
    d, page, n = 64, 16, 700
    table = torch.randperm(40 * 44, generator=g, dtype=torch.int32).view(40, 44).cuda()
    kc, vc = (randn(g, 40 * 44, 8, page, d) for _ in range(2))
    q = randn(g, 40 * 64, 8, d)
    ws = P.alloc_attention_workspace(q, P.PagedCache(kc, vc, table), 64, n)
    for seqs, new in ((40, 64), (40, 1), (3, 1), (1, 64), (1, 9)):
        cache, t = P.PagedCache(kc, vc, table[:seqs]), seqs * new
        off, ln = ints([i * new for i in range(seqs + 1)]), ints([n - new] * seqs)
        out = torch.empty(t, 8, d, device="cuda", dtype=torch.bfloat16)
        ws.fill_(0xFF)
        P.mopar_attention_cache(q[:t], out, cache, off, new, ln, n, ws=ws)
        s = seqs - 1
        k, v = (cache_rows(x.cpu(), table.cpu(), s, n) for x in (kc, vc))
        seen = torch.arange(n)[None] <= n - new + torch.arange(new)[:, None]
        ref, tol = attend(q[s * new:t], k, v, seen, d ** -0.5)
        check(out[s * new:], ref, tol, f"{seqs} sequences, {new} tokens")


def test_absent_pages_are_not_visible():
    for bad in (-1, 10 ** 9):
        over_cache(gen(5), "bf16", 4, 2, 64, 16, [300, 40], [3, 2], None, absent=(0, 4, bad))
    over_cache(gen(5), "f32", 2, 2, 64, 16, [10, 300], [1, 1], None, absent=(0, 0, -1))      # nothing left to see


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("page", [1, 16, 64])
@pytest.mark.parametrize("new", [1, 20, 40])
def test_absent_pages_take_no_weight(dt, page, new):
    """All scores zero: every visible token weighs the same, and absent ones nothing."""
    n = 200
    kc = torch.zeros(n // page + 1, 2, page, 64, device="cuda", dtype=DT[dt])
    vc = torch.ones_like(kc)
    table = torch.arange(-(-n // page), dtype=torch.int32).reshape(1, -1)
    table[0, 1::3] = -1
    table[0, 0] = 10 ** 6
    q = torch.ones(new, 4, 64, device="cuda", dtype=DT[dt])
    out = torch.empty_like(q)
    cache = P.PagedCache(kc, vc, table.cuda())
    P.mopar_attention_cache(q, out, cache, ints([0, new]), new, ints([n - new]), n, ws=P.alloc_attention_workspace(q, cache, new, n))
    # whole-number sums are exact; the reciprocal and the product round once each, by at most 2^-24
    assert bool(((out.double() - 1).abs() <= 2.0 ** -23).all())


def test_max_len_cuts_a_sequence():
    over_cache(gen(6), "bf16", 4, 2, 64, 16, [300, 40], [1, 1], None, max_len=200, poison=False)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_hidden_drafts_do_not_reach_a_row(dt):
    g = gen(7)
    heads, kv, d, page, past, n = 4, 2, 64, 16, 50, 20
    table, pages = page_table([past + n], page, g)
    kc, vc = (randn(g, pages, kv, page, d, dt=dt) for _ in range(2))
    q = randn(g, n, heads, d, dt=dt)
    seen = torch.eye(n, dtype=torch.bool)
    p, at = int(table[0, (past + 6) // page]), (past + 6) % page
    for value in (float("nan"), float("inf")):
        vc[p, :, at], kc[p, :, at] = value, value
        out = torch.empty_like(q)
        cache = P.PagedCache(kc, vc, table.cuda())
        P.mopar_attention_cache(q, out, cache, ints([0, n]), n, ints([past]), past + n, mask=pack_mask(seen, 1).cuda(),
                                ws=P.alloc_attention_workspace(q, cache, n, past + n))
        o = out.float().cpu()
        assert not bool(torch.isfinite(o[6]).all())
        o[6] = 0
        assert bool(torch.isfinite(o).all())


def tiny_weights(g, n, heads, kv, d, dt, at, peak):
    """Queries, keys and values of which key `peak` outweighs all others by e^300, so that their weights are 0 in float32;
    infinities and a NaN among the values at `at`, `at` + 1 and `at` + 2."""
    q = torch.ones(n, heads, d, device="cuda", dtype=DT[dt])
    k, v = randn(g, n, kv, d, dt="f32") * 0.1, randn(g, n, kv, d, dt=dt)
    k[peak] += 300.0 / d ** 0.5
    v[at, 0, 3], v[at + 1, 0, 4], v[at + 2, 0, 5] = float("inf"), float("-inf"), float("nan")
    v[at, 0, 6], v[at + 1, 0, 6] = float("inf"), float("-inf")
    return q, k.to(DT[dt]), v


def check_tiny_weights(out, q, k, v, seen):
    """Results of finite values against the plain form with zeros for the others, whose error is bounded by that of each
    weighted value (the sum of |p v|); where a row sees values that are not finite, their sum."""
    off = ~torch.isfinite(v)
    ref, tol = attend(q, k, torch.where(off, torch.zeros_like(v), v), seen, q.shape[2] ** -0.5)
    heads = q.shape[1] // v.shape[1]
    for j, h, i in torch.nonzero(off.cpu()).tolist():
        for row in torch.nonzero(seen[:, j])[:, 0].tolist():
            for x in range(h * heads, (h + 1) * heads):
                ref[row, x, i] += v[j, h, i].item()
    assert not bool(torch.isfinite(ref).all())
    check(out, ref, tol)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("at,peak", [(5, 150), (5, 9), (100, 20), (250, 290), (290, 200)])
def test_prompt_infinities_of_tiny_weight(dt, at, peak):
    """In whole and partly hidden tiles, before and after the peak: they reach the rows that see them."""
    q, k, v = tiny_weights(gen(20), 300, 4, 1, 64, dt, at, peak)
    check_tiny_weights(prompt(q, k, v, [300]), q, k, v, causal(300))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("new,heads", [(1, 2), (20, 2), (40, 8)])
@pytest.mark.parametrize("n,at,peak", [(60, 5, 55), (300, 5, 150), (300, 290, 100), (4000, 5, 3990), (4000, 3000, 3), (4000, 3990, 2000)])
def test_cache_infinities_of_tiny_weight(dt, new, heads, n, at, peak):
    """The same over a cache: tiles of every size, a unit by one block and shared by many."""
    page, d = 16, 64
    g = gen(21)
    q, k, v = tiny_weights(g, n, heads, 1, d, dt, at, peak)
    table, pages = page_table([n], page, g)
    kc, vc = (torch.full((pages, 1, page, d), float("nan"), device="cuda", dtype=DT[dt]) for _ in range(2))
    cache = P.PagedCache(kc, vc, table.cuda())
    P.mopar_cache_append(cache, k, v, ints([0] * n), torch.arange(n, dtype=torch.int32, device="cuda"))
    out = torch.empty(new, heads, d, device="cuda", dtype=DT[dt])
    P.mopar_attention_cache(q[:new], out, cache, ints([0, new]), new, ints([n - new]), n, ws=P.alloc_attention_workspace(q[:new], cache, new, n))
    seen = torch.arange(n)[None] <= n - new + torch.arange(new)[:, None]
    check_tiny_weights(out, q[:new], k, v, seen)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 20])
@pytest.mark.parametrize("n,at", [(60, 7), (4000, 7), (4000, 2500)])
def test_cache_infinite_scores(dt, new, n, at):
    """A score of +infinity or NaN makes NaN of its row, also where it is in one of many parts; one of -infinity has no weight."""
    page, d = 16, 64
    g = gen(22)
    table, pages = page_table([n], page, g)
    kc, vc = (randn(g, pages, 3, page, d, dt=dt) for _ in range(2))
    q = torch.ones(new, 6, d, device="cuda", dtype=DT[dt])
    p = int(table[0, at // page])
    kc[p, 0, at % page, 5], kc[p, 1, at % page, 5], kc[p, 2, at % page, 5] = float("inf"), float("nan"), float("-inf")
    cache = P.PagedCache(kc, vc, table.cuda())
    out = torch.empty(new, 6, d, device="cuda", dtype=DT[dt])
    P.mopar_attention_cache(q, out, cache, ints([0, new]), new, ints([n - new]), n, ws=P.alloc_attention_workspace(q, cache, new, n))
    assert bool(out[:, :4].isnan().all())
    k, v = (cache_rows(x.cpu(), table, 0, n)[:, 2:] for x in (kc, vc))
    seen = torch.arange(n)[None] <= n - new + torch.arange(new)[:, None]
    seen[:, at], k[at] = False, 0
    ref, tol = attend(q[:, 4:], k, v, seen, d ** -0.5)
    check(out[:, 4:], ref, tol)


def test_pools_past_32_bit_offsets():
    g = gen(8)
    kv, page, d, n = 8, 256, 128, 700
    pages = 17000                                            # 8.9 GB a pool
    kc, vc = (torch.zeros(pages, kv, page, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    table = ints([[pages - 1, 8193, pages - 2]])
    k, v = randn(g, n, kv, d), randn(g, n, kv, d)
    cache = P.PagedCache(kc, vc, table)
    P.mopar_cache_append(cache, k, v, ints([0] * n), torch.arange(n, dtype=torch.int32, device="cuda"))
    q = randn(g, 1, 16, d)
    out = torch.empty_like(q)
    P.mopar_attention_cache(q, out, cache, ints([0, 1]), 1, ints([n - 1]), n, ws=P.alloc_attention_workspace(q, cache, 1, n))
    ref, tol = attend(q, k, v, torch.ones(1, n, dtype=torch.bool), d ** -0.5)
    check(out, ref, tol)
    P.mopar_cache_keep(cache, ints([200]), ints([0, 1]), ints([499]), 1)
    assert torch.equal(kc[pages - 1, :, 200], k[699]) and torch.equal(vc[pages - 1, :, 200], v[699])


def test_more_pages_of_heads_than_32_bits_count():
    g = gen(11)
    kv, d, pages = 65536, 8, 32770                           # 34 GB a pool, of pages of one token
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("80 GB of memory")
    kc, vc = (torch.empty(pages, kv, 1, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    cache = P.PagedCache(kc, vc, ints([[5, pages - 1, 16385, pages - 2]]))
    k, v = randn(g, 4, kv, d), randn(g, 4, kv, d)
    P.mopar_cache_append(cache, k, v, ints([0] * 4), ints([0, 1, 2, 3]))
    for i, page in enumerate((5, pages - 1, 16385, pages - 2)):
        assert torch.equal(kc[page, :, 0], k[i]) and torch.equal(vc[page, :, 0], v[i])
    P.mopar_cache_keep(cache, ints([0]), ints([0, 2]), ints([1, 3]), 2)
    assert torch.equal(kc[5, :, 0], k[1]) and torch.equal(vc[pages - 1, :, 0], v[3])
    del cache, kc, vc
    torch.cuda.empty_cache()


def test_append_without_sequences_turns_queries():
    g = gen(12)
    pool = randn(g, 4, 2, 16, 64)
    before, q, k = pool.clone(), randn(g, 3, 4, 64), randn(g, 3, 2, 64)
    out, want = torch.empty_like(q), torch.empty_like(q)
    cache = P.PagedCache(pool, pool.clone(), torch.empty(0, 2, device="cuda", dtype=torch.int32))
    rot, pos = P.Rotary(64), ints([4, 5, 6])
    P.mopar_cache_append(cache, k, k, ints([0, 0, -1]), ints([0, 1, 2]), rotary=rot, pos=pos, q=q, q_out=out)
    P.mopar_rotary_apply(rot, q, want, pos)
    assert torch.equal(out, want) and torch.equal(pool, before)


@pytest.mark.parametrize("dt,lens,new", [("bf16", [500, 7], [1, 9]), ("f32", [500, 2 ** 31 - 1], [3, 1]), ("bf16", [2 ** 31 - 1, 3], [64, 64])])
def test_a_limit_past_every_slot(dt, lens, new):
    """max_len 2^31 - 1 and lengths to match: a sequence ends with its table's slots."""
    g = gen(13)
    heads, kv, d, page, slots = 4, 2, 64, 16, 640
    table = torch.randperm(2 * slots // page, generator=g, dtype=torch.int32).view(2, -1).cuda()
    kc, vc = (randn(g, 2 * slots // page, kv, page, d, dt=dt) for _ in range(2))
    cache, t, top = P.PagedCache(kc, vc, table), sum(new), max(new)
    q = randn(g, t, heads, d, dt=dt)
    out = torch.empty_like(q)
    most = 2 ** 31 - 1
    P.mopar_attention_cache(q, out, cache, ints([0, new[0], t]), top, ints(lens), most, ws=P.alloc_attention_workspace(q, cache, top, most))
    for s, (lo, n) in enumerate(zip((0, new[0]), new)):
        total = min(lens[s] + n, slots)
        seen = torch.arange(total)[None] <= min(lens[s], slots) + torch.arange(n)[:, None]
        k, v = (cache_rows(x.cpu(), table.cpu(), s, total) for x in (kc, vc))
        ref, tol = attend(q[lo:lo + n], k, v, seen, d ** -0.5)
        check(out[lo:lo + n], ref, tol, f"sequence {s}")


def test_streams_and_graphs():
    """Every call on a stream of its own, captured, and replayed over changed inputs with eager work between."""
    g = gen(9)
    heads, kv, d, page, n = 8, 2, 128, 16, 6
    lens = [700, 33]
    table, pages = page_table([x + n for x in lens], page, g)
    kc, vc = (randn(g, pages, kv, page, d) for _ in range(2))
    cache = P.PagedCache(kc, vc, table.cuda())
    rows = randn(g, 2 * n, heads + 2 * kv, d)
    q, k, v = rows[:, :heads], rows[:, heads:heads + kv], rows[:, heads + kv:]
    q_out, out, pout = (torch.zeros(2 * n, heads, d, device="cuda", dtype=torch.bfloat16) for _ in range(3))
    slot = ints([lens[s] + i for s in range(2) for i in range(n)])
    seq, off, ln = ints([0] * n + [1] * n), ints([0, n, 2 * n]), ints(lens)
    poff, path = ints([0, 2, 3]), ints([1, 4, 3])
    rot = P.Rotary(d)
    ws = P.alloc_attention_workspace(q, cache, n, 706)

    def step():
        P.mopar_cache_append(cache, k, v, seq, slot, rotary=rot, pos=slot, q=q, q_out=q_out)
        P.mopar_attention_cache(q_out, out, cache, off, n, ln, 706, ws=ws)
        P.mopar_attention_prompt(q_out, k, v, pout, off, n)
        P.mopar_cache_keep(cache, ln, poff, path, 2)
        return [t.clone() for t in (q_out, out, pout, kc, vc)]

    pools = kc.clone(), vc.clone()
    inputs = [rows.clone(), randn(g, *rows.shape), randn(g, *rows.shape)]
    want = []
    for x in inputs:
        kc.copy_(pools[0]), vc.copy_(pools[1]), rows.copy_(x)
        want.append(step())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        kc.copy_(pools[0]), vc.copy_(pools[1]), rows.copy_(inputs[0])
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[0]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.mopar_cache_append(cache, k, v, seq, slot, rotary=rot, pos=slot, q=q, q_out=q_out)
        P.mopar_attention_cache(q_out, out, cache, off, n, ln, 706, ws=ws)
        P.mopar_attention_prompt(q_out, k, v, pout, off, n)
        P.mopar_cache_keep(cache, ln, poff, path, 2)
    for i in (1, 2, 0, 2):
        kc.copy_(pools[0]), vc.copy_(pools[1]), rows.copy_(inputs[i])
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((q_out, out, pout, kc, vc), want[i]))
        (rows * 2).sum().item()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_run_of_them_together(dt):
    """Prompts attended and stored, a tree drafted and attended, its accepted path kept, then single tokens: every
    result equals causal attention over the tokens the sequence has by then."""
    g = gen(11)
    heads, kv, d, page, prompts, drafts, steps = 4, 2, 64, 8, [37, 5, 90], 12, 3
    rot = P.Rotary(d, layout="interleaved", scaling="linear", factor=2.0)
    total = [n + drafts + steps for n in prompts]
    table, pages = page_table(total, page, g)
    kc, vc = (torch.full((pages, kv, page, d), float("nan"), device="cuda", dtype=DT[dt]) for _ in range(2))
    cache = P.PagedCache(kc, vc, table.cuda())
    keys, vals = [torch.empty(0, kv, d, dtype=DT[dt], device="cuda") for _ in prompts], [torch.empty(0, kv, d, dtype=DT[dt], device="cuda") for _ in prompts]

    def rows(t):
        r = randn(g, t, heads + 2 * kv, d, dt=dt)
        return r[:, :heads], r[:, heads:heads + kv], r[:, heads + kv:]

    # prompts
    t = sum(prompts)
    q, k, v = rows(t)
    seq = ints([s for s, n in enumerate(prompts) for _ in range(n)])
    pos = ints([i for n in prompts for i in range(n)])
    off = ints([0, 37, 42, 132])
    qr, kr, out = torch.empty_like(q), torch.empty(t, kv, d, device="cuda", dtype=DT[dt]), torch.empty(t, heads, d, device="cuda", dtype=DT[dt])
    P.mopar_cache_append(cache, k, v, seq, pos, rotary=rot, pos=pos, q=q, q_out=qr)
    P.mopar_rotary_apply(rot, k, kr, pos)
    P.mopar_attention_prompt(qr, kr, v, out, off, 90)
    at = 0
    for s, n in enumerate(prompts):
        keys[s], vals[s] = kr[at:at + n], v[at:at + n]
        ref, tol = attend(qr[at:at + n], keys[s], vals[s], causal(n), d ** -0.5)
        check(out[at:at + n], ref, tol, "prompt")
        at += n
    # a tree of drafts: token i at depth of its ancestors
    anc, bits = tree_mask(drafts, g)
    depth = anc.sum(1) - 1
    q, k, v = rows(3 * drafts)
    seq = ints([s for s in range(3) for _ in range(drafts)])
    slot = ints([n + i for n in prompts for i in range(drafts)])
    pos = ints([n + int(x) for n in prompts for x in depth])
    qr, kr, out = torch.empty_like(q), torch.empty(3 * drafts, kv, d, device="cuda", dtype=DT[dt]), torch.empty(3 * drafts, heads, d, device="cuda", dtype=DT[dt])
    P.mopar_cache_append(cache, k, v, seq, slot, rotary=rot, pos=pos, q=q, q_out=qr)
    P.mopar_rotary_apply(rot, k, kr, pos)
    lens = ints(prompts)
    ws = P.alloc_attention_workspace(qr, cache, drafts, max(total))
    P.mopar_attention_cache(qr, out, cache, ints([0, drafts, 2 * drafts, 3 * drafts]), drafts, lens, max(total),
                            mask=bits.repeat(3, 1).cuda(), ws=ws)
    paths = []
    for s, n in enumerate(prompts):
        lo = s * drafts
        path = [int(j) for j in torch.nonzero(anc[drafts - 1 - 4 * s])[:, 0]]
        paths.append(path)
        kk, vv = torch.cat([keys[s], kr[lo:lo + drafts]]), torch.cat([vals[s], v[lo:lo + drafts]])
        ref, tol = attend(qr[lo:lo + drafts], kk, vv, torch.cat([torch.ones(drafts, n, dtype=torch.bool), anc], 1), d ** -0.5)
        check(out[lo:lo + drafts], ref, tol, "tree")
        keys[s], vals[s] = torch.cat([keys[s], kr[lo:lo + drafts][path]]), torch.cat([vals[s], v[lo:lo + drafts][path]])
    poff = [0]
    for p in paths:
        poff.append(poff[-1] + len(p))
    P.mopar_cache_keep(cache, lens, ints(poff), ints([i for p in paths for i in p]), drafts)
    now = [n + len(p) for n, p in zip(prompts, paths)]
    for _ in range(steps):
        q, k, v = rows(3)
        pos, qr, out = ints(now), torch.empty(3, heads, d, device="cuda", dtype=DT[dt]), torch.empty(3, heads, d, device="cuda", dtype=DT[dt])
        kr = torch.empty(3, kv, d, device="cuda", dtype=DT[dt])
        P.mopar_cache_append(cache, k, v, ints([0, 1, 2]), pos, rotary=rot, pos=pos, q=q, q_out=qr)
        P.mopar_rotary_apply(rot, k, kr, pos)
        P.mopar_attention_cache(qr, out, cache, ints([0, 1, 2, 3]), 1, pos, max(total), ws=ws)
        for s in range(3):
            keys[s], vals[s] = torch.cat([keys[s], kr[s:s + 1]]), torch.cat([vals[s], v[s:s + 1]])
            ref, tol = attend(qr[s:s + 1], keys[s], vals[s], torch.ones(1, now[s] + 1, dtype=torch.bool), d ** -0.5)
            check(out[s:s + 1], ref, tol, "single token")
        now = [n + 1 for n in now]
