"""A decoder's steps in 8 bits on the GPU against plain float64 forms: the norm, rows to 8 bits, their products, log
probabilities, and a run of them together with the cache."""
import math

import pytest
import torch

import paper_2404_02445_amd as P
from tests import decoder_ref as R
from tests.decoder_ref import U, check

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, dt="bf16", by=1.0):
    return (torch.randn(shape, generator=g) * by).to(DT[dt]).cuda()


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def marked(rows, width):
    """8-bit rows to be written, with marks in all that must stay: the ends of rows, a row before and one behind."""
    stride = (width + 15) // 16 * 16 + 16
    q = torch.full((rows + 2, stride), 99, dtype=torch.int8, device="cuda")
    s = torch.full((rows,), 99.0, device="cuda")
    return q, P.Rows8(q[1:rows + 1, :width], s)


def check_marks(q, width):
    assert bool((q[0] == 99).all() and (q[-1] == 99).all() and (q[:, width:] == 99).all()), "bytes past the rows were written"


def check_scales(got, want, tol):
    check(got, want, want.abs().nan_to_num(0.0) * tol + 1e-45)


# --- norm ------------------------------------------------------------------------------------------

NORM_SIZES = [(1, 1), (3, 7), (5, 8), (2, 511), (4, 512), (3, 520), (2, 2047), (9, 2048), (2, 2056), (5, 4096), (1, 4104), (3, 8192), (2, 8200),
              (2, 16391), (1, 32768), (3, 32776), (2, 70001)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,width", NORM_SIZES)
@pytest.mark.parametrize("residual", [False, True])
def test_norm(dt, tokens, width, residual):
    g = gen(tokens * 31 + width)
    x, w = randn(g, tokens, width, dt=dt), randn(g, width, dt=dt)
    x[:, ::5] *= 30
    res = randn(g, tokens, width, dt=dt) if residual else None
    total = torch.full_like(x, 7.0) if residual else None
    out = torch.full_like(x, 7.0)
    q, out8 = marked(tokens, width)
    P.mopar_rms_norm(x, w, 1e-5, residual=res, total=total, out=out, out8=out8)
    h, want, tol, steps, scales = R.norm(x, w, 1e-5, res)
    check(out, want, tol)
    if residual:
        assert torch.equal(total.cpu(), h)
    assert torch.equal(out8.values.cpu(), steps)
    check_scales(out8.scales, scales, R.sum_bound(width) + 8 * U)
    check_marks(q, width)
    # one output at a time: the same bits
    alone, only8 = torch.full_like(x, 7.0), marked(tokens, width)[1]
    P.mopar_rms_norm(x, w, 1e-5, residual=res, out=alone)
    P.mopar_rms_norm(x, w, 1e-5, residual=res, out8=only8)
    assert torch.equal(alone, out) and torch.equal(only8.values, out8.values) and torch.equal(only8.scales, out8.scales)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("width", [40, 5000, 33000])
@pytest.mark.parametrize("which", ["total is x", "total is residual", "out is x", "out is residual", "both"])
def test_norm_in_place(dt, width, which):
    g = gen(width)
    x, res, w = randn(g, 4, width, dt=dt), randn(g, 4, width, dt=dt), randn(g, width, dt=dt)
    want_t, want, want8 = torch.empty_like(x), torch.empty_like(x), P.alloc_rows8(4, width, "cuda")
    P.mopar_rms_norm(x, w, residual=res, total=want_t, out=want, out8=want8)
    a, b, t, o = x.clone(), res.clone(), torch.empty_like(x), torch.empty_like(x)
    total, out = {"total is x": (a, o), "total is residual": (b, o), "out is x": (None, a), "out is residual": (None, b), "both": (a, b)}[which]
    got8 = P.alloc_rows8(4, width, "cuda")
    P.mopar_rms_norm(a, w, residual=b, total=total, out=out, out8=got8)
    assert torch.equal(out, want) and (total is None or torch.equal(total, want_t))
    assert torch.equal(got8.values, want8.values) and torch.equal(got8.scales, want8.scales)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_norm_strides_and_alignment(dt):
    """Rows off every vector width, inside wider ones, and one row for all."""
    g = gen(5)
    wide = randn(g, 6, 731, dt=dt)
    x, res, w = wide[:, 3:360], randn(g, 1, 357, dt=dt).expand(6, 357), randn(g, 358, dt=dt)[1:]
    room = torch.full((6, 800), 7.0, device="cuda", dtype=DT[dt])
    out, total = room[:, 5:362], room[:, 401:758]
    out8 = P.alloc_rows8(6, 357, "cuda")
    P.mopar_rms_norm(x, w, 1e-5, residual=res, total=total, out=out, out8=out8)
    h, want, tol, steps, scales = R.norm(x, w, 1e-5, res)
    check(out, want, tol)
    assert torch.equal(total.cpu(), h) and torch.equal(out8.values.cpu(), steps)
    assert bool((room[:, :5] == 7).all() and (room[:, 362:401] == 7).all() and (room[:, 758:] == 7).all())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_norm_rows_that_are_odd(dt):
    """Zeros, infinities, NaN and subnormals stay in their rows."""
    g = gen(6)
    x, w = randn(g, 7, 300, dt=dt), randn(g, 300, dt=dt)
    x[0], x[1, 17], x[2, 299], x[3, 0], x[5] = 0, math.inf, math.nan, -math.inf, 1e-38
    out, out8 = torch.empty_like(x), P.alloc_rows8(7, 300, "cuda")
    P.mopar_rms_norm(x, w, 1e-5, out=out, out8=out8)
    h, want, tol, steps, scales = R.norm(x, w, 1e-5)
    assert torch.equal(out8.values.cpu(), steps)
    check_scales(out8.scales, scales, R.sum_bound(300) + 8 * U)
    for r in (0, 4, 5, 6):
        check(out[r], want[r], tol[r] + 1e-38)
    assert float(out8.scales[0]) == 0 and bool(out8.scales[1:4].isnan().all()) and not bool(out[2].isfinite().any())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_norm_of_zeros_without_eps(dt):
    """A row of zeros has scale 0 where its factor is infinite, too; others do without eps."""
    g = gen(16)
    x, w = randn(g, 3, 300, dt=dt), randn(g, 300, dt=dt)
    x[1] = 0
    out8 = P.alloc_rows8(3, 300, "cuda")
    P.mopar_rms_norm(x, w, 0.0, out8=out8)
    steps = R.steps(x.cpu().double() * w.cpu().double())[0]
    scales = R.norm(x[::2], w, 0.0)[4]
    assert torch.equal(out8.values.cpu(), steps) and float(out8.scales[1]) == 0
    check_scales(out8.scales[::2], scales, R.sum_bound(300) + 8 * U)


def test_norm_steps_at_their_borders():
    """Values in the middle between two steps, and next to it: halves to even, as 64-bit arithmetic rounds them."""
    k = torch.arange(-127, 127, dtype=torch.float64)
    middle = (2 * k + 1) / 2                                        # times 1: the row's largest is 127
    for dt in (torch.float32, torch.bfloat16):
        x = torch.cat([torch.tensor([127.0]), middle, torch.zeros(1)]).to(dt)
        rows = torch.stack([x, x * 0.5, x * 2 ** -20, torch.where(x.abs() < 127, x * (1 + 2.0 ** -7), x), torch.where(x.abs() < 127, x * (1 - 2.0 ** -8), x)])
        rows = rows.clamp(-127, 127).to(dt).cuda()
        out8 = P.alloc_rows8(rows.shape[0], rows.shape[1], "cuda")
        for weight in (torch.ones(rows.shape[1], dtype=dt, device="cuda"), torch.full((rows.shape[1],), 0.375, dtype=dt, device="cuda")):
            P.mopar_rms_norm(rows, weight, out8=out8)
            assert torch.equal(out8.values.cpu(), R.steps(rows.cpu().double() * weight.cpu().double())[0])
        P.mopar_quantize_rows(rows, out8)
        assert torch.equal(out8.values.cpu(), R.steps(rows.cpu().double())[0])


# --- rows to 8 bits ----------------------------------------------------------------------------------

@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "silu", "gelu"])
@pytest.mark.parametrize("tokens,width", [(1, 1), (3, 9), (5, 512), (700, 1021), (2, 2048), (3, 4100), (2, 8192), (4, 14336), (2, 32768), (2, 40003)])
def test_quantize(dt, act, tokens, width):
    g = gen(tokens + width)
    rows = randn(g, tokens, 2 * width, dt=dt, by=3.0)
    gate, x = rows[:, :width], rows[:, width:]
    q, out8 = marked(tokens, width)
    P.mopar_quantize_rows(x, out8, gate=None if act == "none" else gate, act=act)
    steps, top = R.steps(R.gated(x, gate, act))
    assert torch.equal(out8.values.cpu(), steps)
    check_scales(out8.scales, top / 127, 2.02 * U)
    check_marks(q, width)
    check(out8.dequantized(), steps.double() * (top / 127)[:, None], steps.double().abs() * (top / 127)[:, None] * 4 * U + 1e-45)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_quantize_far_gates(dt, act):
    """Gates that pass all, nothing, or far down the activation's tail; rows of one sign; infinities and NaN."""
    g = gen(8)
    x, gate = randn(g, 10, 600, dt=dt), randn(g, 10, 600, dt=dt)
    gate[0], gate[1], gate[2], gate[3] = 300.0, -300.0, gate[2].abs() * -3, gate[3].abs() * -1 - 4
    gate[4, ::2], gate[5, 3], gate[6, 4], gate[7, 5], x[8, 6] = -8.0, math.inf, -math.inf, math.nan, math.inf
    gate[9] = 3e38
    x[9] = x[9].clamp(-1, 1) * 0.5
    out8 = P.alloc_rows8(10, 600, "cuda")
    P.mopar_quantize_rows(x, out8, gate=gate, act=act)
    p = R.gated(x, gate, act)
    p[6, 4] = math.nan                                               # (0 times infinity in either form)
    steps, top = R.steps(p)
    some = top.isnan() | (top > 1e-36)                                 # below: no weight in float32
    assert torch.equal(out8.values.cpu()[some], steps[some])
    check_scales(out8.scales[some.cuda()], top[some] / 127, 2.02 * U)
    assert bool((out8.dequantized().cpu()[~some].abs() < 1e-35).all()) and int((~some).sum()) == 1
    assert bool(out8.scales[5:9].isnan().all())


def test_more_rows_than_a_launch_takes():
    """2^24 rows and some: the rows of a launch's end and of the next."""
    rows = (1 << 24) + 1000
    x = (torch.arange(rows, device="cuda", dtype=torch.int32) % 251 - 125).float()[:, None]
    x = torch.cat([x, torch.full_like(x, 127)], 1)
    out8 = P.alloc_rows8(rows, 2, "cuda")
    out8.values.fill_(3)
    P.mopar_quantize_rows(x, out8)
    assert torch.equal(out8.values.float(), x) and bool((out8.scales == 1).all())
    out = torch.empty_like(x)
    P.mopar_rms_norm(x, torch.ones(2, device="cuda"), out=out)
    r = 1 / torch.sqrt(x.double().square().mean(1, keepdim=True) + 1e-6)
    assert bool(((out.double() - x * r).abs() <= (x * r).abs() * (R.sum_bound(2) + 9 * U)).all())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("width", [600, 33000])
def test_quantize_gates_beyond_float32(dt, act, width):
    """Gates of the type's lowest value, and products of an activation that float32 hardly holds with a value near its largest."""
    g = gen(9)
    x = randn(g, 6, width, dt=dt).clamp(-3, 3)
    gate = torch.zeros_like(x)
    gate[0], gate[0, 7:9] = torch.finfo(gate.dtype).min, 1.5
    x[1], gate[1] = x[1] * 1e38, -100.0 if act == "silu" else -9.0
    gate[2], x[2], x[2, 1] = -95.0 if act == "silu" else -13.0, x[2] * 1e-3, 1e37
    x[3], gate[3] = x[3] * 1e30, randn(g, 1, width, dt=dt)[0] - (88.0 if act == "silu" else 12.0)
    gate[4], gate[4, 5], x[4, 5] = torch.finfo(gate.dtype).min, -12.0, 1e38
    gate[5] = torch.finfo(gate.dtype).min
    out8 = P.alloc_rows8(6, width, "cuda")
    P.mopar_quantize_rows(x, out8, gate=gate, act=act)
    steps, top = R.steps(R.gated(x, gate, act))
    assert torch.equal(out8.values.cpu(), steps)
    check(out8.scales, top / 127, top / 127 * 2.02 * U + 1e-38)


def test_quantize_small_and_large_rows():
    """Rows at both ends of float32."""
    x = torch.tensor([[1e-38, -3e-39, 0.0], [1e-44, 7e-45, -1e-45], [3.3e38, -1e38, 1.0], [1e-31, 5e-32, 2e-33], [0.0, -0.0, 0.0]], device="cuda")
    out8 = P.alloc_rows8(5, 3, "cuda")
    P.mopar_quantize_rows(x, out8)
    steps, top = R.steps(x.cpu().double())
    assert torch.equal(out8.values.cpu(), steps)
    check(out8.scales, top / 127, top / 127 * 1.01 * U + 1e-45)


# --- products ----------------------------------------------------------------------------------------

def rows8(g, rows, width, extra=0):
    """Random 8-bit rows whose spare bytes are not zero."""
    q = torch.randint(-128, 128, (rows, (width + 15) // 16 * 16 + extra), generator=g, dtype=torch.int8).cuda()
    return P.Rows8(q[:, :width], (torch.rand(rows, generator=g) * 0.01).cuda())


LINEAR_SIZES = [(1, 1, 1), (1, 16, 16), (2, 5, 33), (1, 4096, 4096), (3, 100, 1000), (5, 64, 127), (16, 48, 128), (17, 300, 129), (33, 77, 4111), (64, 512, 14336),
                (64, 65, 640), (65, 129, 2000), (100, 1000, 333), (128, 128, 256), (129, 257, 511), (200, 2051, 1001), (256, 512, 1024),
                (300, 300, 16), (512, 1024, 384), (777, 640, 4096), (1024, 1536, 512), (2000, 31, 700), (2048, 2304, 768), (31, 20000, 513), (1300, 2600, 144)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", LINEAR_SIZES)
def test_linear(dt, m, n, k):
    g = gen(m + n + k)
    x, w = rows8(g, m, k), rows8(g, n, k, extra=32)
    bias = randn(g, n, dt=dt) if (m + n + k) % 2 else None
    out = torch.full((m, n), 7.0, device="cuda", dtype=DT[dt])
    P.mopar_linear8(x, w, out, bias=bias)
    want, tol = R.linear((x.values, x.scales), (w.values, w.scales), DT[dt], bias)
    check(out, want, tol)
    shared = torch.full((m, n), 7.0, device="cuda", dtype=DT[dt])
    P.mopar_linear8(x, w, shared, bias=bias, ws=P.alloc_linear8_workspace(x, w, out))
    assert torch.equal(out, shared)


def linear_on_gpu(x, w, bias, dt):
    """The reference of large products (float64 on the GPU)."""
    y = x.values.double() @ w.values.double().t().contiguous() * x.scales.double()[:, None] * w.scales.double()[None]
    tol = y.abs() * 4 * U
    if bias is not None:
        y = y + bias.double()
        tol += y.abs() * U
    return y, tol * 1.01 + y.abs() * R.HALF_STEP[DT[dt]] * 1.01


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(3100, 3504, 272), (3101, 3503, 513), (4096, 2304, 1031), (8000, 9000, 384), (300, 40001, 520), (1500, 1600, 700), (1537, 1603, 257),
                                   (2100, 2200, 400), (128, 24000, 1008), (70, 30011, 330), (5000, 5000, 301)])
def test_linear_large(dt, m, n, k):
    """Tiles of 256 and 128, several a block; sums that end inside a step and inside a chunk; edges of tiles in both directions."""
    g = gen(m + n + k)
    x, w = rows8(g, m, k, extra=16), rows8(g, n, k)
    bias = randn(g, n, dt=dt) if k % 2 else None
    out = torch.full((m, n), 7.0, device="cuda", dtype=DT[dt])
    P.mopar_linear8(x, w, out, bias=bias)
    want, tol = linear_on_gpu(x, w, bias, dt)
    assert bool(((out.double() - want).abs() <= tol).all())
    again = torch.full((m + 2, n + 24), 7.0, device="cuda", dtype=DT[dt])          # inside wider rows, on and off 16 bytes
    for at in (8, 3):
        again.fill_(7.0)
        P.mopar_linear8(x, w, again[1:m + 1, at:at + n], bias=bias)
        assert torch.equal(again[1:m + 1, at:at + n], out)
        again[1:m + 1, at:at + n] = 7.0
        assert bool((again == 7).all())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(3, 37, 100), (70, 135, 272), (300, 517, 1040), (1030, 1043, 2064)])
def test_linear_strides_and_alignment(dt, m, n, k):
    """Results inside wider rows, off every vector width; nothing beside them is written."""
    g = gen(m)
    x, w, bias = rows8(g, m, k, extra=48), rows8(g, n, k), randn(g, n + 1, dt=dt)[1:]
    room = torch.full((m + 2, n + 6), 7.0, device="cuda", dtype=DT[dt])
    ws = P.alloc_linear8_workspace(x, w, room)
    for at in (1, 3, 4):
        room.fill_(7.0)
        out = room[1:m + 1, at:at + n]
        P.mopar_linear8(x, w, out, bias=bias, ws=ws)
        want, tol = R.linear((x.values, x.scales), (w.values, w.scales), DT[dt], bias)
        check(out, want, tol)
        assert bool((room[0] == 7).all() and (room[-1] == 7).all() and (room[:, :at] == 7).all() and (room[:, at + n:] == 7).all())


def test_linear_largest_sums():
    """131071 products of -128 and -128: the largest sum that 32 bits hold; scales at their ends, NaN and 0 among them."""
    k = 131071
    stride = 131072
    q = torch.full((20, stride), -128, dtype=torch.int8, device="cuda")
    s = torch.tensor([1.0, 0.0, math.nan, math.inf, 1e-30] * 4, device="cuda")
    x = P.Rows8(q[:, :k], s)
    w = P.Rows8(q[:7, :k], torch.ones(7, device="cuda"))
    out = torch.empty(20, 7, device="cuda")
    for ws in (None, P.alloc_linear8_workspace(x, w, out)):
        out.fill_(7.0)
        P.mopar_linear8(x, w, out, ws=ws)
        want = (torch.full((20, 7), 128.0 * 128 * k, dtype=torch.float64) * s.cpu().double()[:, None])
        check(out, want, want.abs().nan_to_num(0.0, 0.0) * 4 * U)


def test_linear_rows_behind_the_last_are_left():
    g = gen(12)
    x, w = rows8(g, 40, 256), rows8(g, 70, 256)
    room = torch.full((64, 70), 7.0, device="cuda", dtype=torch.bfloat16)
    few = P.Rows8(x.values[:9], x.scales[:9])
    P.mopar_linear8(few, w, room[:9])
    assert bool((room[9:] == 7).all())
    P.mopar_linear8(P.Rows8(x.values[:0], x.scales[:0]), w, room[:0])          # nothing to do


# --- log probabilities ---------------------------------------------------------------------------------

def check_logprobs(x, tokens, scale=1.0, top=0):
    rows, vocab = x.shape
    ref = R.logprobs(x, tokens, scale, top)
    for space in (None, P.alloc_token_logprobs_workspace(x, top)):
        lp, en = torch.full((rows,), 7.0, device="cuda"), torch.full((rows,), 7.0, device="cuda")
        rank = torch.full((rows,), 7, device="cuda", dtype=torch.int32)
        tl = torch.full((rows, top), 7.0, device="cuda") if top else None
        ti = torch.full((rows, top), 7, device="cuda", dtype=torch.int32) if top else None
        P.mopar_token_logprobs(x, tokens, lp, entropy=en, rank=rank, top_logprob=tl, top_id=ti, scale=scale, ws=space)
        assert torch.equal(rank.cpu().long(), ref["rank"])
        check(lp, ref["logprob"], ref["logprob_tol"], "logprob")
        check(en, ref["entropy"], torch.full_like(ref["entropy"], ref["entropy_tol"]), "entropy")
        if top:
            assert torch.equal(ti.cpu().long(), ref["top_id"])
            check(tl, ref["top_logprob"], ref["top_tol"], "alternatives")
        # optional outputs left out: the same bits
        alone = torch.full((rows,), 7.0, device="cuda")
        P.mopar_token_logprobs(x, tokens, alone, scale=scale, ws=space)
        assert torch.equal(alone.isnan(), lp.isnan()) and torch.equal(alone.nan_to_num(), lp.nan_to_num())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (3, 2, 2), (5, 7, 0), (4, 63, 63), (2, 64, 64), (3, 65, 20), (2, 511, 5), (7, 513, 1), (2, 2049, 64), (40, 5000, 5),
                                            (1, 32003, 20), (3, 50000, 64), (600, 4099, 3), (1, 131072, 0), (4, 128000, 20), (1100, 700, 2)])
def test_logprobs(dt, rows, vocab, top):
    g = gen(rows + vocab)
    x = randn(g, rows, vocab, dt=dt, by=3.0)
    tokens = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32).cuda()
    tokens[::2] = x[::2].argmax(1).int()
    check_logprobs(x, tokens, top=top)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,top", [(5, 8192, 64), (257, 3001, 7), (300, 32768, 5), (300, 33001, 64), (513, 40000, 3), (1023, 1000, 0), (9, 65536, 64), (20, 70001, 20),
                                            (60, 66001, 0), (128, 65536, 64), (129, 65536, 1), (33, 65537, 33)])
def test_logprobs_of_many_rows_and_long_ones(dt, rows, vocab, top):
    """Each choice of waves and shares, ties and rows without weight among them."""
    g = gen(rows + vocab)
    x = randn(g, rows, vocab, dt=dt, by=2.0)
    x[1::7] = (x[1::7] * 2).round()
    x[2::11] = x[2::11].sort(1).values
    x[3::13, : vocab - 3] = -math.inf
    x[4] = -math.inf
    tokens = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32).cuda()
    check_logprobs(x, tokens, top=top)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("order", ["ascending", "descending", "equal", "two values", "last lane"])
def test_logprobs_orders(dt, order):
    """Rows that a list of alternatives meets in the worst order, and ties, which go to the lowest index."""
    vocab = 9001
    x = torch.linspace(-8, 8, vocab).repeat(3, 1)
    if order == "descending":
        x = x.flip(1)
    if order == "equal":
        x[:] = 0.25
    if order == "two values":
        x = (torch.arange(vocab) % 37 == 5).float().repeat(3, 1)
    if order == "last lane":
        x = torch.where(torch.arange(vocab) % 512 >= 504, x, -9.0)
    x = x.to(DT[dt]).cuda()
    for top in (1, 20, 64):
        check_logprobs(x, ints([0, 5, vocab - 1]), top=top)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_logprobs_masks(dt):
    """-infinity and the type's lowest value as masks, rows that they leave empty, infinities, NaN, zeros of both signs, tokens of padding."""
    g = gen(4)
    vocab, low = 5003, torch.finfo(DT[dt]).min
    x = randn(g, 16, vocab, dt=dt)
    x[0, 10:], x[1, :-1], x[2], x[3] = -math.inf, -math.inf, -math.inf, low
    x[4, ::2], x[5, 100:] = low, low
    x[6, 77], x[7, 5], x[8], x[9, 3], x[10, 4] = math.inf, math.nan, math.nan, -math.inf, -math.nan
    x[11], x[12, 1:] = torch.where(torch.arange(vocab) % 2 == 0, -0.0, 0.0).to(DT[dt]).cuda(), math.nan
    x[13] *= 1e30
    tokens = ints([3, 3, 3, 3, 4, 5000, 9, 9, 9, 3, 9, 9, 0, 9, -1, vocab])
    check_logprobs(x, tokens, top=8)
    check_logprobs(x, tokens, top=0)


@pytest.mark.parametrize("scale", [0.01, 1.7, 200.0, 1e-30])
def test_logprobs_scale(scale):
    g = gen(9)
    x = randn(g, 5, 3000, dt="f32", by=2.0)
    check_logprobs(x, ints([0, 1, 2, 3, 4]), scale=scale, top=4)


def test_logprobs_strides():
    """Rows inside wider ones, off every vector width, and one row for all tokens."""
    g = gen(10)
    wide = randn(g, 6, 9001)
    check_logprobs(wide[:, 3:8004], ints([0, 1, 2, 3, 4, 8000]), top=5)
    check_logprobs(wide[:1, 1:7000].expand(6, 6999), ints([0, 1, 2, 3, 4, 6998]), top=5)


# --- together ------------------------------------------------------------------------------------------

def test_no_tokens():
    x, w = torch.empty(0, 64, device="cuda"), torch.ones(64, device="cuda")
    P.mopar_rms_norm(x, w, out=x.clone())
    P.mopar_quantize_rows(x, P.alloc_rows8(0, 64, "cuda"))
    P.mopar_token_logprobs(x, ints([]), torch.empty(0, device="cuda"))


class Layer:
    """A small decoder layer and its head, as a serving loop drives them: 8-bit weights made by mopar_quantize_rows."""

    def __init__(self, g, width=256, heads=4, kv=2, ffn=704, vocab=3001):
        self.width, self.heads, self.kv, self.ffn, self.vocab, self.d = width, heads, kv, ffn, vocab, 64
        self.n1, self.n2, self.n3 = (1 + randn(g, width, by=0.1) for _ in range(3))
        shapes = dict(qkv=((heads + 2 * kv) * 64, width), o=(width, heads * 64), up=(2 * ffn, width), down=(width, ffn), head=(vocab, width))
        self.raw = {k: randn(g, *s, by=s[1] ** -0.5) for k, s in shapes.items()}
        self.w = {}
        for k, t in self.raw.items():
            self.w[k] = P.alloc_rows8(*t.shape, "cuda")
            P.mopar_quantize_rows(t, self.w[k])
        self.rotary = P.Rotary(64)

    def buffers(self, t):
        z = lambda *s: torch.zeros(*s, device="cuda", dtype=torch.bfloat16)  # noqa: E731
        e = lambda w: P.alloc_rows8(t, w, "cuda")  # noqa: E731
        b = dict(h=z(t, self.width), qkv=z(t, (self.heads + 2 * self.kv) * 64), att=z(t, self.heads * 64), o=z(t, self.width), up=z(t, 2 * self.ffn),
                 down=z(t, self.width), logits=z(t, self.vocab), a8=e(self.width), b8=e(self.heads * 64), c8=e(self.ffn),
                 lp=torch.zeros(t, device="cuda"), en=torch.zeros(t, device="cuda"), tl=torch.zeros(t, 4, device="cuda"),
                 ti=torch.zeros(t, 4, device="cuda", dtype=torch.int32))
        b["ws"] = torch.empty(max(P.mopar_linear8_workspace_bytes(t, n.rows, n.width) for n in self.w.values()), device="cuda", dtype=torch.uint8)
        b["ws2"] = P.alloc_token_logprobs_workspace(b["logits"], 4)
        return b

    def step(self, b, x, attend, tokens):
        """One layer and the head; attend(qkv rows) fills b["att"]."""
        W = self.w
        P.mopar_rms_norm(x, self.n1, out8=b["a8"])
        P.mopar_linear8(b["a8"], W["qkv"], b["qkv"], ws=b["ws"])
        attend(b["qkv"].view(x.shape[0], -1, 64))
        P.mopar_quantize_rows(b["att"], b["b8"])
        P.mopar_linear8(b["b8"], W["o"], b["o"], ws=b["ws"])
        P.mopar_rms_norm(b["o"], self.n2, residual=x, total=b["h"], out8=b["a8"])
        P.mopar_linear8(b["a8"], W["up"], b["up"], ws=b["ws"])
        P.mopar_quantize_rows(b["up"][:, self.ffn:], b["c8"], gate=b["up"][:, :self.ffn])
        P.mopar_linear8(b["c8"], W["down"], b["down"], ws=b["ws"])
        P.mopar_rms_norm(b["down"], self.n3, residual=b["h"], total=b["h"], out8=b["a8"])
        P.mopar_linear8(b["a8"], W["head"], b["logits"], ws=b["ws"])
        P.mopar_token_logprobs(b["logits"], tokens, b["lp"], entropy=b["en"], top_logprob=b["tl"], top_id=b["ti"], ws=b["ws2"])

    def plain(self, x):
        """The same in float64 with the weights' values: logits of every row (causal)."""
        deq = {k: v.dequantized().cpu().double() for k, v in self.w.items()}
        t = x.shape[0]
        norm = lambda v, n: v / torch.sqrt(v.square().mean(1, keepdim=True) + 1e-6) * n.cpu().double()  # noqa: E731
        x = x.cpu().double()
        qkv = (norm(x, self.n1) @ deq["qkv"].T).view(t, -1, 64)
        from tests.serving_ref import rotate
        pos = torch.arange(t)
        q, k, v = rotate(qkv[:, :self.heads], pos, 64)[0], rotate(qkv[:, self.heads:self.heads + self.kv], pos, 64)[0], qkv[:, self.heads + self.kv:]
        att = torch.empty(t, self.heads, 64, dtype=torch.float64)
        for h in range(self.heads):
            kh = h // (self.heads // self.kv)
            s = (q[:, h] @ k[:, kh].T / 8).masked_fill(torch.ones(t, t, dtype=torch.bool).triu(1), -math.inf)
            att[:, h] = torch.softmax(s, 1) @ v[:, kh]
        h1 = x + att.reshape(t, -1) @ deq["o"].T
        u = norm(h1, self.n2) @ deq["up"].T
        gate, up = u[:, :self.ffn], u[:, self.ffn:]
        h2 = h1 + (gate * torch.sigmoid(gate) * up) @ deq["down"].T
        return norm(h2, self.n3) @ deq["head"].T


def test_a_prompt_and_steps_over_its_cache():
    """A prompt of three sequences through the layer, then one token each over the cache: both against float64, and the
    single tokens against the same rows of a longer prompt."""
    g = gen(77)
    layer, lens = Layer(g), [19, 1, 40]
    seqs = [randn(g, n + 1, layer.width) for n in lens]
    t = sum(lens)
    from tests.serving_ref import page_table
    table, pages = page_table([n + 1 for n in lens], 16, g)
    kc, vc = (torch.zeros(pages, layer.kv, 16, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    cache = P.PagedCache(kc, vc, table.cuda())
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    H, K = layer.heads, layer.kv

    def prompt(rows):
        q, k, v = rows[:, :H], rows[:, H:H + K], rows[:, H + K:]
        pos = ints([i for n in lens for i in range(n)])
        seq = ints([s for s, n in enumerate(lens) for _ in range(n)])
        P.mopar_cache_append(cache, k, v, seq, pos, rotary=layer.rotary, pos=pos, q=q, q_out=q)
        turned = torch.empty_like(k)
        P.mopar_rotary_apply(layer.rotary, k, turned, pos)
        P.mopar_attention_prompt(q, turned, v, b["att"].view(t, H, 64), ints(off), max(lens))

    b = layer.buffers(t)
    layer.step(b, torch.cat([s[:-1] for s in seqs]), prompt, ints([5] * t))
    want = [layer.plain(s) for s in seqs]
    err = (b["logits"].cpu().double() - torch.cat([w[:-1] for w in want])).norm() / torch.cat([w[:-1] for w in want]).norm()
    # Activations in 8 bits with a largest of about 4 to 5 standard deviations: a step is 1/29 of one, its rounding 1/100 (uniform: 29
    # sqrt 12); six such roundings and the bf16 ones meet in the logits, each of its own sign: sqrt 8 of a 1/100, and half as much again.
    assert err < 0.045, float(err)
    ref = R.logprobs(b["logits"], ints([5] * t), top=4)
    check(b["lp"], ref["logprob"], ref["logprob_tol"])
    assert torch.equal(b["ti"].cpu().long(), ref["top_id"])

    b1 = layer.buffers(3)

    def token(rows):
        q, k, v = rows[:, :H], rows[:, H:H + K], rows[:, H + K:]
        pos = ints(lens)
        P.mopar_cache_append(cache, k, v, ints([0, 1, 2]), pos, rotary=layer.rotary, pos=pos, q=q, q_out=q)
        ws = P.alloc_attention_workspace(q, cache, 1, 64)
        P.mopar_attention_cache(q, b1["att"].view(3, H, 64), cache, ints([0, 1, 2, 3]), 1, ints(lens), 64, ws=ws)

    layer.step(b1, torch.stack([s[-1] for s in seqs]), token, ints([5] * 3))
    last = torch.stack([w[-1] for w in want])
    err = (b1["logits"].cpu().double() - last).norm() / last.norm()
    assert err < 0.045, float(err)


def test_captured_and_replayed():
    """The calls of a step in a graph, replayed over new inputs with eager work between, beside a second graph that shares the
    workspaces: every replay equals the eager result."""
    g = gen(78)
    layer, t = Layer(g), 5
    b, x = layer.buffers(t), randn(g, t, layer.width)
    tokens = ints([1, 2, 3, 4, 5])

    def attend(rows):
        b["att"].copy_(rows[:, :layer.heads].reshape(t, -1))
    names = ("h", "qkv", "down", "logits", "lp", "en", "tl", "ti")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.step(b, x, attend, tokens)
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for gr in graphs:
        with torch.cuda.graph(gr):
            layer.step(b, x, attend, tokens)
    for i in range(4):
        x.copy_(randn(gen(100 + i), t, layer.width))
        layer.step(b, x, attend, tokens)
        torch.cuda.synchronize()
        want = {k: b[k].clone() for k in names}
        for gr in graphs:
            for k in names:
                b[k].zero_()
            gr.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(b[k], want[k]) for k in names)


def test_other_streams():
    """Calls on a stream of the caller's run there, in its order."""
    g = gen(79)
    x, w = randn(g, 300, 4096), randn(g, 4096)
    side = torch.cuda.Stream()
    a8, b8 = P.alloc_rows8(300, 4096, "cuda"), P.alloc_rows8(300, 4096, "cuda")
    wq = rows8(g, 512, 4096)
    out, got = torch.empty(300, 512, device="cuda"), torch.empty(300, 512, device="cuda")
    P.mopar_rms_norm(x, w, out8=a8)
    P.mopar_linear8(a8, wq, out)
    side.wait_stream(torch.cuda.current_stream())
    P.mopar_rms_norm(x, w, out8=b8, stream=side)
    P.mopar_linear8(b8, wq, got, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(out, got)
