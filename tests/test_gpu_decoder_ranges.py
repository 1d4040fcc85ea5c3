"""Norms, gated rows and log probabilities whose factors float32 holds and whose products it does not: past its largest
value, below its smallest, or rounded on the way where it holds few bits."""
import math

import pytest
import torch

import paper_2404_02445_amd as P
from tests import decoder_ref as R
from tests.decoder_ref import U, check
from tests.test_gpu_decoder import DT, check_marks, gen, ints, marked, randn

pytestmark = pytest.mark.gpu

# one width for each way that a row is held: half a wave, a wave, a block, and read twice
WIDTHS = [200, 600, 2056, 33000]


def check_gated(x, gate, act):
    q, out8 = marked(*x.shape)
    P.mopar_quantize_rows(x, out8, gate=gate, act=act)
    p = R.gated(x, gate, act)
    steps, top = R.steps(p)
    # float64 rounds, too: a function (within 4 half steps in either library), three products and the division of 127 p by a leave
    # at most 10 half steps on each side, 127 * 20 * 2^-53 of a value.  Where it lies so near a middle (x half the row's largest under the same
    # gate: 63.5), either step is right.
    value = p * 127 / top[:, None]
    tie = ((value - value.floor() - 0.5).abs() <= 127 * 20 * 2.0 ** -53) & ((out8.values.cpu() - value).abs() <= 0.5000001)
    assert bool(((out8.values.cpu() == steps) | tie).all())
    want = (top / 127).float().double()              # (infinite past float32's range)
    check(out8.scales, want, want.abs().nan_to_num(0.0, 0.0) * 2.02 * U + 1e-45)
    check_marks(q, x.shape[1])
    return out8


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("width", WIDTHS)
def test_gated_rows_past_float32(dt, act, width):
    """Finite gates and values whose products are not finite in float32: steps of the products, their scales where float32 holds them."""
    g = gen(width)
    x, gate = randn(g, 6, width, dt=dt).clamp(-3, 3), randn(g, 6, width, dt=dt).clamp(-4, 4)
    gate[0, 3], x[0, 3] = 3e38, 2.0                   # one such product
    gate[1] *= 8e37                                   # most of a row
    x[2], gate[2] = x[2] * 1e38, gate[2] * 9.0
    x[3], gate[3] = x[3] * 1e38, gate[3] * 8e37       # a scale that float32 does not hold
    gate[4], x[4], x[4, 0] = gate[4] * 8e37, x[4] * 9.0, math.inf
    out8 = check_gated(x, gate, act)
    assert bool(out8.scales[:3].isfinite().all()) and bool(out8.scales[3].isinf()) and bool(out8.scales[4].isnan())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("width", WIDTHS)
def test_gated_rows_below_float32(dt, act, width):
    """Rows of products that float32 holds in part or not at all: the steps are those of the products, whatever their scale comes to."""
    g = gen(width)
    x, gate = randn(g, 6, width, dt=dt), randn(g, 6, width, dt=dt)
    x[0], gate[0] = x[0] * 1e-30, gate[0] * 1e-30
    x[1], gate[1] = x[1] * 1e-25, gate[1] * 1e-18
    x[2], gate[2] = x[2] * 1e-12, -95.0 if act == "silu" else -13.0
    x[3] = 0
    gate[4] = 0
    check_gated(x, gate, act)


# --- norms -------------------------------------------------------------------------------------------

def far_norms(dt, width):
    """Rows and weights whose products leave float32's range while squares, sums and results do not; eps of each set."""
    g = gen(width + 1)
    x, w = randn(g, 6, width, dt=dt), randn(g, width, dt=dt)
    x[2], x[3, ::3], x[4, 1:] = 0, 0, 0
    return [("past", x * 1e15, w * 1e30, 1e-5), ("below", x * 1e-18, w * 1e-22, 1e-5), ("far below", x * 1e-15, w * 1e-32, 0.0), ("some below", x, w * 1e-38, 1e-5),
            ("some far below", x * 1e-10, torch.where(torch.arange(width, device="cuda") % 2 == 0, w * 1e-32, w), 0.0)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("which", range(5))
def test_norm_steps_outside_float32(dt, width, which):
    name, x, w, eps = far_norms(dt, width)[which]
    q, out8 = marked(*x.shape)
    P.mopar_rms_norm(x, w, eps, out8=out8)
    steps = R.steps(x.cpu().double() * w.cpu().double())[0]
    assert torch.equal(out8.values.cpu(), steps), name
    some = (x != 0).any(1).cpu()                      # (without eps the factor of a row of zeros is infinite)
    want = R.norm(x[some.cuda()], w, eps)[4].float().double()
    check(out8.scales[some.cuda()], want, want * (R.sum_bound(width) + 8 * U) + 1e-45)
    assert not bool(out8.scales[~some.cuda()].any())
    check_marks(q, width)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("which", range(5))
@pytest.mark.parametrize("form", ["out", "both", "in place", "residual", "total"])
def test_norm_results_outside_float32(dt, width, which, form):
    name, x, w, eps = far_norms(dt, width)[which]
    some = (x != 0).any(1)
    want, tol = (t[some.cpu()] for t in R.norm(x, w, eps)[1:3])
    res = torch.zeros_like(x) if form in ("residual", "total") else None
    out = x.clone() if form == "in place" else torch.full_like(x, 7.0)
    total = torch.empty_like(x) if form == "total" else None
    P.mopar_rms_norm(out if form == "in place" else x, w, eps, residual=res, total=total, out=out, out8=marked(*x.shape)[1] if form == "both" else None)
    # (check() lets 1e-37 pass: results are taken to where that is nothing.  Results below 2^-126 have a rounding of half their type's smallest
    # value; a product below it one of 2^-150, times r where r is at most 2^24.)
    by = 2.0 ** 60 if "below" in name else 1.0
    r = 1 / torch.sqrt(x[some].cpu().double().square().mean(1, keepdim=True) + eps)
    tol = tol + 2.0 ** (-134 if dt == "bf16" else -150) * 1.01 + torch.where(r > 2.0 ** 24, 0.0, r * 2.0 ** -150 * 1.01)
    check(out[some].double() * by, want * by, tol * by, name)
    if eps:
        assert not bool(out[~some].any())


# --- where float32 holds few bits ----------------------------------------------------------------------

def test_silu_gates_where_its_reciprocal_ends():
    """1 / (1 + e^-gate) at the end of float32's normal range: what it loses there is counted in what a step may be off."""
    gates = torch.linspace(-87.5, -87.34, 60)
    near = torch.linspace(0.49, 0.52, 40)             # steps that the far gates' products come to
    x = torch.full((40, 61), 1e30)
    x[:, 0] = 127 * 1.0268e-6 / near / 30
    gate = torch.cat([torch.full((40, 1), 30.0), gates.expand(40, 60)], 1)
    check_gated(x.cuda(), gate.cuda(), "silu")


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gates_of_few_bits(dt, act):
    """Subnormal gates beside values near float32's largest: half of such a gate may be no float32."""
    tiny = 2.0 ** (-149 if dt == "f32" else -133)
    gate = (torch.arange(1, 202, dtype=torch.float64) * tiny).to(DT[dt])[None].repeat(3, 1)
    x = torch.full_like(gate, 1e38)
    x[1], gate[2, ::2] = 3e30, -gate[2, ::2]      # (201: no step is a tie)
    check_gated(x.cuda(), gate.cuda(), act)


@pytest.mark.parametrize("scale", [0.25, 0.5, 1.0, 3e-5])
def test_logprobs_of_logits_at_both_ends(scale):
    """Logits whose difference passes float32 where its product with the scale does not."""
    x = torch.tensor([[3e38, -3e38, 2.9e38, -2e38, 0.0], [3.4e38, -3.4e38, -math.inf, 3.4e38, 1.0], [1.7e38, -1.8e38, 1.0, 2.0, 3.0]], device="cuda")
    ref = R.logprobs(x, ints([1, 1, 1]), scale, 5)
    lp, en = torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    tl, ti = torch.empty(3, 5, device="cuda"), ints([[0] * 5] * 3)
    P.mopar_token_logprobs(x, ints([1, 1, 1]), lp, entropy=en, top_logprob=tl, top_id=ti, scale=scale)
    assert torch.equal(ti.cpu().long(), ref["top_id"])
    for got, name, tol in ((lp, "logprob", "logprob_tol"), (tl, "top_logprob", "top_tol")):
        check(got, ref[name].float().double(), ref[tol])
    check(en, ref["entropy"], torch.full_like(ref["entropy"], ref["entropy_tol"]))
