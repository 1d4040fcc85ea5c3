"""Plain float64 forms of a decoder's steps in 8 bits, on the CPU, and the bounds of what float32 arithmetic and one
rounding may differ from them."""
import math

import torch

from tests.serving_ref import HALF_STEP, check  # noqa: F401

U = 2.0 ** -24          # half a step of float32


def sum_bound(n, threads=64):
    """Relative error of a float32 sum of n positive values: what a thread adds one after the other, then a tree over at most
    1024 threads, and a few roundings around it."""
    return (n / threads + 100) * U


def stream(x, residual):
    """The residual stream in the rows' type."""
    return x if residual is None else (x.double() + residual.double()).to(x.dtype)


def steps(p):
    """Rows of 8-bit steps of p (float64) and their largest magnitudes; a row that is not finite gives zeros and NaN."""
    top = p.abs().amax(1, keepdim=True)
    fine = torch.isfinite(p).all(1, keepdim=True)
    q = torch.where(fine & (top > 0), (p * 127 / torch.where(top > 0, top, 1.0)).round(), 0.0).nan_to_num(0.0)
    return q.to(torch.int8), torch.where(fine, top, math.nan)[:, 0]


def norm(x, weight, eps, residual=None):
    """h, out (float64) and its bound, steps, scales (float64)."""
    x, weight = x.cpu(), weight.cpu()
    h = stream(x, None if residual is None else residual.cpu())
    r = 1 / torch.sqrt(h.double().square().mean(1, keepdim=True) + eps)
    p = h.double() * weight.double()
    q, top = steps(p)
    out = p * r
    tol = out.abs() * (sum_bound(x.shape[1]) + 8 * U + HALF_STEP[x.dtype] * 1.01)
    return h, out, tol, q, top * r[:, 0] / 127


def gated(x, gate, act):
    x, g = x.cpu().double(), None if gate is None else gate.cpu().double()
    if act == "silu":
        return g / (1 + torch.exp(-g)) * x
    if act == "gelu":
        return 0.5 * g * torch.special.erfc(-g / math.sqrt(2)) * x
    return x


def linear(x, w, out_dtype, bias=None):
    """x, w: (values, scales).  float64 results and the bound: the sum to float32 1, two factors 2, a bias 1; then one rounding."""
    (qx, sx), (qw, sw) = ((v.cpu(), s.cpu()) for v, s in (x, w))
    y = (qx.double() @ qw.double().T) * sx.double()[:, None] * sw.double()[None]       # (sums below 2^53: exact)
    tol = y.abs() * 4 * U
    if bias is not None:
        y = y + bias.cpu().double()
        tol = tol + y.abs() * U
    return y, tol * 1.01 + y.abs() * HALF_STEP[out_dtype] * 1.01 + 1e-38


def logprobs(x, tokens, scale=1.0, top=0):
    """logprob and its bound, entropy and its bound, rank, top_logprob and its bound, top_id."""
    raw = x.cpu().double()
    z, n = raw * scale, x.shape[1]
    tokens = tokens.cpu().long()
    m = z.amax(1, keepdim=True)
    e = torch.exp(z - torch.where(torch.isinf(m) & (m < 0), 0.0, m))
    s = e.sum(1, keepdim=True)
    nothing = (s == 0)[:, 0]
    p = e / s
    entropy = torch.where(p > 0, -p * torch.log(p), torch.where(p.isnan(), math.nan, 0.0)).sum(1)
    entropy[nothing] = 0.0

    def of(ids):
        lp = (torch.gather(z, 1, ids) - m) - torch.log(s)          # (m first: it may be far larger than the logarithm)
        return torch.where(nothing[:, None], -math.inf, lp)
    known = (tokens >= 0) & (tokens < n)
    ids = torch.where(known, tokens, 0)[:, None]
    mine = torch.gather(raw, 1, ids)
    logprob = torch.where(known, of(ids)[:, 0], -math.inf)
    rank = torch.where(known, (raw > mine).sum(1), n)
    # exponents: 3 roundings of z log2(e), of which weight 2^z leaves under 1 in all; 2 of the exponential; then the sum
    base = sum_bound(n, 256) + 8 * U

    def bound(lp, far):
        return base + 4 * U * (lp.abs().nan_to_num(0, 0, 0) + far.abs().nan_to_num(0, 0, 0) + math.log(n) + 1)
    out = dict(logprob=logprob, logprob_tol=bound(logprob, torch.gather(z, 1, ids)[:, 0] - m[:, 0]), entropy=entropy,
               entropy_tol=3 * base * (math.log(n) + 1), rank=rank)
    if top:
        key = torch.where(raw.isnan(), -math.inf, raw)
        order = torch.sort(key, dim=1, descending=True, stable=True).indices
        # (NaN behind -infinity, and no alternative)
        order = torch.gather(order, 1, torch.sort(torch.gather(raw, 1, order).isnan().int(), dim=1, stable=True).indices)[:, :top]
        real = ~torch.gather(raw, 1, order).isnan()
        out["top_id"] = torch.where(real, order, -1)
        out["top_logprob"] = torch.where(real, of(order), math.nan)
        out["top_tol"] = bound(out["top_logprob"], torch.gather(z, 1, order) - m)
    return out
