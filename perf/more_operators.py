"""Operators of a decoder's step around its attention, with weights and activations in 8 bits: what is
measured, over the sizes it is measured at.

Four operators that a serving loop runs one after the other in every step:

* ``norm``    -- the residual stream added up and normalised by its root mean square, the result in
  the rows' type or as 8-bit rows with a scale each (``mopar_rms_norm``);
* ``quant``   -- rows to 8 bits with a scale each, plain or the product with an activated gate
  (``mopar_quantize_rows``): what a second product reads, and how weights are made;
* ``linear``  -- the product of 8-bit rows with 8-bit weights, a scale for each token and each channel
  (``mopar_linear8``);
* ``logprob`` -- log probabilities of given tokens, their ranks, the entropy and the most likely
  alternatives (``mopar_token_logprobs``).

``own`` says which side ``run`` computes: the framework's entry points, or a plain form of
elementary torch operations in float32 (float64 where values lie next to the border of two 8-bit
steps), rounded once at the end.  ``exact`` evaluates the definitions in float64, apart from both.
8-bit rows are returned as the values that they stand for.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
ESZ = {"f32": 4, "bf16": 2}


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # five float32 rows of an odd width, nothing added: launch latency, rows off every vector width
        dict(name="norm_f32_odd", op="norm", dt="f32", tokens=5, width=1003, residual=False, to="rows"),
        # eight sequences' next tokens on the way into a layer's first product: launch latency
        dict(name="norm_decode_b8", op="norm", dt="bf16", tokens=8, width=4096, residual=True, to="8bit"),
        # the tokens of a long prompt on the same way
        dict(name="norm_prompt_16k", op="norm", dt="bf16", tokens=16384, width=4096, residual=True, to="8bit"),
        # the gated middle of a feed-forward layer for 64 sequences' next tokens, gate and value in fused rows
        dict(name="quant_gate_b64", op="quant", dt="bf16", tokens=64, width=14336, gate="silu"),
        # the same for the tokens of a prompt, another gate and an odd width
        dict(name="quant_gate_prompt", op="quant", dt="bf16", tokens=4001, width=11007, gate="gelu"),
        # one new token against a square weight: the time to read the weight
        dict(name="linear_decode_b1", op="linear", dt="bf16", tokens=1, width=4096, n=4096, bias=False),
        # 64 new tokens, a long sum and few columns: neither rows nor columns fill the card
        dict(name="linear_decode_b64", op="linear", dt="bf16", tokens=64, width=14336, n=4096, bias=False),
        # odd sizes, a bias, float32 results: a small head of a model
        dict(name="linear_f32_odd", op="linear", dt="f32", tokens=333, width=1001, n=2051, bias=True),
        # the first product of a feed-forward layer over a prompt: the largest work
        dict(name="linear_prompt_8k", op="linear", dt="bf16", tokens=8192, width=4096, n=14336, bias=False),
        # what four sequences' next tokens could have been: few rows of a large vocabulary
        dict(name="logprob_decode_b4", op="logprob", dt="bf16", tokens=4, vocab=128000, top=20),
        # a float32 row set of an odd vocabulary without alternatives: perplexity
        dict(name="logprob_f32_odd", op="logprob", dt="f32", tokens=257, vocab=32003, top=0),
        # a prompt scored: every token's probability and its five alternatives
        dict(name="logprob_prompt_2k", op="logprob", dt="bf16", tokens=2048, vocab=128000, top=5),
    ]


def _log(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _size(rng, lo, hi):
    """... as sizes come: any integer, or a multiple of 16, 64 or 256."""
    n, m = _log(rng, lo, hi), rng.choice([1, 16, 64, 256])
    return max(n // m * m, min(m, hi))


def _draw_once(rng):
    op, dt = rng.choice(["norm", "quant", "linear", "linear", "logprob"]), rng.choice(["bf16", "bf16", "f32"])
    if op == "norm":
        return dict(op=op, dt=dt, tokens=_log(rng, 1, 16384), width=_size(rng, 32, 16384), residual=rng.random() < 0.6,
                    to=rng.choice(["rows", "8bit", "8bit", "both"]))
    if op == "quant":
        return dict(op=op, dt=dt, tokens=_log(rng, 1, 8192), width=_size(rng, 32, 32768), gate=rng.choice(["none", "silu", "silu", "gelu"]))
    if op == "linear":
        return dict(op=op, dt=dt, tokens=_log(rng, 1, 16384), width=_size(rng, 16, 32768), n=_size(rng, 1, 65536), bias=rng.random() < 0.3)
    vocab = _size(rng, 64, 262144)
    return dict(op=op, dt=dt, tokens=_log(rng, 1, 4096), vocab=vocab, top=rng.choice([0, 1, 5, 20, min(64, vocab)]))


def _cost(case):
    """A bound on what a case asks of the card: seconds at matrix and copy rates of the plain forms."""
    w = work(case)
    return w["flops"] / 1.3e14 + w["bytes"] / 4e12


def draw(rng):
    limit = max(_cost(c) for c in listed() if c["op"] == "linear")
    most = max(work(c)["bytes"] for c in listed())
    while True:
        case = _draw_once(rng)
        if _cost(case) <= limit and work(case)["bytes"] <= most:
            return case


def work(case):
    op, es, t = case["op"], ESZ[case["dt"]], case["tokens"]
    if op == "norm":        # rows (and what is added) read, the sum, the rows and the 8-bit rows written
        w = case["width"]
        rows = 1 + 2 * case["residual"] + (case["to"] != "8bit")
        eight = (w + 4) * (case["to"] != "rows")
        return {"bytes": t * (rows * w * es + eight) + w * es, "flops": 4 * t * w}
    if op == "quant":       # rows and gates read, 8-bit rows and scales written
        w = case["width"]
        return {"bytes": t * (w * es * (2 if case["gate"] != "none" else 1) + w + 4), "flops": 3 * t * w}
    if op == "linear":      # 8-bit rows, weights, both scales and the bias read, results written
        k, n = case["width"], case["n"]
        return {"bytes": t * (k + 4) + n * (k + 4 + es * case["bias"]) + t * n * es, "flops": 2 * t * n * k}
    return {"bytes": t * (case["vocab"] * es + 16 + 8 * case["top"]), "flops": 5 * t * case["vocab"]}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _rows8(g, rows, width):
    """8-bit rows as a program keeps them: a row starts at a multiple of 16 bytes; a scale for each."""
    stride = (width + 15) // 16 * 16
    q = (torch.randn(rows, stride, generator=g, device=DEV) * 32).round_().clamp_(-127, 127).to(torch.int8)
    return q[:, :width], torch.rand(rows, generator=g, device=DEV) * 0.01 + 1e-3


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * seed + 17)
    dt, op, t = TDT[case["dt"]], case["op"], case["tokens"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=dt)

    st = dict(case=case)
    if op in ("norm", "quant"):
        w = case["width"]
        stride = (w + 15) // 16 * 16
        st.update(q=torch.zeros(t, stride, device=DEV, dtype=torch.int8)[:, :w], scale=torch.zeros(t, device=DEV))
    if op == "norm":
        x = normal(t, w)
        x[:, ::97] *= 8                                       # a few channels far larger than the others
        st.update(x=x, weight=1 + 0.2 * normal(w), residual=normal(t, w) if case["residual"] else None,
                  total=torch.zeros_like(x) if case["residual"] else None,
                  out=torch.zeros_like(x) if case["to"] != "8bit" else None)
    elif op == "quant":
        rows = normal(t, 2 * w if case["gate"] != "none" else w) * 2
        st.update(x=rows[:, -w:], gate=rows[:, :w] if case["gate"] != "none" else None)
    elif op == "linear":
        x, w = _rows8(g, t, case["width"]), _rows8(g, case["n"], case["width"])
        st.update(x=x, w=w, bias=normal(case["n"]) if case["bias"] else None, out=torch.zeros(t, case["n"], device=DEV, dtype=dt))
    else:
        v, top = case["vocab"], case["top"]
        x = normal(t, v)
        x *= (torch.rand(t, 1, generator=g, device=DEV) * 4 + 0.5).to(dt)          # flat and peaked rows
        x[::5, ::3] = -math.inf                                                     # tokens that a grammar rules out
        token = torch.randint(0, v, (t,), generator=g, device=DEV, dtype=torch.int32)
        best = torch.argmax(x[::2], 1)                                              # half of the tokens as a model picks them
        token[::2] = best.to(torch.int32)
        st.update(x=x, token=token, logprob=torch.zeros(t, device=DEV), entropy=torch.zeros(t, device=DEV),
                  rank=torch.zeros(t, device=DEV, dtype=torch.int32),
                  top_logprob=torch.zeros(t, top, device=DEV) if top else None,
                  top_id=torch.zeros(t, top, device=DEV, dtype=torch.int32) if top else None)
    if own:
        import paper_2404_02445_amd as P
        if op in ("norm", "quant"):
            st["rows8"] = P.Rows8(st["q"], st["scale"])
        elif op == "linear":
            st["x8"], st["w8"] = P.Rows8(*st["x"]), P.Rows8(*st["w"])
            st["ws"] = P.alloc_linear8_workspace(st["x8"], st["w8"], st["out"])
        else:
            st["ws"] = P.alloc_token_logprobs_workspace(st["x"], case["top"])
    return st


EPS = 1e-5


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------

def _to_8bit(p):
    """p (float64) in 8 bits: the steps, and a row's largest magnitude; rows of zeros give zeros."""
    top = p.abs().amax(1, keepdim=True)
    return torch.round(p * 127 / torch.where(top > 0, top, torch.ones_like(top))), top


def _plain_norm(st):
    x, case = st["x"], st["case"]
    h = x if st["residual"] is None else (x.float() + st["residual"].float()).to(x.dtype)
    outs = [] if st["residual"] is None else [h]
    r = torch.rsqrt(h.double().square().mean(1, keepdim=True) + EPS)
    if case["to"] != "8bit":
        outs.append((h.float() * r.float() * st["weight"].float()).to(x.dtype))
    if case["to"] != "rows":
        q, top = _to_8bit(h.double() * st["weight"].double())
        outs.append(q.float() * (top * r / 127).float())
    return outs


def _plain_quant(st):
    x, gate = st["x"].double(), st["case"]["gate"]
    if gate != "none":
        z = st["gate"].double()
        x = x * (z / (1 + torch.exp(-z)) if gate == "silu" else 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5))))
    q, top = _to_8bit(x)
    return q.float() * (top / 127).float()


def _plain_linear(st):
    (x, sx), (w, sw) = st["x"], st["w"]
    y = torch.matmul(x.float(), w.float().t()) * sx[:, None] * sw[None]
    if st["bias"] is not None:
        y = y + st["bias"].float()
    st["out"].copy_(y)
    return st["out"]


def _plain_logprob(st):
    x, token, top = st["x"].float(), st["token"].long()[:, None], st["case"]["top"]
    m = x.amax(1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    total = e.sum(1, keepdim=True, dtype=torch.float64)
    log_total = torch.log(total)
    entropy = log_total - torch.where(e > 0, e * d, torch.zeros_like(e)).sum(1, keepdim=True, dtype=torch.float64) / total
    mine = torch.gather(x, 1, token)
    outs = [(mine - m - log_total).float()[:, 0], entropy.float()[:, 0], (x > mine).sum(1, dtype=torch.int32)]
    if top:
        bits = (x + 0.0).view(torch.int32)                               # ordered as the floats are, ties to the lowest index
        key = (bits ^ ((bits >> 31) & 0x7fffffff)).long() * 2 ** 32 + (2 ** 32 - 1 - torch.arange(x.shape[1], device=DEV))
        ids = (2 ** 32 - 1) - (torch.topk(key, top, 1).values & (2 ** 32 - 1))
        outs += [(torch.gather(x, 1, ids) - m - log_total).float(), ids.to(torch.int32)]
    return outs


def run(state):
    op = state["case"]["op"]
    if not own:
        return {"norm": _plain_norm, "quant": _plain_quant, "linear": _plain_linear, "logprob": _plain_logprob}[op](state)
    import paper_2404_02445_amd as P
    if op == "norm":
        to = state["case"]["to"]
        P.mopar_rms_norm(state["x"], state["weight"], EPS, residual=state["residual"], total=state["total"], out=state["out"],
                         out8=state["rows8"] if to != "rows" else None)
        outs = [t for t in (state["total"], state["out"]) if t is not None]
        return outs if to == "rows" else outs + [state["q"] * state["scale"][:, None]]
    if op == "quant":
        P.mopar_quantize_rows(state["x"], state["rows8"], gate=state["gate"], act=state["case"]["gate"])
        return state["q"] * state["scale"][:, None]
    if op == "linear":
        return P.mopar_linear8(state["x8"], state["w8"], state["out"], bias=state["bias"], ws=state["ws"])
    P.mopar_token_logprobs(state["x"], state["token"], state["logprob"], entropy=state["entropy"], rank=state["rank"],
                           top_logprob=state["top_logprob"], top_id=state["top_id"], ws=state["ws"])
    outs = [state["logprob"], state["entropy"], state["rank"]]
    return outs if state["top_id"] is None else outs + [state["top_logprob"], state["top_id"]]


# ---------------------------------------------------------------------------
# the definitions in float64
# ---------------------------------------------------------------------------

def _stands_for64(v, factor):
    """What 8-bit rows of v times factor stand for: steps of a 127th of a row's largest magnitude, halves to even."""
    out = torch.zeros_like(v)
    for row in range(0, v.shape[0], 1024):
        part = v[row:row + 1024]
        top = torch.maximum(part.max(1).values, -part.min(1).values)[:, None]
        step = torch.where(top == 0, 1.0, part * 127 / top).round() * (top != 0)
        out[row:row + 1024] = step * (top * factor[row:row + 1024] / 127)
    return out


def exact(case, seed):
    st, op = prepare(case, seed), case["op"]
    if op == "norm":
        h, outs = st["x"], []
        if st["residual"] is not None:
            h = (h.double() + st["residual"].double()).to(h.dtype)               # the stream is kept in the rows' type
            outs.append(st["x"].double() + st["residual"].double())
        h = h.double()
        r = 1 / torch.sqrt((h * h).sum(1, keepdim=True) / case["width"] + EPS)
        v = h * st["weight"].double()
        if case["to"] != "8bit":
            outs.append(v * r)
        if case["to"] != "rows":
            outs.append(_stands_for64(v, r))
        return outs
    if op == "quant":
        v = st["x"].double()
        if case["gate"] == "silu":
            v = v * st["gate"].double() * torch.sigmoid(st["gate"].double())
        if case["gate"] == "gelu":
            v = v * (st["gate"].double() * torch.special.erfc(-st["gate"].double() / math.sqrt(2)) / 2)
        return _stands_for64(v, torch.ones(v.shape[0], 1, device=DEV, dtype=torch.float64))
    if op == "linear":
        (x, sx), (w, sw) = st["x"], st["w"]
        wd = w.double() * sw.double()[:, None]
        out = torch.stack([torch.mv(wd, r) for r in x.double()]) if x.shape[0] < 4 else x.double() @ wd.T.contiguous()
        out *= sx.double()[:, None]
        return out if st["bias"] is None else out.add_(st["bias"].double())
    x, ids = st["x"], st["token"].long()
    logp, entropy = torch.empty(len(ids), device=DEV, dtype=torch.float64), torch.empty(len(ids), device=DEV, dtype=torch.float64)
    tops = torch.empty(len(ids), case["top"], device=DEV, dtype=torch.float64)
    for i in range(0, len(ids), 64):
        lp = torch.log_softmax(x[i:i + 64].double(), 1)
        logp[i:i + 64] = torch.gather(lp, 1, ids[i:i + 64, None])[:, 0]
        entropy[i:i + 64] = -(torch.exp(lp) * lp).nan_to_num(nan=0.0).sum(1)
        tops[i:i + 64] = torch.topk(lp, case["top"], 1).values
    return [logp, entropy, None] + ([tops, None] if case["top"] else [])
