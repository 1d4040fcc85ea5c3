"""Operators of a decoder-style language model served with a paged key/value cache: what is
measured, over the sizes it is measured at.

Five operators that a serving loop runs one after the other in every layer:

* ``rotary``  -- rotary positions on the query and key heads of packed token rows
  (``mopar_rotary_apply``);
* ``append``  -- the same on the way into the cache: query heads turned, key heads turned and
  stored with their values in the pages of their sequence (``mopar_cache_append``);
* ``prompt``  -- causal attention over packed prompts of different lengths, grouped heads
  (``mopar_attention_prompt``);
* ``tree``    -- attention of newly drafted tokens, a tree of them or a single one, over the paged
  cache of their sequence (``mopar_attention_cache``);
* ``keep``    -- after verification, the accepted path of a drafted tree moved to where the
  sequence goes on, in every layer's cache (``mopar_cache_keep``).

``own`` says which side ``run`` computes: the framework's entry points, or a plain form of
elementary torch operations in float32 (angles in float64), rounded once at the end.  ``exact``
evaluates the definitions in float64, apart from both.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda"
TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
ESZ = {"f32": 4, "bf16": 2}
RATE = {"f32": 1.3e14, "bf16": 1.4e15}      # matrix rates that bound a drawn case's size


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # four short float32 sequences, a part of each head turned, pairs of neighbours: launch latency
        dict(name="rotary_f32_part", op="rotary", dt="f32", heads=24, rest=12, d=64, rot=32, layout="interleaved",
             scaling="none", factor=1.0, tokens=308, far=0),
        # a long context taken in at once: query and key heads of fused rows, scaled angles of far positions
        dict(name="rotary_prompt_16k", op="rotary", dt="bf16", heads=40, rest=8, d=128, rot=128, layout="half",
             scaling="yarn", factor=16.0, tokens=16384, far=100000),
        # one new token for each of eight sequences: launch latency
        dict(name="append_decode_b8", op="append", dt="bf16", heads=32, kv=8, d=128, rot=128, layout="half",
             scaling="none", factor=1.0, page=16, seqs=8, lo=1, hi=1, past=2000, shape=1),
        # the rows of three prompts, 8192 tokens at most each, into empty caches
        dict(name="append_prompts", op="append", dt="bf16", heads=32, kv=8, d=128, rot=128, layout="half",
             scaling="none", factor=1.0, page=64, seqs=3, lo=1500, hi=8192, past=0, shape=2),
        # four sequences of 77 tokens in float32, twelve heads of their own keys: a small model's prompt
        dict(name="prompt_f32_s77", op="prompt", dt="f32", heads=12, kv=12, d=64, seqs=4, lo=77, hi=77, shape=1),
        # sixteen ragged prompts packed into one batch, four query heads to a key head
        dict(name="prompt_packed_b16", op="prompt", dt="bf16", heads=32, kv=8, d=128, seqs=16, lo=20, hi=1100, shape=3),
        # one long prompt: the largest work
        dict(name="prompt_8k", op="prompt", dt="bf16", heads=32, kv=8, d=128, seqs=1, lo=8192, hi=8192, shape=1),
        # one token over one long float32 cache, every head its own keys: the split over the long axis
        dict(name="decode_f32_b1_16k", op="tree", dt="f32", heads=12, kv=12, d=64, page=16, seqs=1, qlo=1, qhi=1,
             lo=16400, hi=16400, tree=False, shape=1),
        # an ordinary decode step: one token for each of 64 sequences of up to 4096 cached tokens
        dict(name="decode_b64", op="tree", dt="bf16", heads=32, kv=8, d=128, page=16, seqs=64, qlo=1, qhi=1,
             lo=100, hi=4096, tree=False, shape=4),
        # verification of a drafted tree of up to 48 tokens in each of 16 sequences
        dict(name="tree_b16_n48", op="tree", dt="bf16", heads=32, kv=8, d=128, page=64, seqs=16, qlo=20, qhi=48,
             lo=1000, hi=8000, tree=True, shape=5),
        # the accepted tokens of four sequences, one layer: launch latency
        dict(name="keep_b4", op="keep", dt="f32", kv=12, d=64, page=16, layers=1, seqs=4, chains=3, depth=5, past=100,
             shape=1),
        # the accepted tokens of 32 sequences in the caches of 16 layers
        dict(name="keep_b32_l16", op="keep", dt="bf16", kv=8, d=128, page=16, layers=16, seqs=32, chains=4, depth=8,
             past=60, shape=2),
    ]


def _log(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_once(rng):
    op = rng.choice(["rotary", "append", "prompt", "prompt", "tree", "tree", "tree", "keep"])
    dt = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([32, 64, 64, 96, 128, 128, 128])
    kv = rng.choice([1, 2, 3, 4, 5, 8, 8])
    heads = kv * rng.choice([1, 2, 3, 4, 4, 5, 7, 8])
    page = rng.choice([1, 8, 16, 16, 32, 64, 128, 256])
    scaling = rng.choice(["none", "none", "linear", "ntk", "yarn"])
    turn = dict(rot=d if rng.random() < 0.6 else 2 * rng.randint(2, d // 2), layout=rng.choice(["half", "interleaved"]),
                scaling=scaling, factor=1.0 if scaling == "none" else round(rng.uniform(1.5, 40.0), 2))
    shape = rng.randint(0, 10 ** 6)
    if op == "rotary":
        return dict(op=op, dt=dt, heads=heads + kv, rest=rng.choice([0, kv]), d=d, **turn, tokens=_log(rng, 1, 32768),
                    far=rng.choice([0, 0, _log(rng, 1000, 1000000)]))
    if op == "append":
        seqs, hi = _log(rng, 1, 128), _log(rng, 1, 8192)
        return dict(op=op, dt=dt, heads=heads, kv=kv, d=d, **turn, page=page, seqs=seqs, lo=rng.randint(1, hi), hi=hi,
                    past=rng.choice([0, _log(rng, 1, 4000)]), shape=shape)
    if op == "prompt":
        seqs, hi = _log(rng, 1, 64), _log(rng, 1, 8192)
        return dict(op=op, dt=dt, heads=heads, kv=kv, d=d, seqs=seqs, lo=rng.randint(1, hi), hi=hi, shape=shape)
    if op == "tree":
        tree = rng.random() < 0.5
        qhi = _log(rng, 2, 128) if tree else rng.choice([1, 1, 1, _log(rng, 1, 64)])
        hi = _log(rng, 1, 65536)
        return dict(op=op, dt=dt, heads=heads, kv=kv, d=d, page=page, seqs=_log(rng, 1, 128),
                    qlo=rng.randint(1, qhi), qhi=qhi, lo=rng.randint(1, hi), hi=hi, tree=tree, shape=shape)
    return dict(op=op, dt=dt, kv=kv, d=d, page=page, layers=rng.randint(1, 24), seqs=_log(rng, 1, 64),
                chains=rng.randint(1, 8), depth=rng.randint(1, 12), past=_log(rng, 1, 400), shape=shape)


def _cost(case):
    """A bound on what a case asks of the card: seconds at matrix and copy rates, and bytes held."""
    w = work(case)
    held = w["bytes"]
    if case["op"] == "tree":          # the plain form lays the caches out side by side, float32
        held = 16 * case["seqs"] * (case["hi"] + case["qhi"]) * case["kv"] * (case["d"] + case["qhi"] * case["heads"] // case["kv"])
    return w["flops"] / RATE[case["dt"]] + w["bytes"] / 4e12, held


def draw(rng):
    limit = _cost(next(c for c in listed() if c["name"] == "prompt_8k"))[0]
    while True:
        case = _draw_once(rng)
        seconds, held = _cost(case)
        if seconds <= limit and held <= 8e9:
            return case


# ---------------------------------------------------------------------------
# sizes that follow from a case alone
# ---------------------------------------------------------------------------

def _lengths(case, lo, hi, salt=0):
    """One length a sequence in [lo, hi]; the first is the longest there is."""
    r = random.Random(case["shape"] * 7 + salt)
    n = [r.randint(lo, hi) for _ in range(case["seqs"])]
    n[0] = hi
    return n


def _paths(case):
    """Accepted path of every sequence: the first tokens of one of its chains (chain-major order)."""
    r = random.Random(case["shape"])
    out = []
    for _ in range(case["seqs"]):
        chain, m = r.randrange(case["chains"]), r.randint(0, case["depth"])
        out.append([chain * case["depth"] + i for i in range(m)])
    out[0] = [(case["chains"] - 1) * case["depth"] + i for i in range(case["depth"])]
    return out


def _past(case, lo):
    """Tokens that every sequence has in the cache before."""
    r = random.Random(case["shape"] * 7 + 2)
    return [r.randint(lo, case["past"]) for _ in range(case["seqs"])]


def work(case):
    op, es, d = case["op"], ESZ[case["dt"]], case["d"]
    if op == "rotary":      # turned heads read and written, positions read
        t = case["tokens"]
        return {"bytes": t * (2 * case["heads"] * d * es + 4), "flops": 3 * t * case["heads"] * case["rot"]}
    if op == "append":      # query, key and value rows read, written; position, sequence and slot read
        t = sum(_lengths(case, case["lo"], case["hi"]))
        h = case["heads"] + 2 * case["kv"]
        return {"bytes": t * (2 * h * d * es + 12), "flops": 3 * t * (case["heads"] + case["kv"]) * case["rot"]}
    if op == "prompt":      # every visible (query, key) pair: two products of d; q, k, v read, the result written
        n = _lengths(case, case["lo"], case["hi"])
        pairs = sum(m * (m + 1) // 2 for m in n)
        return {"bytes": sum(n) * (2 * case["heads"] + 2 * case["kv"]) * d * es, "flops": 4 * pairs * d * case["heads"]}
    if op == "tree":        # keys and values of every sequence read once, queries read, results written
        n, q = _lengths(case, case["lo"], case["hi"]), _lengths(case, case["qlo"], case["qhi"], 1)
        keys = sum(a + b for a, b in zip(n, q))
        return {"bytes": keys * 2 * case["kv"] * d * es + sum(q) * 2 * case["heads"] * d * es,
                "flops": 4 * sum(b * a for a, b in zip(n, q)) * d * case["heads"]}
    t = sum(len(p) for p in _paths(case))
    return {"bytes": max(t, 1) * 4 * case["kv"] * d * es * case["layers"], "flops": 0}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


def _offsets(n):
    out = [0]
    for m in n:
        out.append(out[-1] + m)
    return out


def _pages(need, page, rng):
    """A page table for sequences of `need` tokens: pages dealt out in random order, some free; unused
    entries -1."""
    per = [(m + page - 1) // page for m in need]
    total = sum(per) + 3
    order = list(range(total))
    rng.shuffle(order)
    width, table, at = max(per), [], 0
    for n in per:
        table.append(order[at:at + n] + [-1] * (width - n))
        at += n
    return table, total


def _rotary_args(case):
    return dict(head_dim=case["d"], rot_dim=case["rot"], layout=case["layout"], base=500000.0 if case["d"] == 128 else 10000.0,
                scaling=case["scaling"], factor=case["factor"], context=8192)


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * seed + 17)
    rng = random.Random(seed)
    dt, d, op = TDT[case["dt"]], case["d"], case["op"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV, dtype=dt)

    st = dict(case=case)
    if op in ("rotary", "append"):
        st["args"] = _rotary_args(case)
    if op == "rotary":
        t, heads = case["tokens"], case["heads"]
        rows = normal(t, (heads + case["rest"]) * d)
        st.update(x=rows[:, :heads * d].view(t, heads, d), y=torch.zeros(t, heads, d, device=DEV, dtype=dt),
                  pos=_ints([case["far"] + i for i in range(t)]))
    elif op == "append":
        n, heads, kv, page = _lengths(case, case["lo"], case["hi"]), case["heads"], case["kv"], case["page"]
        past = _past(case, 0)
        t = sum(n)
        rows = normal(t, (heads + 2 * kv) * d).view(t, heads + 2 * kv, d)
        table, pages = _pages([a + b for a, b in zip(n, past)], page, rng)
        seq = [s for s, m in enumerate(n) for _ in range(m)]
        slot = [past[s] + i for s, m in enumerate(n) for i in range(m)]
        st.update(q=rows[:, :heads], k=rows[:, heads:heads + kv], v=rows[:, heads + kv:],
                  q_out=torch.zeros(t, heads, d, device=DEV, dtype=dt), pos=_ints(slot), seq=_ints(seq), slot=_ints(slot),
                  kc=torch.zeros(pages, kv, page, d, device=DEV, dtype=dt),
                  vc=torch.zeros(pages, kv, page, d, device=DEV, dtype=dt), table=_ints(table))
    elif op == "prompt":
        n, heads, kv = _lengths(case, case["lo"], case["hi"]), case["heads"], case["kv"]
        t = sum(n)
        rows = normal(t, (heads + 2 * kv) * d).view(t, heads + 2 * kv, d)
        rows[:, :heads] *= torch.linspace(0.5, 2.0, heads, device=DEV).to(dt)[None, :, None]   # flat and peaked heads
        st.update(q=rows[:, :heads], k=rows[:, heads:heads + kv], v=rows[:, heads + kv:], n=n,
                  out=torch.zeros(t, heads, d, device=DEV, dtype=dt), offsets=_ints(_offsets(n)))
    elif op == "tree":
        n, m = _lengths(case, case["lo"], case["hi"]), _lengths(case, case["qlo"], case["qhi"], 1)
        heads, kv, page, t = case["heads"], case["kv"], case["page"], sum(m)
        table, pages = _pages([a + b for a, b in zip(n, m)], page, rng)
        words = (max(m) + 63) // 64
        rows = []                 # ancestors of every drafted token, itself among them
        for c in m if case["tree"] else []:
            anc = []
            for i in range(c):
                anc.append((anc[rng.randint(max(0, i - 9), i - 1)] if i else 0) | (1 << i))
            rows += anc
        mask = None
        if case["tree"]:
            word = (1 << 64) - 1
            mask = [[(a >> (64 * w)) & word for w in range(words)] for a in rows]
            mask = _ints([[v - (1 << 64) if v >> 63 else v for v in r] for r in mask], torch.int64)
        q = normal(t, heads, d)
        q *= torch.linspace(0.5, 2.0, heads, device=DEV).to(dt)[None, :, None]
        st.update(q=q, out=torch.zeros_like(q), kc=normal(pages, kv, page, d), vc=normal(pages, kv, page, d), table=_ints(table),
                  offsets=_ints(_offsets(m)), lens=_ints(n), m=m, n=n, mask=mask)
    else:
        paths, kv, page, layers = _paths(case), case["kv"], case["page"], case["layers"]
        past = _past(case, 1)
        table, pages = _pages([p + case["chains"] * case["depth"] for p in past], page, rng)
        st.update(kc=normal(layers, pages, kv, page, d), vc=normal(layers, pages, kv, page, d), table=_ints(table),
                  lens=_ints(past), offsets=_ints(_offsets([len(p) for p in paths])),
                  path=_ints([i for p in paths for i in p] or [0]), max_path=max(len(p) for p in paths),
                  seq=_ints([s for s, p in enumerate(paths) for _ in p], torch.int64),
                  rank=_ints([i for p in paths for i in range(len(p))], torch.int64))
    if own:
        import paper_2404_02445_amd as P
        if "args" in st:
            st["rotary"] = P.Rotary(**st["args"])
        if "kc" in st:
            st["cache"] = P.PagedCache(st["kc"], st["vc"], st["table"])
        if op == "tree":
            st["ws"] = P.alloc_attention_workspace(st["q"], st["cache"], max(st["m"]), max(st["n"]) + max(st["m"]))
    return st


# ---------------------------------------------------------------------------
# the plain form
# ---------------------------------------------------------------------------

def _frequencies(a):
    """Angle per position of every pair, float64, and the factor on sines and cosines."""
    r, base, f = a["rot_dim"], a["base"], a["factor"]
    j = torch.arange(r // 2, device=DEV, dtype=torch.float64)
    if a["scaling"] == "ntk":
        base = base * f ** (r / (r - 2))
    w = base ** (-2.0 * j / r)
    if a["scaling"] == "linear":
        w = w / f
    if a["scaling"] != "yarn":
        return w, 1.0
    keep = ((a["context"] * w / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)     # 1 to 32 turns in the context
    return w * keep + w / f * (1.0 - keep), 0.1 * math.log(f) + 1.0


def _turn(a, x, pos):
    """Rotary positions of x [tokens, heads, d], float32."""
    r = a["rot_dim"]
    w, m = _frequencies(a)
    ang = pos.double()[:, None] * w[None]
    c, s = (torch.cos(ang) * m).float()[:, None], (torch.sin(ang) * m).float()[:, None]
    y = x.float().clone()
    if a["layout"] == "half":
        p, q = x[..., :r // 2].float(), x[..., r // 2:r].float()
        y[..., :r // 2], y[..., r // 2:r] = p * c - q * s, q * c + p * s
    else:
        p, q = x[..., 0:r:2].float(), x[..., 1:r:2].float()
        y[..., 0:r:2], y[..., 1:r:2] = p * c - q * s, q * c + p * s
    return y


def _softmax(s, visible):
    """Softmax over the last dimension of the visible entries; rows without any give zeros."""
    s = torch.where(visible, s, torch.full_like(s, -math.inf))
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total == 0, torch.ones_like(total), total)


def _plain_prompt(st):
    c, at = st["case"], 0
    group, scale = c["heads"] // c["kv"], c["d"] ** -0.5
    for n in st["n"]:
        q, k, v = (st[x][at:at + n].float().transpose(0, 1) for x in "qkv")              # [heads, n, d]
        k, v = k.repeat_interleave(group, 0), v.repeat_interleave(group, 0)
        for lo in range(0, n, 2048):
            hi = min(n, lo + 2048)
            seen = torch.arange(hi, device=DEV)[None] <= torch.arange(lo, hi, device=DEV)[:, None]
            p = _softmax(torch.matmul(q[:, lo:hi], k[:, :hi].transpose(1, 2)) * scale, seen)
            st["out"][at + lo:at + hi] = torch.matmul(p, v[:, :hi]).transpose(0, 1).to(st["out"].dtype)
        at += n
    return st["out"]


def _plain_tree(st):
    c, n, m = st["case"], st["n"], st["m"]
    seqs, kv, d, page, group = c["seqs"], c["kv"], c["d"], c["page"], c["heads"] // c["kv"]
    top_q = max(m)
    length = st["table"].shape[1] * page
    rows = st["table"].clamp(min=0).long()
    k = st["kc"][rows].float().permute(0, 2, 1, 3, 4).reshape(seqs, kv, length, d)
    v = st["vc"][rows].float().permute(0, 2, 1, 3, 4).reshape(seqs, kv, length, d)
    # drafted rows side by side, padded to the longest
    row = st["offsets"][:-1].long()[:, None] + torch.arange(top_q, device=DEV)[None]
    real = torch.arange(top_q, device=DEV)[None] < (st["offsets"][1:] - st["offsets"][:-1])[:, None]
    row = torch.where(real, row, torch.zeros_like(row))
    q = st["q"][row].float().view(seqs, top_q, kv, group, d).permute(0, 2, 1, 3, 4).reshape(seqs, kv, top_q * group, d)
    s = torch.matmul(q, k.transpose(2, 3)) * d ** -0.5
    key = torch.arange(length, device=DEV)[None]
    draft = key - st["lens"][:, None]                                                     # [seqs, length]
    if st["mask"] is None:
        own_draft = draft[:, None] <= torch.arange(top_q, device=DEV)[None, :, None]
    else:
        bits = st["mask"][row]                                                            # [seqs, top_q, words]
        at = draft.clamp(0, 64 * bits.shape[2] - 1)[:, None].expand(-1, top_q, -1)
        own_draft = (torch.gather(bits, 2, at // 64) >> (at % 64)) & 1 == 1
    visible = (draft < 0)[:, None] | (own_draft & (draft >= 0)[:, None] & (draft[:, None] < real.sum(1)[:, None, None]))
    visible = visible[:, None, :, None].expand(seqs, kv, top_q, group, length).reshape(seqs, kv, top_q * group, length)
    o = torch.matmul(_softmax(s, visible), v)
    o = o.view(seqs, kv, top_q, group, d).permute(0, 2, 1, 3, 4).reshape(seqs, top_q, kv * group, d)
    st["out"].copy_(o[real].to(st["out"].dtype))
    return st["out"]


def _place(st, seq, slot):
    page = st["case"]["page"]
    return st["table"][seq, slot // page].long(), slot % page


def run(state):
    op = state["case"]["op"]
    if own:
        import paper_2404_02445_amd as P
        if op == "rotary":
            P.mopar_rotary_apply(state["rotary"], state["x"], state["y"], state["pos"])
            return state["y"]
        if op == "append":
            P.mopar_cache_append(state["cache"], state["k"], state["v"], state["seq"], state["slot"], rotary=state["rotary"],
                                 pos=state["pos"], q=state["q"], q_out=state["q_out"])
            return state["q_out"], state["kc"], state["vc"]
        if op == "prompt":
            return P.mopar_attention_prompt(state["q"], state["k"], state["v"], state["out"], state["offsets"], max(state["n"]))
        if op == "tree":
            return P.mopar_attention_cache(state["q"], state["out"], state["cache"], state["offsets"], max(state["m"]), state["lens"],
                                           max(state["n"]) + max(state["m"]), mask=state["mask"], ws=state["ws"])
        P.mopar_cache_keep(state["cache"], state["lens"], state["offsets"], state["path"], state["max_path"])
        return state["kc"], state["vc"]
    if op == "rotary":
        state["y"].copy_(_turn(state["args"], state["x"], state["pos"]))
        return state["y"]
    if op == "append":
        page, at = _place(state, state["seq"].long(), state["slot"].long())
        dt = state["kc"].dtype
        state["q_out"].copy_(_turn(state["args"], state["q"], state["pos"]))
        state["kc"][page, :, at] = _turn(state["args"], state["k"], state["pos"]).to(dt)
        state["vc"][page, :, at] = state["v"]
        return state["q_out"], state["kc"], state["vc"]
    if op == "prompt":
        return _plain_prompt(state)
    if op == "tree":
        return _plain_tree(state)
    seq, rank = state["seq"], state["rank"]
    past = state["lens"][seq].long()
    src, src_at = _place(state, seq, past + state["path"][:seq.numel()].long())
    dst, dst_at = _place(state, seq, past + rank)
    for x in (state["kc"], state["vc"]):
        x[:, dst, :, dst_at] = x[:, src, :, src_at]
    return state["kc"], state["vc"]


# ---------------------------------------------------------------------------
# the definitions in float64
# ---------------------------------------------------------------------------

def _rotate64(a, x, pos):
    """Each pair (x_p, x_q) as a complex number times m exp(i pos w)."""
    r, out = a["rot_dim"], x.double().clone()
    for j in range(r // 2):
        if a["scaling"] == "ntk":
            w = (a["base"] * a["factor"] ** (r / (r - 2))) ** (-2 * j / r)
        else:
            w = a["base"] ** (-2 * j / r)
        m = 1.0
        if a["scaling"] == "linear":
            w /= a["factor"]
        if a["scaling"] == "yarn":
            turns = a["context"] * w / (2 * math.pi)
            ramp = min(1.0, max(0.0, (turns - 1) / 31))
            w, m = w * ramp + (w / a["factor"]) * (1 - ramp), 1 + 0.1 * math.log(a["factor"])
        ang = pos.double() * w
        z = torch.polar(torch.full_like(ang, m), ang)[:, None]
        p, q = (j, j + r // 2) if a["layout"] == "half" else (2 * j, 2 * j + 1)
        t = torch.complex(x[..., p].double(), x[..., q].double()) * z
        out[..., p], out[..., q] = t.real, t.imag
    return out


def _attend64(q, k, v, hidden, scale):
    """One head: q [a, d], k and v [b, d], hidden [a, b] True where a row does not see a key."""
    s = (q @ k.T) * scale
    s[hidden] = -math.inf
    s = s - s.max(1, keepdim=True).values.nan_to_num(neginf=0.0)
    p = s.exp_()
    den = p.sum(1, keepdim=True)
    return (p @ v) / torch.where(den > 0, den, 1.0)


def exact(case, seed):
    st, op = prepare(case, seed), case["op"]
    if op == "rotary":
        return _rotate64(st["args"], st["x"], st["pos"])
    if op == "append":
        kc, vc = st["kc"].double(), st["vc"].double()
        k, seq, slot, table = _rotate64(st["args"], st["k"], st["pos"]), st["seq"].tolist(), st["slot"].tolist(), st["table"].tolist()
        where = torch.tensor([table[s][i // case["page"]] * case["page"] + i % case["page"] for s, i in zip(seq, slot)], device=DEV)
        for pool, rows in ((kc, k), (vc, st["v"].double())):
            for h in range(case["kv"]):
                flat = pool[:, h].reshape(-1, case["d"])
                flat[where] = rows[:, h]
                pool[:, h] = flat.view(pool.shape[0], case["page"], case["d"])
        return _rotate64(st["args"], st["q"], st["pos"]), kc, vc
    if op in ("prompt", "tree"):
        group, scale = case["heads"] // case["kv"], 1 / math.sqrt(case["d"])
        out, at, lens = st["out"].double(), 0, st["n"]
        new = st["n"] if op == "prompt" else st["m"]
        if sum(a * b for a, b in zip(lens, new)) * case["heads"] * case["d"] > 6e12:
            return None
        for s, (n, m) in enumerate(zip(lens, new)):
            if op == "prompt":
                k, v = st["k"][at:at + n].double(), st["v"][at:at + n].double()
                hidden = torch.ones(n, n, dtype=torch.bool, device=DEV).triu_(1)
            else:
                pages = [p for p in st["table"][s].tolist() if p >= 0]
                k, v = (torch.cat([st[x][p].double().transpose(0, 1) for p in pages])[:n + m] if len(pages) < 64 else
                        st[x][torch.tensor(pages, device=DEV)].double().transpose(1, 2).flatten(0, 1)[:n + m] for x in ("kc", "vc"))
                hidden = torch.zeros(m, n + m, dtype=torch.bool, device=DEV)
                if st["mask"] is None:
                    hidden[:, n:] = torch.ones(m, m, dtype=torch.bool, device=DEV).triu_(1)
                else:
                    rows = [[(w & ((1 << 64) - 1)) for w in r] for r in st["mask"][at:at + m].tolist()]
                    hidden[:, n:] = torch.tensor([[not (r[j // 64] >> (j % 64)) & 1 for j in range(m)] for r in rows], device=DEV)
            for h in range(case["heads"]):
                out[at:at + m, h] = _attend64(st["q"][at:at + m, h].double(), k[:, h // group], v[:, h // group], hidden, scale)
            at += m
        return out
    kc, vc, table, lens = st["kc"].double(), st["vc"].double(), st["table"].tolist(), st["lens"].tolist()
    for pool in (kc, vc):           # each accepted row in turn, first to last
        for s, path in enumerate(_paths(case)):
            at = [divmod(lens[s] + i, case["page"]) for i in range(case["chains"] * case["depth"] + 1)]
            for i, j in enumerate(path):
                pool[:, table[s][at[i][0]], :, at[i][1]] = pool[:, table[s][at[j][0]], :, at[j][1]]
    return kc, vc
