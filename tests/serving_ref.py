"""Plain float64 forms of decoding with a paged cache, on the CPU, and the bounds of what float32 arithmetic and
one rounding may differ from them."""
import math

import torch

HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def frequencies(r, base=10000.0, scaling="none", factor=1.0, context=0.0, slow=1.0, fast=32.0):
    j = torch.arange(r // 2, dtype=torch.float64)
    if scaling == "ntk":
        base = base * factor ** (r / (r - 2))
    w = base ** (-2 * j / r)
    if scaling == "linear":
        w = w / factor
    if scaling == "yarn":
        g = ((context * w / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
        w = w * (g + (1 - g) / factor)
    return w


def rotate(x, pos, r, layout="half", m=1.0, **freq):
    """x [tokens, heads, d] turned; float64.  Also the bound on |x| + |y| of each element's pair (0 where it passes)."""
    x = x.double().cpu()
    ang = pos.double().cpu()[:, None] * frequencies(r, **freq)[None]
    c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
    y, mag = x.clone(), torch.zeros_like(x)
    a, b = (slice(0, r // 2), slice(r // 2, r)) if layout == "half" else (slice(0, r, 2), slice(1, r, 2))
    y[..., a], y[..., b] = m * (x[..., a] * c - x[..., b] * s), m * (x[..., b] * c + x[..., a] * s)
    mag[..., a] = mag[..., b] = m * (x[..., a].abs() + x[..., b].abs())
    return y, mag


def rotate_tol(ref, mag, dtype, far=0):
    """Of a turned element: angle to float32 0.8 half steps, its factor 0.8, sine and cosine 2 each, m and its products
    2, the two products and the sum 2, of at most the pair's magnitude; then one rounding to the type.  The
    reference's own angles (float64) are off by up to 2^-52 of a position's."""
    return mag * (8 * 2.0 ** -24 + far * 2.0 ** -52) + ref.abs() * HALF_STEP[dtype] * 1.01


def attend(q, k, v, seen, scale):
    """q [a, H, d], k and v [b, Hk, d], seen [a, b]: float64 results, and the bound of their error in the type of q."""
    dtype, (a, heads, d), kvh = q.dtype, q.shape, k.shape[1]
    q, k, v = (t.double().cpu() for t in (q, k, v))
    out, tol = torch.zeros(a, heads, d, dtype=torch.float64), torch.zeros(a, heads, d, dtype=torch.float64)
    hidden = ~seen.cpu()
    n = max(k.shape[0], 1)
    for h in range(heads):
        kh, vh = k[:, h // (heads // kvh)], v[:, h // (heads // kvh)]
        if k.shape[0] == 0:
            continue
        s = (q[:, h] @ kh.T) * scale
        s[hidden] = -math.inf
        top = s.max(1, keepdim=True).values
        p = torch.exp(s - top.nan_to_num(neginf=0.0))
        p[hidden] = 0
        den = p.sum(1, keepdim=True)
        p = p / torch.where(den > 0, den, 1.0)
        # what is hidden takes no part, whatever it holds
        used = torch.where(hidden.all(0)[:, None], 0.0, vh)
        if torch.isfinite(used).all():
            o, mag = p @ used, p @ used.abs()
        else:
            o = torch.stack([(p[i][seen[i].cpu()][:, None] * vh[seen[i].cpu()]).sum(0) for i in range(a)])
            mag = o.abs()
        out[:, h] = o
        # scores: d products and sums of float32 and the factor, of at most sum |q k| scale; exponent; n weighted sums
        dots = (q[:, h].abs() @ torch.where(torch.isfinite(kh), kh, 0.0).abs().T) * scale
        dots[hidden] = 0
        es = ((d + 8) * 2.0 ** -24 * dots.max(1, keepdim=True).values)
        rel = 2 * es + (n + 64) * 2.0 ** -24
        if dtype == torch.bfloat16:
            rel = rel + 2.0 ** -8                    # weights rounded for the second product
        tol[:, h] = mag * rel * 1.01 + o.abs() * HALF_STEP[dtype] * 1.01
    return out, tol


def check(got, ref, tol, what=""):
    got = got.double().cpu()
    finite = torch.isfinite(ref)
    assert torch.equal(torch.isfinite(got), finite), f"{what}: finite results differ"
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), f"{what}: NaN results differ"
    assert torch.equal(got[~finite & ~torch.isnan(ref)], ref[~finite & ~torch.isnan(ref)]), f"{what}: infinities differ"
    err, lim = (got - ref).abs()[finite], tol[finite]
    worst = (err - lim).max() if err.numel() else torch.tensor(0.0)
    assert worst <= 1e-37, f"{what}: error {err[(err - lim).argmax()]:.3e} over {lim[(err - lim).argmax()]:.3e}"


def page_table(need, page, gen, spare=3):
    """Pages dealt out in random order for sequences of `need` slots; unused entries -1."""
    per = [-(-n // page) for n in need]
    total = sum(per) + spare
    order, width, table, at = torch.randperm(total, generator=gen).tolist(), max(max(per), 1), [], 0
    for n in per:
        table.append(order[at:at + n] + [-1] * (width - n))
        at += n
    return torch.tensor(table, dtype=torch.int32).reshape(len(need), width), total


def cache_rows(pool, table, s, n):
    """Slots 0 .. n - 1 of sequence s: [n, heads, d] (absent pages: zeros)."""
    page = pool.shape[2]
    rows = []
    for i in range(n):
        p = int(table[s, i // page])
        rows.append(pool[p, :, i % page] if 0 <= p < pool.shape[0] else torch.zeros_like(pool[0, :, 0]))
    return torch.stack(rows) if rows else pool.new_zeros(0, pool.shape[1], pool.shape[3])


def tree_mask(n, gen):
    """Ancestors, itself among them, of n drafted tokens in a random tree: bool [n, n] and int64 [n, words]."""
    anc = torch.zeros(n, n, dtype=torch.bool)
    for i in range(n):
        if i:
            anc[i] = anc[int(torch.randint(max(0, i - 9), i, (1,), generator=gen))]
        anc[i, i] = True
    return anc, pack_mask(anc, (n + 63) // 64)


def pack_mask(seen, words):
    out = torch.zeros(seen.shape[0], words, dtype=torch.int64)
    for j in range(seen.shape[1]):
        bit = 1 << (j % 64)
        out[:, j // 64] |= seen[:, j].long() * (bit - (1 << 64) if bit >> 63 else bit)
    return out
