"""The block operators in 64 bits, from their formulas, with bounds on how far a
correct 32-bit computation may be off."""
import math

import torch

F64 = torch.float64
EPS32 = 2.0 ** -24                                     # relative error of one rounding to 32 bits
EPS = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: EPS32}
TINY16 = 2.0 ** -24                                    # fp16's smallest step


def unpack(codes):
    out = torch.empty(*codes.shape[:-1], 2 * codes.shape[-1], dtype=F64, device=codes.device)
    out[..., 0::2] = (codes & 15).to(F64)
    out[..., 1::2] = (codes >> 4).to(F64)
    return out


def weight(w):
    c = unpack(w.codes)
    s = w.scales.to(F64).repeat_interleave(w.group, 1)
    return (c - 8) * s if w.mins is None else c * s + w.mins.to(F64).repeat_interleave(w.group, 1)


def matmul(x, w, residual=None, gated=False):
    """(result, bound).  A product of K terms whose weights may be rounded to
    fp16 once and whose sums are in 32 bits: (2^-11 + K 2^-24) sum |x| |W|."""
    W, X = weight(w), x.to(F64)
    y = X @ W.T
    off = (2.0 ** -11 + w.cols * EPS32) * (X.abs() @ W.abs().T)
    if gated:
        n = w.rows // 2
        a, b, da, db = y[:, :n], y[:, n:], off[:, :n], off[:, n:]
        act = a * torch.sigmoid(a)
        # |silu'| <= 1.1; a few roundings of exp and the division
        off = 1.1 * da * (b.abs() + db) + act.abs() * db + 32 * EPS32 * (act * b).abs()
        y = act * b
    if residual is not None:
        y = y + residual.to(F64)
    return y, off + EPS[x.dtype] * (y.abs() + off) + TINY16


def rotate(x, cos, sin, interleaved):
    """The turn as the header rounds it: each product and sum to 32 bits."""
    rot = 2 * cos.shape[1]
    x = x.float().clone()
    i = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
    j = i + 1 if interleaved else i + rot // 2
    a, b = x[..., i].clone(), x[..., j].clone()
    c, s = cos[:, None], sin[:, None]
    x[..., i] = (a * c) - (b * s)
    x[..., j] = (b * c) + (a * s)
    return x


def cache_pack(x):
    """Codes and (scale, minimum) of fp32 values, rounding as the header says."""
    g = x.unflatten(-1, (-1, 64))
    lo, hi = (f.clamp(-65504.0, 65504.0) for f in (g.amin(-1), g.amax(-1)))
    nan = torch.isnan(g).any(-1)
    m = torch.where(nan, math.nan, lo).half()
    # (by a tensor: a division by a Python number is a product with its reciprocal)
    d = torch.where(nan, 0.0, (hi - lo) / torch.full_like(lo, 15.0)).half()
    df = d.float()[..., None]
    q = torch.where(df > 0, torch.round((g - m.float()[..., None]) / torch.where(df > 0, df, 1.0)), 0.0)
    q = torch.nan_to_num(q, nan=0.0, posinf=15.0, neginf=0.0).clamp(0, 15).to(torch.uint8).flatten(-2)
    return q[..., 0::2] | (q[..., 1::2] << 4), torch.stack([d, m], -1)


def cache_values(codes, scales):
    c = unpack(codes).unflatten(-1, (-1, 64))
    s = scales.to(F64)
    return (c * s[..., :1] + s[..., 1:]).flatten(-2)


def attend(cache, q, table, lens, starts, scale, window):
    """(result, bound, written): written marks the tokens of some request.

    Scores are off by at most ds = scale (2^-11 + (D + 4) 2^-24) sum |q| |k| (keys
    possibly rounded to fp16), so a weight by exp(2 ds); weights and values may
    be rounded to fp16 (2^-11 each) and are summed in 32 bits."""
    T, Hq, D = q.shape
    out = torch.zeros(T, Hq, D, dtype=F64, device=q.device)
    off = torch.zeros_like(out)
    written = torch.zeros(T, dtype=torch.bool, device=q.device)
    G = Hq // cache.kv_heads
    for r in range(table.shape[0]):
        s0, s1, n = int(starts[r]), int(starts[r + 1]), int(lens[r])
        for t in range(max(s0, 0), min(s1, T)):
            written[t] = True
            pos = n - (s1 - t)
            first = max(0, pos - window + 1) if window else 0
            end = min(pos + 1, table.shape[1] * cache.page_size)
            j = torch.arange(first, max(first, end), device=q.device)
            if not j.numel():
                continue
            page = table[r].long()[j // cache.page_size]
            ok = (page >= 0) & (page < cache.pages)
            j, page = j[ok], page[ok]
            if not j.numel():
                continue
            at = j % cache.page_size
            k = cache_values(cache.k_codes[page, :, at], cache.k_scales[page, :, at])
            v = cache_values(cache.v_codes[page, :, at], cache.v_scales[page, :, at])
            for h in range(Hq):
                x = q[t, h].to(F64)
                a = k[:, h // G] @ x * scale
                p = torch.softmax(a, 0)
                out[t, h] = p @ v[:, h // G]
                ds = (abs(scale) * (2.0 ** -11 + (D + 4) * EPS32) * (k[:, h // G].abs() @ x.abs())).max()
                mag = p @ v[:, h // G].abs() + v[:, h // G].abs().max() * 2.0 ** -14
                off[t, h] = (torch.expm1(2 * ds) + 2.0 ** -9 + (j.numel() + 64) * EPS32) * mag
    return out, off + EPS[q.dtype] * (out.abs() + off) + TINY16, written


def logprobs(x, tokens, top):
    """The formulas in 64 bits, with bounds for sums over chains of V/128 + 64
    terms in 32 bits."""
    x = x.to(F64)
    V = x.shape[1]
    bad = torch.isnan(x).any(1) | (x == math.inf).any(1)
    hi = x.amax(1)
    empty = hi == -math.inf
    base = torch.where(empty | bad, 0.0, hi)[:, None]
    z = torch.where(bad[:, None], 0.0, x - base)
    e = torch.exp(z)
    s = e.sum(1)
    lse = torch.where(empty, 0.0, base[:, 0] + torch.log(torch.where(s > 0, s, 1.0)))
    p = e / torch.where(s > 0, s, 1.0)[:, None]
    dot = (p * torch.where(e > 0, z, 0.0)).sum(1)
    ent = torch.where(empty, 0.0, torch.log(torch.where(s > 0, s, 1.0)) - dot)
    ok = (tokens >= 0) & (tokens < V)
    lp = x.gather(1, tokens.long().clamp(0, V - 1)[:, None])[:, 0] - lse
    lp = torch.where(empty, -math.inf, lp)
    lp = torch.where(bad | ~ok, math.nan, lp)
    n = min(top, V)
    vals, ids = torch.sort(torch.where(bad[:, None], 0.0, x), dim=1, descending=True, stable=True)
    vals = torch.nn.functional.pad(vals[:, :n], (0, top - n), value=-math.inf)
    ids = torch.nn.functional.pad(ids[:, :n], (0, top - n), value=-1)
    none = (vals == -math.inf) | bad[:, None]
    ids = torch.where(none, -1, ids).to(torch.int32)
    vals = torch.where(bad[:, None], math.nan, torch.where(none, -math.inf, vals - lse[:, None]))
    chain = (V / 128 + 64) * EPS32
    dl = chain + 8 * EPS32 * (1 + lse.abs())
    de = 2 * chain * (1 + dot.abs()) + 8 * EPS32 * (1 + ent.abs())
    return lp, torch.where(bad, math.nan, ent), vals, ids, dl, de


def close(got, want, bound, what=""):
    """Every finite value within its bound, every other one equal."""
    got = got.to(F64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fin = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    other = ~fin & ~torch.isnan(want)
    assert torch.equal(got[other], want[other]), f"{what}: infinities in other places"
    err = (got - want).abs()[fin]
    lim = bound.expand_as(want)[fin]
    bad = err > lim
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {err.numel()} off, worst {float((err / lim.clamp_min(1e-300)).max()):.3g} bounds"
