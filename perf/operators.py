"""Timing cases of the operators that a served decoder block is made of.

Four operators: products with 4-bit weights and group scales; appending keys and
values to a paged 4-bit cache, with the position rotation on the way (and reading
tokens of it back); attention over that cache; log probabilities of given tokens
with entropy and top alternatives.  Model widths, head counts, vocabularies, prompt
lengths and the window are those of the repository's own workloads, or generic.

``own`` selects the side: False computes each operator in plain form, in 32 bits;
True calls the package.
"""
import math

import torch

own = False

DEV = "cuda"
GROUP = 64                    # cache elements that share a scale and a minimum
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---- cases --------------------------------------------------------------------
def _product(T, N, K, group=64, dtype="bf16", mins=False, gated=False, residual=False, name=None):
    c = dict(op="product", T=T, N=N, K=K, group=group, dtype=dtype, mins=mins, gated=gated, residual=residual)
    return dict(c, name=name) if name else c


def _append(B, new, ctx, Hq, Hkv, D, page, dtype="bf16", interleaved=False, rot=None, name=None):
    c = dict(op="append", B=B, new=new, ctx=ctx, Hq=Hq, Hkv=Hkv, D=D, page=page, dtype=dtype,
             interleaved=interleaved, rot=D if rot is None else rot)
    return dict(c, name=name) if name else c


def _attend(B, new, ctx, Hq, Hkv, D, page, dtype="bf16", window=0, ragged=False, name=None):
    c = dict(op="attend", B=B, new=new, ctx=ctx, Hq=Hq, Hkv=Hkv, D=D, page=page, dtype=dtype, window=window,
             ragged=ragged)
    return dict(c, name=name) if name else c


def _logprobs(T, V, top, dtype="bf16", pad=0, masked=0.0, name=None):
    c = dict(op="logprobs", T=T, V=V, top=top, dtype=dtype, pad=pad, masked=masked)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token through the attention output of the 4096-wide model, added to the residual stream
        _product(1, 4096, 4096, residual=True, name="product-1tok-4096"),
        # the largest decode batch through the gated half of the 8192-wide model's MLP
        _product(8, 28672, 8192, gated=True, name="product-8tok-gated-8192"),
        # odd sizes, minima beside the scales, small groups, half precision
        _product(5, 1001, 1376, group=32, dtype="f16", mins=True, name="product-5tok-odd"),
        # a prompt of mean length through the way back down
        _product(1152, 8192, 28672, group=128, residual=True, name="product-prompt-1152"),
        # one new token for each of eight requests
        _append(8, 1, 2304, 64, 8, 128, 64, name="append-8x1"),
        # the longest prompt of the 8192-wide workload
        _append(1, 2048, 2048, 64, 8, 128, 64, name="append-prompt-2048"),
        # the decode batch over prompt and generated tokens
        _attend(8, 1, 2304, 64, 8, 128, 64, name="attend-8x2304"),
        # long contexts, 16 query heads to a cached one
        _attend(8, 1, 65536, 128, 8, 128, 64, name="attend-8x65536"),
        # sliding-window block, ragged lengths (0 and 1 among them), several tokens at once, odd heads
        _attend(13, 3, 1500, 21, 3, 64, 16, dtype="f16", window=128, ragged=True, name="attend-window-ragged"),
        # a prompt attending to itself and to what came before it
        _attend(1, 1152, 2304, 64, 8, 128, 64, name="attend-prompt-1152"),
        # the head's logits of a decode batch, with alternatives
        _logprobs(8, 128256, 5, name="logprobs-8tok"),
        # scoring a prompt, odd rows, some tokens forbidden
        _logprobs(1152, 128256, 20, dtype="f32", pad=3, masked=0.1, name="logprobs-prompt-1152"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["product", "product", "append", "attend", "attend", "logprobs"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if op == "product":
        group = rng.choice([32, 64, 128])
        T, N = _log_int(rng, 1, 1152), _log_int(rng, 64, 28672)
        K = group * max(1, _log_int(rng, 256, 28672) // group)
        gated = rng.random() < 0.3
        while T * N * K * (2 if gated else 1) > 1152 * 8192 * 28672:
            T = max(1, T // 2)
        return _product(T, N, K, group, dtype, rng.random() < 0.5, gated, rng.random() < 0.3)
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 3, 8, 8, 32])
    G = rng.choice([1, 2, 5, 7, 8, 16]) if Hkv <= 8 else 1
    page = rng.choice([16, 32, 64, 128])
    if op == "append":
        B, new = _log_int(rng, 1, 32), _log_int(rng, 1, 2048)
        while B * new * Hkv * (G + 2) * D > 2048 * 80 * 128:
            B, new = max(1, B // 2), max(1, new // 2)
        ctx = new + _log_int(rng, 1, 1000)
        return _append(B, new, ctx, Hkv * G, Hkv, D, page, dtype, rng.random() < 0.3,
                       rng.choice([D, D, D // 2]))
    if op == "attend":
        kind = rng.choice(["one", "one", "few", "prompt"])
        B = _log_int(rng, 1, 16)
        new = {"one": 1, "few": rng.randint(2, 9), "prompt": _log_int(rng, 16, 1152)}[kind]
        ctx = new + _log_int(rng, 1, 65536)
        # (the plain form holds every score of the padded batch, and the whole batch in 32 bits)
        while B * new * Hkv * G * ctx > 1152 * 64 * 2304 or B * ctx * Hkv * D > 8 * 65536 * 8 * 128:
            B, ctx = max(1, B // 2), max(new, ctx // 2)
            new = min(new, ctx) if ctx > new or new == 1 else new // 2
        return _attend(B, new, ctx, Hkv * G, Hkv, D, page, dtype, rng.choice([0, 0, 128, 333]),
                       rng.random() < 0.5)
    T, V = _log_int(rng, 1, 1152), _log_int(rng, 1000, 128256)
    return _logprobs(T, V, rng.choice([0, 1, 5, 20, 32]), rng.choice(["bf16", "f16", "f32"]),
                     rng.choice([0, 0, 3, 8]), rng.choice([0.0, 0.0, 0.1, 0.9]))


# ---- inputs -------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _bytes(g, *shape):
    return torch.randint(0, 256, shape, generator=g, device=DEV, dtype=torch.uint8)


def _lengths(case):
    """Cached tokens and new tokens of each request (plain lists)."""
    B, new, ctx = case["B"], case["new"], case["ctx"]
    if not case.get("ragged"):
        return [ctx] * B, [new] * B
    lens, news = [], []
    for b in range(B):
        n = 1 + (b * 5) % new
        if b % 4 == 3:                       # an empty request, or one that starts
            n = (b // 4) % 2
            lens.append(n)
        else:
            lens.append(max(n, ctx - (b * 7919) % max(1, ctx)))
        news.append(n)
    return lens, news


def _scales(g, *shape):
    """Scale and minimum of cached groups: values of about unit variance, some groups off centre."""
    s = 0.15 + 0.25 * torch.rand(*shape, generator=g, device=DEV)
    m = -7.5 * s + 0.5 * torch.randn(*shape, generator=g, device=DEV)
    return torch.stack([s, m], -1).half()


def _pages(g, B, ctx, page):
    """A table of pages in shuffled order, with a few pages that no request holds."""
    per = -(-ctx // page)
    total = B * per + 3
    order = torch.randperm(total, generator=g, device=DEV)[:B * per]
    return order.reshape(B, per).to(torch.int32).contiguous(), total


def _table(n, rot):
    """Cosines and sines of position x frequency, as a model keeps them."""
    inv = 10000.0 ** (-torch.arange(rot // 2, device=DEV, dtype=torch.float64) * 2 / rot)
    ang = torch.arange(n, device=DEV, dtype=torch.float64)[:, None] * inv
    return ang.cos().float().contiguous(), ang.sin().float().contiguous()


def _inputs(case, seed):
    g, op = _gen(seed), case["op"]
    dt = DTYPES[case["dtype"]]
    s = dict(case=case)
    if op == "product":
        T, N, K = case["T"], case["N"], case["K"]
        rows, G = (2 * N if case["gated"] else N), K // case["group"]
        s["x"] = _randn(g, T, K, dtype=dt)
        s["codes"] = _bytes(g, rows, K // 2)
        s["scales"] = ((0.5 + torch.rand(rows, G, generator=g, device=DEV)) * (0.2 / math.sqrt(K))).half()
        s["mins"] = (-(6 + 3 * torch.rand(rows, G, generator=g, device=DEV)) * s["scales"]).half() \
            if case["mins"] else None
        s["residual"] = _randn(g, T, N, dtype=dt) if case["residual"] else None
        return s
    if op == "logprobs":
        T, V, pad = case["T"], case["V"], case["pad"]
        x = (3 * torch.randn(T, V + pad, generator=g, device=DEV)).to(dt)
        if case["masked"]:
            hide = torch.rand(T, V + pad, generator=g, device=DEV) < case["masked"]
            x.masked_fill_(hide, -math.inf)
        s["logits"] = x[:, :V]
        s["tokens"] = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
        return s
    B, Hq, Hkv, D, page = case["B"], case["Hq"], case["Hkv"], case["D"], case["page"]
    lens, news = _lengths(case)
    T = sum(news)
    s["table"], total = _pages(g, B, max(case["ctx"], 1), page)
    s["q"] = _randn(g, T, Hq, D, dtype=dt)
    shape = (total, Hkv, page)
    if op == "append":
        s["k"] = (_randn(g, T, Hkv, D) + 2 * _randn(g, 1, Hkv, D)).to(dt)
        s["v"] = _randn(g, T, Hkv, D, dtype=dt)
        at = torch.cat([torch.arange(l - n, l, device=DEV) for l, n in zip(lens, news)])
        of = torch.cat([torch.full((n,), b, device=DEV) for b, n in enumerate(news)])
        s["positions"] = at.to(torch.int32)
        s["slots"] = s["table"].long()[of, at // page] * page + at % page
        s["cos"], s["sin"] = _table(case["ctx"], case["rot"])
        s["q_out"] = torch.empty_like(s["q"])
        for n in ("k", "v"):
            s[n + "_codes"] = torch.zeros(*shape, D // 2, dtype=torch.uint8, device=DEV)
            s[n + "_scales"] = torch.zeros(*shape, D // GROUP, 2, dtype=torch.float16, device=DEV)
        return s
    for n in ("k", "v"):
        s[n + "_codes"] = _bytes(g, *shape, D // 2)
        s[n + "_scales"] = _scales(g, *shape, D // GROUP)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    s["starts"] = torch.tensor(starts, dtype=torch.int32, device=DEV)
    s["max_new"], s["max_len"] = max(news), max(lens)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:                                   # the handles that a program keeps: views of the same tensors
        from paper_2606_03770_gb300 import ops
        if case["op"] == "product":
            s["w"] = ops.QuantWeight(s["codes"], s["scales"], s["mins"])
        elif case["op"] in ("append", "attend"):
            s["cache"] = ops.Cache(s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"])
    return s


# ---- the operators ------------------------------------------------------------
def run(s):
    op = s["case"]["op"]
    if own:
        return _own(op, s)
    return {"product": _plain_product, "append": _plain_append, "attend": _plain_attend,
            "logprobs": _plain_logprobs}[op](s)


def _own(op, s):
    from paper_2606_03770_gb300 import ops
    c = s["case"]
    if op == "product":
        return ops.quant_matmul(s["x"], s["w"], residual=s["residual"], gated=c["gated"])
    if op == "append":
        ops.cache_append(s["cache"], s["k"], s["v"], s["slots"], s["positions"], s["cos"], s["sin"], q=s["q"],
                         q_out=s["q_out"], interleaved=c["interleaved"])
        k, v = ops.cache_read(s["cache"], s["slots"], dtype=s["k"].dtype)
        return dict(q=s["q_out"], k=k, v=v)
    if op == "attend":
        return ops.cache_attend(s["cache"], s["q"], s["table"], s["lens"], s["starts"], max_new=s["max_new"],
                                max_len=s["max_len"], window=c["window"])
    logprob, entropy, values, ids = ops.token_logprobs(s["logits"], s["tokens"], top=c["top"])
    return dict(logprob=logprob, entropy=entropy, values=values, ids=ids)


def _unpack(codes):
    """Two codes to a byte, the lower four bits first."""
    return torch.stack([codes & 15, codes >> 4], -1).flatten(-2)


def _plain_product(s):
    c = s["case"]
    g = c["group"]
    q = _unpack(s["codes"]).float().unflatten(1, (-1, g))
    sc = s["scales"].float()[..., None]
    w = q * sc + s["mins"].float()[..., None] if s["mins"] is not None else (q - 8) * sc
    y = s["x"].float() @ w.flatten(1).T
    if c["gated"]:
        a, b = y[:, :c["N"]], y[:, c["N"]:]
        y = a / (1 + torch.exp(-a)) * b
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(s["x"].dtype)


def _plain_rotate(x, cos, sin, interleaved):
    rot = 2 * cos.shape[-1]
    x = x.float()
    r, rest = x[..., :rot], x[..., rot:]
    a, b = (r[..., 0::2], r[..., 1::2]) if interleaved else (r[..., :rot // 2], r[..., rot // 2:])
    cos, sin = cos[:, None], sin[:, None]
    a, b = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([r, rest], -1)


def _plain_append(s):
    c = s["case"]
    at = s["positions"].long()
    cos, sin = s["cos"][at], s["sin"][at]
    s["q_out"].copy_(_plain_rotate(s["q"], cos, sin, c["interleaved"]).to(s["q"].dtype))
    page, slot = s["k_codes"].shape[2], s["slots"]
    p, o = slot // page, slot % page
    k = _plain_rotate(s["k"], cos, sin, c["interleaved"])
    for n, x in (("k", k), ("v", s["v"].float())):
        x = x.unflatten(-1, (-1, GROUP))
        lo, hi = x.amin(-1), x.amax(-1)
        m, sc = lo.half(), ((hi - lo) / 15).half()
        d = sc.float()[..., None]
        q = torch.where(d > 0, torch.round((x - m.float()[..., None]) / d).clamp(0, 15), 0.0).to(torch.uint8)
        q = q.flatten(-2)
        s[n + "_codes"][p, :, o] = q[..., 0::2] | (q[..., 1::2] << 4)
        s[n + "_scales"][p, :, o] = torch.stack([sc, m], -1)
    return dict(q=s["q_out"], k=_plain_read(s, "k", p, o), v=_plain_read(s, "v", p, o))


def _plain_read(s, n, p, o):
    q = _unpack(s[n + "_codes"][p, :, o]).float().unflatten(-1, (-1, GROUP))
    sm = s[n + "_scales"][p, :, o].float()
    return (q * sm[..., :1] + sm[..., 1:]).flatten(-2).to(s[n].dtype)


def _plain_gather(s, n):
    """A request's pages side by side: [B][Hkv][keys][D], in 32 bits."""
    t = s["table"].long()
    q = _unpack(s[n + "_codes"][t]).float().unflatten(-1, (-1, GROUP))
    sm = s[n + "_scales"][t].float()
    return (q * sm[..., :1] + sm[..., 1:]).flatten(-2).transpose(1, 2).flatten(2, 3)


def _plain_attend(s):
    c = s["case"]
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    q, lens, starts = s["q"], s["lens"].long(), s["starts"].long()
    news = starts[1:] - starts[:-1]
    i = torch.arange(s["max_new"], device=q.device)
    live = i < news[:, None]                                     # [B][new]
    at = (starts[:-1, None] + i).clamp(max=max(0, q.shape[0] - 1))
    x = q[at].float() * live[..., None, None]                    # [B][new][Hq][D]
    x = x.unflatten(2, (Hkv, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    a = x @ _plain_gather(s, "k").transpose(2, 3) * (1 / math.sqrt(D))
    a = a.unflatten(2, (s["max_new"], -1))                       # [B][Hkv][new][G][keys]
    key = torch.arange(a.shape[-1], device=q.device)
    pos = ((lens - news)[:, None] + i)[..., None]                # [B][new][1]
    see = (key <= pos) & live[..., None]
    if c["window"]:
        see = see & (key > pos - c["window"])
    a = a.masked_fill(~see[:, None, :, None], -math.inf)
    top = a.amax(-1, keepdim=True)
    e = torch.exp(a - torch.where(top > -math.inf, top, 0.0))
    total = e.sum(-1, keepdim=True)
    e = e / torch.where(total > 0, total, 1.0)
    o = e.flatten(2, 3) @ _plain_gather(s, "v")
    o = o.unflatten(2, (s["max_new"], -1)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    return o[live].to(q.dtype)


def _plain_logprobs(s):
    x, top = s["logits"].float(), s["case"]["top"]
    hi = x.amax(-1, keepdim=True)
    hi = torch.where(hi > -math.inf, hi, 0.0)
    e = torch.exp(x - hi)
    total = e.sum(-1, keepdim=True)
    lse = hi + torch.log(total)
    entropy = (lse - (e * torch.where(e > 0, x, 0.0)).sum(-1, keepdim=True) / total)[:, 0]
    logprob = (x.gather(1, s["tokens"].long()[:, None]) - lse)[:, 0]
    # the stable order puts equal values by their index
    values, ids = torch.sort(x, dim=-1, descending=True, stable=True)
    values, ids = values[:, :top], ids[:, :top]
    ids = torch.where(values > -math.inf, ids, -1).to(torch.int32)
    return dict(logprob=logprob, entropy=entropy, values=values - lse, ids=ids)


# ---- what a pass cannot do without --------------------------------------------
def _pairs(case):
    """Visible (query, key) pairs and keys that some query sees, over all requests."""
    pairs = keys = 0
    w = case["window"]
    for length, n in zip(*_lengths(case)):
        first = length - n
        for p in (range(first, length) if w else ()):
            pairs += min(w, p + 1)
        if not w:
            pairs += n * (first + 1 + length) // 2
        if n:
            keys += length if not w else min(length, n + w - 1)
    return pairs, keys


def work(case):
    op = case["op"]
    size = 4 if case["dtype"] == "f32" else 2
    if op == "product":
        T, N, K = case["T"], case["N"], case["K"]
        rows = 2 * N if case["gated"] else N
        weights = rows * K // 2 + rows * (K // case["group"]) * 2 * (2 if case["mins"] else 1)
        return {"bytes": weights + size * T * (K + N * (2 if case["residual"] else 1)), "flops": 2 * T * rows * K}
    if op == "logprobs":
        T, V = case["T"], case["V"]
        return {"bytes": T * V * size + T * (12 + 8 * case["top"]), "flops": 5 * T * V}
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    token = Hkv * (D // 2 + 4 * (D // GROUP))              # a token's keys, or its values
    T = sum(_lengths(case)[1])
    if op == "append":
        # q, k, v in, q and the cache's tokens out; those back in, keys and values out
        return {"bytes": T * (4 * Hq * D + 8 * Hkv * D + 4 * token + 4 * case["rot"]),
                "flops": T * D * (3 * Hq + 13 * Hkv)}
    pairs, keys = _pairs(case)
    return {"bytes": 2 * keys * token + 4 * T * Hq * D, "flops": 4 * D * Hq * pairs}


# ---- 64 bits ------------------------------------------------------------------
def exact(case, seed):
    return {"product": _exact_product, "append": _exact_append, "attend": _exact_attend,
            "logprobs": _exact_logprobs}[case["op"]](case, _inputs(case, seed))


def _exact_codes(b):
    out = torch.empty(*b.shape[:-1], 2 * b.shape[-1], dtype=torch.float64, device=b.device)
    out[..., 0::2] = (b % 16).double()
    out[..., 1::2] = (b // 16).double()
    return out


def _exact_product(case, s):
    x, rows = s["x"].double(), s["codes"].shape[0]
    y = torch.empty(case["T"], rows, dtype=torch.float64, device=DEV)
    for r in range(0, rows, 2048):
        w = _exact_codes(s["codes"][r:r + 2048])
        sc = torch.repeat_interleave(s["scales"][r:r + 2048].double(), case["group"], 1)
        if s["mins"] is None:
            w = (w - 8.0) * sc
        else:
            w = w * sc + torch.repeat_interleave(s["mins"][r:r + 2048].double(), case["group"], 1)
        y[:, r:r + 2048] = x @ w.t()
    if case["gated"]:
        gate, up = y.split(case["N"], 1)
        y = gate * torch.sigmoid(gate) * up
    if s["residual"] is not None:
        y += s["residual"].double()
    return y


def _exact_append(case, s):
    T, rot, D = s["q"].shape[0], case["rot"], case["D"]
    at = s["positions"].long()
    ang = torch.complex(s["cos"][at].double(), s["sin"][at].double())[:, None]

    def rotate(x):
        y = x.double().clone()
        if case["interleaved"]:
            i, j = torch.arange(0, rot, 2), torch.arange(1, rot, 2)
        else:
            i, j = torch.arange(rot // 2), torch.arange(rot // 2, rot)
        z = torch.complex(y[..., i], y[..., j]) * ang
        y[..., i], y[..., j] = z.real, z.imag
        return y

    def cached(x):
        x = x.reshape(T, case["Hkv"], D // GROUP, GROUP)
        lo = x.min(-1, keepdim=True).values
        step = ((x.max(-1, keepdim=True).values - lo) / 15).half().double()
        lo = lo.half().double()
        n = torch.where(step > 0, torch.round((x - lo) / torch.where(step > 0, step, 1.0)), 0.0).clamp(0, 15)
        return (lo + n * step).reshape(T, case["Hkv"], D)

    return dict(q=rotate(s["q"]), k=cached(rotate(s["k"])), v=cached(s["v"].double()))


def _exact_attend(case, s):
    lens, news = _lengths(case)
    D, page, G = case["D"], case["page"], case["Hq"] // case["Hkv"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    t = 0
    for b, (length, n) in enumerate(zip(lens, news)):
        if not n:
            continue
        pages = s["table"][b, :-(-length // page)].long()
        first = max(0, length - n + 1 - case["window"]) if case["window"] else 0
        for h in range(case["Hkv"]):
            kv = []
            for name in ("k", "v"):
                sm = s[name + "_scales"][pages, h].double().reshape(-1, D // GROUP, 2)
                c = _exact_codes(s[name + "_codes"][pages, h]).reshape(-1, D // GROUP, GROUP)
                kv.append((sm[..., 1:] + sm[..., :1] * c).reshape(-1, D)[first:length])
            key = torch.arange(first, length, device=DEV)
            for i in range(0, n, 256):
                q = s["q"][t + i:t + min(n, i + 256), h * G:(h + 1) * G].double()
                pos = torch.arange(length - n + i, length - n + i + q.shape[0], device=DEV)
                a = torch.einsum("igd,kd->igk", q, kv[0]) / math.sqrt(D)
                hide = key[None] > pos[:, None]
                if case["window"]:
                    hide |= key[None] <= pos[:, None] - case["window"]
                a = a.masked_fill(hide[:, None], -math.inf)
                out[t + i:t + i + q.shape[0], h * G:(h + 1) * G] = torch.softmax(a, -1) @ kv[1]
        t += n
    return out


def _exact_logprobs(case, s):
    parts = []
    for r in range(0, case["T"], 64):
        x = s["logits"][r:r + 64].double()
        lp = x - torch.logsumexp(x, -1, keepdim=True)
        p = lp.exp()
        y = s["tokens"][r:r + 64].long()
        ent = -torch.where(p > 0, p * lp, 0.0).sum(-1)
        # equal values by their index: the order of (value, -index)
        order = torch.argsort(x, dim=-1, descending=True, stable=True)[:, :case["top"]]
        got = lp.gather(1, order)
        parts.append((lp[torch.arange(len(y), device=DEV), y], ent, got,
                      torch.where(got > -math.inf, order, -1).to(torch.int32)))
    return dict(zip(("logprob", "entropy", "values", "ids"), (torch.cat(p) for p in zip(*parts))))
