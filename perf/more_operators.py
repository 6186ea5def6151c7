"""Timing cases of the operators that a decode step with drafted tokens adds to a served block.

Three operators: attention of a tree of drafted tokens over the paged 4-bit cache;
verification of the drafted tokens against the target's probabilities, from given random
numbers; keeping the accepted path's tokens in the cache.  Model widths, head counts and
vocabularies are those of the repository's own workloads, or generic.

``own`` selects the side: False computes each operator in plain form, in 32 bits (the
verification, whose comparisons decide about whole numbers, in 64); True calls the package.
"""
import math

import torch

own = False

DEV = "cuda"
GROUP = 64                    # cache elements that share a scale and a minimum
DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ---- cases --------------------------------------------------------------------
# A tree is given by its branching, level by level: "3.2.1" is a root with three children,
# each of these with two, each of those with one.  Nodes are numbered level by level.
def _tree(B, tree, ctx, Hq, Hkv, D, page, dtype="bf16", window=0, ragged=False, name=None):
    c = dict(op="tree", B=B, tree=tree, ctx=ctx, Hq=Hq, Hkv=Hkv, D=D, page=page, dtype=dtype, window=window,
             ragged=ragged)
    return dict(c, name=name) if name else c


def _verify(B, tree, V, dtype="bf16", draft=True, heat="one", pad=0, masked=0.0, ragged=False, name=None):
    c = dict(op="verify", B=B, tree=tree, V=V, dtype=dtype, draft=draft, heat=heat, pad=pad, masked=masked,
             ragged=ragged)
    return dict(c, name=name) if name else c


def _keep(layers, B, tree, ctx, Hkv, D, page, ragged=False, name=None):
    c = dict(op="keep", layers=layers, B=B, tree=tree, ctx=ctx, Hkv=Hkv, D=D, page=page, ragged=ragged)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one request of the 4096-wide model with a chain of four drafted tokens
        _tree(1, "1.1.1.1", 517, 32, 32, 128, 64, name="tree-1x5"),
        # a decode batch over prompt and generated tokens, a small tree each
        _tree(8, "3.2.1", 2304, 64, 8, 128, 64, name="tree-8x16"),
        # the same batch with long contexts, few drafted tokens
        _tree(8, "2.1.1", 65536, 64, 8, 128, 64, name="tree-8x7-65536"),
        # the widest tree, 16 query heads to a cached one
        _tree(2, "9.3.1", 16384, 128, 8, 128, 64, name="tree-2x64-16384"),
        # sliding-window block, ragged lengths and trees (empty ones among them), odd heads
        _tree(13, "2.2.1", 1500, 21, 3, 64, 16, dtype="f16", window=128, ragged=True, name="tree-window-ragged"),
        # one request's chain, the smallest vocabulary
        _verify(1, "1.1.1.1", 32000, name="verify-1x5"),
        # a decode batch, a small tree each
        _verify(8, "3.2.1", 128256, name="verify-8x16"),
        # many requests with chains, 32-bit logits, a temperature
        _verify(64, "1.1.1.1.1.1.1", 128256, dtype="f32", heat="warm", name="verify-64x8-f32"),
        # drafts without probabilities, greedy requests among them, odd rows, forbidden tokens
        _verify(13, "4.2", 50001, dtype="f16", draft=False, heat="mixed", pad=3, masked=0.1, ragged=True,
                name="verify-nodraft-odd"),
        # one layer of one request
        _keep(1, 1, "3.2.1", 517, 32, 128, 64, name="keep-1layer"),
        # every layer of the 80-layer model, the whole batch
        _keep(80, 8, "3.2.1", 517, 8, 128, 64, name="keep-80layers"),
        # small heads and pages, ragged trees
        _keep(7, 13, "4.2.2", 333, 3, 64, 16, ragged=True, name="keep-odd"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_tree(rng, most, chains=0.4):
    """A branching of 2 to `most` nodes: a chain, or wide at the top."""
    if rng.random() < chains:
        return ".".join(["1"] * rng.randint(1, min(most, 12) - 1))
    levels = [rng.randint(2, 6)]
    for _ in range(rng.randint(0, 4)):
        b = rng.randint(1, max(1, 6 // (1 + len(levels))))
        if _count(levels + [b]) > most:
            break
        levels.append(b)
    return ".".join(map(str, levels))


def draw(rng):
    op = rng.choice(["tree", "tree", "verify", "verify", "keep"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    if op == "verify":
        tree = _draw_tree(rng, 64)
        B, V = _log_int(rng, 1, 64), _log_int(rng, 1000, 128256)
        while B * _count(_levels(tree)) * V > 64 * 8 * 128256:
            B = max(1, B // 2)
            if B == 1:
                V = V // 2
        return _verify(B, tree, V, rng.choice(["bf16", "f16", "f32"]), rng.random() < 0.7,
                       rng.choice(["one", "warm", "mixed"]), rng.choice([0, 0, 3, 8]), rng.choice([0.0, 0.0, 0.1, 0.9]),
                       rng.random() < 0.5)
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 3, 8, 8, 32])
    page = rng.choice([16, 32, 64, 128])
    if op == "keep":
        layers, B = _log_int(rng, 1, 80), _log_int(rng, 1, 32)
        tree = _draw_tree(rng, 64, 0)        # (of a chain's path every token is in its place)
        ctx = 64 + _log_int(rng, 1, 600)
        while layers * B * ctx * Hkv * D > 80 * 8 * 517 * 8 * 128:
            layers, B = max(1, layers // 2), max(1, B // 2)
        return _keep(layers, B, tree, ctx, Hkv, D, page, rng.random() < 0.5)
    G = rng.choice([1, 2, 5, 7, 8, 16]) if Hkv <= 8 else 1
    tree = _draw_tree(rng, 64)
    new = _count(_levels(tree))
    B, ctx = _log_int(rng, 1, 16), new + _log_int(rng, 1, 65536)
    # (the plain form holds every score of the padded batch, and the whole batch in 32 bits)
    while B * new * Hkv * G * ctx > 2 * 64 * 128 * 16384 or B * ctx * Hkv * D > 8 * 65536 * 8 * 128:
        if B > 1:
            B //= 2
        else:
            ctx = new + (ctx - new) // 2
    return _tree(B, tree, ctx, Hkv * G, Hkv, D, page, dtype, rng.choice([0, 0, 128, 333]), rng.random() < 0.5)


# ---- trees ----------------------------------------------------------------------
def _levels(tree):
    return [int(b) for b in tree.split(".")]


def _count(levels):
    n = width = 1
    for b in levels:
        width *= b
        n += width
    return n


def _parents(tree):
    """The parent of each node, -1 for the root."""
    out, level = [-1], [0]
    for b in _levels(tree):
        below = []
        for p in level:
            for _ in range(b):
                below.append(len(out))
                out.append(p)
        level = below
    return out


def _sizes(case):
    """Cached tokens and nodes of each request (a tree's first nodes are a tree)."""
    B, ctx, new = case["B"], case.get("ctx", 1 << 30), _count(_levels(case["tree"]))
    if not case.get("ragged"):
        return [ctx] * B, [new] * B
    lens, news = [], []
    for b in range(B):
        n = 1 + (b * 5 + new - 1) % new
        if b % 4 == 3:                       # an empty request, or one that starts with its one token
            n = (b // 4) % 2
            lens.append(n)
        else:
            lens.append(max(n, ctx - (b * 7919) % max(1, ctx)))
        news.append(n)
    return lens, news


# ---- inputs -------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


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


def _batch(case, s):
    lens, news = _sizes(case)
    starts = [0]
    for n in news:
        starts.append(starts[-1] + n)
    par = _parents(case["tree"])
    s["starts"], s["max_new"] = _i32(starts), max(news)
    s["parents"] = _i32([par[i] for n in news for i in range(n)])
    if "ctx" in case:
        s["lens"], s["max_len"] = _i32(lens), max(lens)
    return lens, news, starts, par


def _inputs(case, seed):
    g, op = _gen(seed), case["op"]
    s = dict(case=case)
    lens, news, starts, par = _batch(case, s)
    T = starts[-1]
    if op == "verify":
        V, dt = case["V"], DTYPES[case["dtype"]]
        shape = (T, V + case["pad"])
        x = 3 * torch.randn(*shape, generator=g, device=DEV)
        # a draft model that is near the target: it accepts some four tokens in five
        y = x + 0.5 * torch.randn(*shape, generator=g, device=DEV)
        if case["masked"]:
            hide = torch.rand(*shape, generator=g, device=DEV) < case["masked"]
            x.masked_fill_(hide, -math.inf)
            y.masked_fill_(hide, -math.inf)
        heats = {"one": [1.0], "warm": [0.8], "mixed": [0.0, 0.7, 1.3]}[case["heat"]]
        heats = [heats[b % len(heats)] for b in range(case["B"])]
        s["temperature"] = None if case["heat"] == "one" else torch.tensor(heats, device=DEV)
        s["logits"], y = x.to(dt)[:, :V], y.to(dt)[:, :V]
        # tokens drawn from the draft's rows of their parents, or the best of them in turn
        parent = [starts[b] + max(0, par[i]) for b, n in enumerate(news) for i in range(n)]
        if case["draft"]:
            s["draft"] = y
            t = torch.tensor([max(heats[b], 1e-3) for b, n in enumerate(news) for _ in range(n)], device=DEV)
            s["tokens"] = torch.empty(T, dtype=torch.int32, device=DEV)
            for r in range(0, T, 64):
                rows = torch.tensor(parent[r:r + 64], device=DEV)
                noise = -torch.log(-torch.log(torch.rand(len(rows), V, generator=g, device=DEV).clamp(1e-20, 1 - 1e-7)))
                s["tokens"][r:r + 64] = (y[rows].float() / t[r:r + 64, None] + noise).argmax(1).int()
        else:
            s["draft"] = None
            rank = [i - par.index(par[i]) for n in news for i in range(n)]
            best = torch.topk(y.float(), max(_levels(case["tree"])), dim=1).indices
            s["tokens"] = best[torch.tensor(parent, device=DEV), torch.tensor(rank, device=DEV)].int()
        s["uniforms"] = torch.rand(T, generator=g, device=DEV)
        return s
    B, Hkv, D, page = case["B"], case["Hkv"], case["D"], case["page"]
    s["table"], total = _pages(g, B, max(case["ctx"], max(lens), 1), page)
    s["kv"], shape = {}, (case.get("layers", 1), total, Hkv, page)
    for n in ("k", "v"):
        s["kv"][n + "_codes"] = torch.randint(0, 256, (*shape, D // 2), generator=g, device=DEV, dtype=torch.uint8)
        s["kv"][n + "_scales"] = _scales(g, *shape, D // GROUP)
    if op == "tree":
        s["q"] = torch.randn(T, case["Hq"], D, generator=g, device=DEV).to(DTYPES[case["dtype"]])
        return s
    # accepted paths.  Of a pass that is made again each token still has to be where it was: one that
    # moves does not lie where another goes.
    pick = torch.randint(0, 1 << 20, (B, 1 + len(_levels(case["tree"]))), generator=g, device=DEV).tolist()
    nodes = [[-1] * s["max_new"] for _ in range(B)]
    s["kept"] = []
    for b, n in enumerate(news):
        path = [0] if n else []
        while path and len(path) < len(pick[b]):
            below = [i for i in range(n) if par[i] == path[-1]]
            if not below:
                break
            path.append(below[pick[b][len(path)] % len(below)])
        while any(i != k and i < len(path) for k, i in enumerate(path)):
            path.pop()
        nodes[b][:len(path)] = path
        s["kept"].append(len(path))
    s["moves"] = [(b, k, i) for b in range(B) for k, i in enumerate(nodes[b][:s["kept"][b]]) if i != k]
    s["kept"], s["nodes"] = _i32(s["kept"]), _i32(nodes)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own and case["op"] != "verify":        # the handles that a program keeps: views of the same tensors
        from paper_2606_03770_gb300 import ops
        kv = s["kv"]
        s["caches"] = [ops.Cache(*layer) for layer in zip(kv["k_codes"], kv["k_scales"], kv["v_codes"], kv["v_scales"])]
        if case["op"] == "keep":
            s["caches"] = ops.CacheLayers(s["caches"])
    return s


# ---- the operators ------------------------------------------------------------
def run(s):
    op = s["case"]["op"]
    if own:
        return _own(op, s)
    return {"tree": _plain_tree, "verify": _plain_verify, "keep": _plain_keep}[op](s)


def _own(op, s):
    from paper_2606_03770_gb300 import ops
    if op == "tree":
        return ops.cache_attend_tree(s["caches"][0], s["q"], s["parents"], s["table"], s["lens"], s["starts"],
                                     max_new=s["max_new"], max_len=s["max_len"], window=s["case"]["window"])
    if op == "verify":
        kept, nodes, ids = ops.verify_drafts(s["logits"], s["tokens"], s["parents"], s["starts"], s["uniforms"],
                                             draft=s["draft"], temperature=s["temperature"], max_new=s["max_new"])
        return dict(kept=kept, nodes=nodes, ids=ids)
    lens = ops.cache_keep(s["caches"], s["table"], s["lens"], s["starts"], s["nodes"], s["kept"])
    return dict(lens=lens, **s["kv"])


def _unpack(codes):
    """Two codes to a byte, the lower four bits first."""
    return torch.stack([codes & 15, codes >> 4], -1).flatten(-2)


def _plain_gather(s, n):
    """A request's pages side by side: [B][Hkv][keys][D], in 32 bits."""
    t = s["table"].long()
    q = _unpack(s["kv"][n + "_codes"][0][t]).float().unflatten(-1, (-1, GROUP))
    sm = s["kv"][n + "_scales"][0][t].float()
    return (q * sm[..., :1] + sm[..., 1:]).flatten(-2).transpose(1, 2).flatten(2, 3)


def _padded(s, x, fill):
    """[tokens] as [B][max_new], and which of them there are."""
    starts = s["starts"].long()
    i = torch.arange(s["max_new"], device=x.device)
    live = i < (starts[1:] - starts[:-1])[:, None]
    at = (starts[:-1, None] + i).clamp(max=max(0, x.shape[0] - 1))
    return torch.where(live, x[at], fill), live, at


def _plain_tree(s):
    c = s["case"]
    Hkv, D = c["Hkv"], c["D"]
    q, lens = s["q"], s["lens"].long()
    parent, live, at = _padded(s, s["parents"].long(), -1)
    news = live.sum(1)
    i = torch.arange(s["max_new"], device=q.device)
    # which nodes are on a node's way up: the parents' matrix, doubled until the longest way is covered
    up = (parent[..., None] == i) | (i[:, None] == i)            # [B][node][ancestor or itself]
    for _ in range(max(1, (s["max_new"] - 1).bit_length())):
        up = (up.float() @ up.float()) > 0
    depth = up.sum(-1) - 1
    x = q[at].float() * live[..., None, None]                    # [B][new][Hq][D]
    x = x.unflatten(2, (Hkv, -1)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    a = x @ _plain_gather(s, "k").transpose(2, 3) * (1 / math.sqrt(D))
    a = a.unflatten(2, (s["max_new"], -1))                       # [B][Hkv][new][G][keys]
    key = torch.arange(a.shape[-1], device=q.device)
    base = (lens - news)[:, None, None]
    place = key - base                                           # [B][1][keys]: a node's, from 0 on
    node = place.clamp(0, s["max_new"] - 1).expand(-1, s["max_new"], -1)
    on_way = up.gather(2, node) & (place >= 0) & (place < news[:, None, None])
    see = (place < 0) | on_way
    if c["window"]:
        stands = torch.where(place < 0, key, base + depth[:, None].expand(-1, s["max_new"], -1).gather(2, node))
        see = see & (stands > base + depth[..., None] - c["window"])
    a = a.masked_fill(~(see & live[..., None])[:, None, :, None], -math.inf)
    top = a.amax(-1, keepdim=True)
    e = torch.exp(a - torch.where(top > -math.inf, top, 0.0))
    total = e.sum(-1, keepdim=True)
    e = e / torch.where(total > 0, total, 1.0)
    o = e.flatten(2, 3) @ _plain_gather(s, "v")
    o = o.unflatten(2, (s["max_new"], -1)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    return o[live].to(q.dtype)


def _plain_softmax(x, heat):
    """Rows of probabilities in 64 bits; heat 0: all on the first of the largest."""
    x = x.double()
    hi = x.amax(-1, keepdim=True)
    e = torch.exp((x - hi) / torch.where(heat > 0, heat, 1.0)[:, None])
    first = (x == hi) & ((x == hi).cumsum(-1) == 1)
    e = torch.where(heat[:, None] > 0, e, first.double())
    return e / e.sum(-1, keepdim=True)


def _plain_verify(s):
    c, W = s["case"], s["max_new"]
    B, V = c["B"], c["V"]
    parent, live, at = _padded(s, s["parents"].long(), -2)
    token, uniform = s["tokens"].long()[at], s["uniforms"].double()[at]
    heat = torch.ones(B, device=DEV) if s["temperature"] is None else s["temperature"]
    heat = heat.double()
    b = torch.arange(B, device=DEV)
    here = torch.zeros(B, dtype=torch.long, device=DEV)          # the node that the walk has come to
    kept = live[:, 0].long()
    nodes = torch.full((B, W + 1), -1, dtype=torch.long, device=DEV)
    ids = torch.full((B, W + 1), -1, dtype=torch.long, device=DEV)
    nodes[:, 0] = torch.where(live[:, 0], 0, -1)
    p = _plain_softmax(s["logits"][at[:, 0]], heat)
    q = _plain_softmax(s["draft"][at[:, 0]], heat) if c["draft"] else None
    for i in range(1, W):
        asked = live[:, i] & (parent[:, i] == here)
        x, u = token[:, i], uniform[:, i]
        is_x = torch.arange(V, device=DEV) == x[:, None]
        # (greedy: the drafted token is all of the draft's)
        d = torch.where(heat[:, None] > 0, q, is_x.double()) if c["draft"] else is_x.double()
        takes = asked & (u * d[b, x] < p[b, x])
        rest = (p - d).clamp_min(0) if c["draft"] else torch.where(is_x, 0.0, p)
        total = rest.sum(-1, keepdim=True)
        rest = torch.where(total > 0, rest / torch.where(total > 0, total, 1.0), p)
        p = torch.where(takes[:, None], _plain_softmax(s["logits"][at[:, i]], heat), torch.where(asked[:, None], rest, p))
        if c["draft"]:
            q = torch.where(takes[:, None], _plain_softmax(s["draft"][at[:, i]], heat), q)
        here = torch.where(takes, i, here)
        ids[b, torch.where(takes, kept - 1, W)] = x
        nodes[b, torch.where(takes, kept, W)] = i
        kept = kept + takes
    # the token whose share of the sums in order holds the random number
    sums = p.cumsum(-1)
    last = (p > 0).long().mul(torch.arange(V, device=DEV)).amax(-1)
    drawn = torch.minimum((sums <= uniform[:, :1] * sums[:, -1:]).sum(-1), last)
    ids[b, torch.where(live[:, 0], kept - 1, W)] = drawn
    return dict(kept=kept.int(), nodes=nodes[:, :W].int(), ids=ids[:, :W].int())


def _plain_keep(s):
    c = s["case"]
    starts, lens = s["starts"].long(), s["lens"].long()
    base = lens - (starts[1:] - starts[:-1])
    k = torch.arange(s["max_new"], device=DEV)
    moved = k < s["kept"][:, None]
    last = s["table"].shape[1] * c["page"] - 1
    old = (base[:, None] + s["nodes"]).clamp(0, last)[moved]
    new = (base[:, None] + k).clamp(0, last)[moved]
    of = torch.arange(c["B"], device=DEV)[:, None].expand_as(moved)[moved]
    page = s["table"].long()
    for x in s["kv"].values():
        x[:, page[of, new // c["page"]], :, new % c["page"]] = x[:, page[of, old // c["page"]], :, old % c["page"]]
    return dict(lens=(base + s["kept"]).int(), **s["kv"])


# ---- what a pass cannot do without --------------------------------------------
def work(case):
    op = case["op"]
    lens, news = _sizes(case)
    par = _parents(case["tree"])
    depth = [0] * len(par)
    for i in range(1, len(par)):
        depth[i] = depth[par[i]] + 1
    if op == "verify":
        # The rows of the nodes that the walk comes to: some four drafted tokens in five are accepted where the
        # draft's probabilities are given, one in four where the best few are drafted.  A row's exponentials and sums.
        size, share = 4 if case["dtype"] == "f32" else 2, 0.8 if case["draft"] else 0.25
        rows = 0.0
        for n in news:
            deepest = depth[n - 1] if n else -1
            rows += sum(share ** k * (2 if case["draft"] and k < deepest else 1) for k in range(deepest + 1))
        return {"bytes": int(rows * case["V"] * size) + 12 * sum(news) + 8 * case["B"] * max(news),
                "flops": int(5 * rows * case["V"])}
    Hkv, D = case["Hkv"], case["D"]
    token = 2 * Hkv * (D // 2 + 4 * (D // GROUP))          # a token's keys and values
    if op == "keep":
        # (half of the drafted levels, the first of them where it was)
        moved = case["layers"] * sum(max(0, depth[n - 1]) / 2 for n in news if n)
        return {"bytes": int(2 * moved * token) + 4 * case["B"] * (max(news) + 4), "flops": 0}
    w, pairs, keys = case["window"], 0, 0
    for length, n in zip(lens, news):
        base = length - n
        for i in range(n):
            pairs += min(base, max(0, w - 1 - depth[i])) + min(depth[i] + 1, w) if w else base + depth[i] + 1
        if n:
            keys += (min(base, w - 1) if w else base) + n
    return {"bytes": keys * token + 4 * sum(news) * case["Hq"] * D, "flops": 4 * D * case["Hq"] * pairs}


# ---- 64 bits ------------------------------------------------------------------
def exact(case, seed):
    return {"tree": _exact_tree, "verify": _exact_verify, "keep": _exact_keep}[case["op"]](case, _inputs(case, seed))


def _exact_codes(b):
    out = torch.empty(*b.shape[:-1], 2 * b.shape[-1], dtype=torch.float64, device=b.device)
    out[..., 0::2] = (b % 16).double()
    out[..., 1::2] = (b // 16).double()
    return out


def _exact_tree(case, s):
    lens, news = _sizes(case)
    D, page, G, w = case["D"], case["page"], case["Hq"] // case["Hkv"], case["window"]
    par, kv = _parents(case["tree"]), {n: x[0] for n, x in s["kv"].items()}
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    t = 0
    for b, (length, n) in enumerate(zip(lens, news)):
        if not n:
            continue
        base = length - n
        ways = []
        for i in range(n):
            way = [i]
            while par[way[-1]] >= 0:
                way.append(par[way[-1]])
            ways.append(way)
        # seen keys: of the context from `first` on, of the nodes as listed
        see = torch.zeros(n, length, dtype=torch.bool)
        for i, way in enumerate(ways):
            deep = len(way) - 1
            see[i, max(0, base + deep - w + 1) if w else 0:base] = True
            for a in way[:w] if w else way:
                see[i, base + a] = True
        see = see.to(DEV)
        pages = s["table"][b, :-(-length // page)].long()
        for h in range(case["Hkv"]):
            k, v = [(lambda sm, c: (sm[..., 1:] + sm[..., :1] * c).reshape(-1, D)[:length])(
                kv[x + "_scales"][pages, h].double().reshape(-1, D // GROUP, 2),
                _exact_codes(kv[x + "_codes"][pages, h]).reshape(-1, D // GROUP, GROUP)) for x in ("k", "v")]
            q = s["q"][t:t + n, h * G:(h + 1) * G].double()
            a = torch.einsum("igd,kd->igk", q, k) / math.sqrt(D)
            a = a.masked_fill(~see[:, None], -math.inf)
            out[t:t + n, h * G:(h + 1) * G] = torch.softmax(a, -1) @ v
        t += n
    return out


def _exact_verify(case, s):
    _, news = _sizes(case)
    par, W = _parents(case["tree"]), s["max_new"]
    tokens, uniforms = s["tokens"].tolist(), s["uniforms"].double().tolist()
    heats = [1.0] * case["B"] if s["temperature"] is None else s["temperature"].double().tolist()
    kept, nodes, ids = [], [], []
    start = 0
    for n, heat in zip(news, heats):
        path, got = [0] if n else [], []
        left = None                                              # what is left of the target's probabilities
        for i in range(n):
            if left is None:
                row = s["logits"][start + path[-1]].double()
                if heat > 0:
                    left = torch.softmax(row / heat, 0)
                    of = torch.softmax(s["draft"][start + path[-1]].double() / heat, 0) if case["draft"] else None
                else:
                    best = int(torch.nonzero(row == row.max())[0])
            if i == 0 or par[i] != path[-1]:
                left = left if heat > 0 else 0
                continue
            x = tokens[start + i]
            if heat <= 0:
                takes = x == best
            elif of is not None:
                takes = uniforms[start + i] * float(of[x]) < float(left[x])
            else:
                takes = uniforms[start + i] < float(left[x])
            if takes:
                path.append(i)
                got.append(x)
                left = None
            elif heat > 0:
                rest = left.clone()
                if of is not None:
                    rest = torch.relu(left - of)
                else:
                    rest[x] = 0
                if float(rest.sum()) > 0:
                    left = rest / rest.sum()
        if n:
            row = s["logits"][start + path[-1]].double()
            if heat <= 0:
                got.append(int(torch.nonzero(row == row.max())[0]))
            else:
                left = torch.softmax(row / heat, 0) if left is None else left
                sums = torch.cumsum(left, 0)
                at = int(torch.searchsorted(sums, uniforms[start] * sums[-1:], right=True)[0])
                got.append(min(at, int(torch.nonzero(left > 0)[-1])))
        kept.append(len(path))
        nodes.append(path + [-1] * (W - len(path)))
        ids.append(got + [-1] * (W - len(got)))
        start += n
    return dict(kept=_i32(kept), nodes=_i32(nodes), ids=_i32(ids))


def _exact_keep(case, s):
    lens, news = _sizes(case)
    page, table = case["page"], s["table"].tolist()
    for x in s["kv"].values():
        old = x.clone()
        for b, k, i in s["moves"]:
            to, at = lens[b] - news[b] + k, lens[b] - news[b] + i
            x[:, table[b][to // page], :, to % page] = old[:, table[b][at // page], :, at % page]
    kept = s["kept"].tolist()
    return dict(lens=_i32([l - n + k for l, n, k in zip(lens, news, kept)]), **s["kv"])
