"""The operators for drafted tokens in 64 bits, from their formulas."""
import math

import torch

import ops_reference as R

F64 = torch.float64


def parent_of(parents, start, i, tokens):
    t = start + i
    p = int(parents[t]) if 0 <= t < tokens else -1
    return p if 0 <= p < i else -1


def way(parents, start, i, tokens):
    """Node i and its ancestors, from itself up."""
    out = [i]
    while (p := parent_of(parents, start, out[-1], tokens)) >= 0:
        out.append(p)
    return out


def attend_tree(cache, q, parents, table, lens, starts, scale, window):
    """(result, bound, written), with R.attend's bounds, but that a weight is rounded to fp16 together with
    its value's scale d: of v = m + d code that is 2^-11 of |d code|, which |v| may be far below, and so 2^-11 of
    sum p |d code| in the sum."""
    T, Hq, D = q.shape
    out = torch.zeros(T, Hq, D, dtype=F64, device=q.device)
    off = torch.zeros_like(out)
    written = torch.zeros(T, dtype=torch.bool, device=q.device)
    G = Hq // cache.kv_heads
    parents = parents.tolist()
    for r in range(table.shape[0]):
        s0, s1, n = int(starts[r]), int(starts[r + 1]), int(lens[r])
        base = n - (s1 - s0)
        for t in range(max(s0, 0), min(s1, T)):
            written[t] = True
            up = way(parents, s0, t - s0, T)
            depth = len(up) - 1
            first = max(0, base + depth - window + 1) if window else 0
            keys = list(range(first, max(first, base)))
            keys += [base + a for d, a in enumerate(up) if (not window or d < window) and base + a >= 0]
            j = torch.tensor([k for k in keys if k < table.shape[1] * cache.page_size], dtype=torch.long, device=q.device)
            if not j.numel():
                continue
            page = table[r].long()[j // cache.page_size]
            ok = (page >= 0) & (page < cache.pages)
            j, page = j[ok], page[ok]
            if not j.numel():
                continue
            at = j % cache.page_size
            k = R.cache_values(cache.k_codes[page, :, at], cache.k_scales[page, :, at])
            v = R.cache_values(cache.v_codes[page, :, at], cache.v_scales[page, :, at])
            low = cache.v_scales[page, :, at][..., 1].to(F64).repeat_interleave(64, -1)
            x = q[t].to(F64).unflatten(0, (-1, G))                         # [heads][G][D]
            k, v, low = k.transpose(0, 1), v.transpose(0, 1), low.transpose(0, 1)
            p = torch.softmax(x @ k.transpose(1, 2) * scale, -1)
            out[t] = (p @ v).flatten(0, 1)
            ds = (abs(scale) * (2.0 ** -11 + (D + 4) * R.EPS32) * (x.abs() @ k.abs().transpose(1, 2))).amax(-1, keepdim=True)
            mag = p @ v.abs() + v.abs().amax((1, 2))[:, None, None] * 2.0 ** -14
            off[t] = ((torch.expm1(2 * ds) + 2.0 ** -9 + (j.numel() + 64) * R.EPS32) * mag
                      + 2.0 ** -11 * (p @ (v - low).abs())).flatten(0, 1)
    return out, off + R.EPS[q.dtype] * (out.abs() + off) + R.TINY16, written


def probabilities(row, heat):
    """64 bits, or None for a row without a distribution."""
    x = row.to(F64)
    hi = x.max()
    if bool(torch.isnan(x).any()) or not -math.inf < float(hi) < math.inf:
        return None
    w = torch.exp((x - hi) / heat)
    return w / w.sum()


def verify(logits, ids, parents, starts, uniforms, draft, temperature, max_new):
    """(kept, nodes, answer) as lists."""
    T, V = logits.shape
    ids, parents = ids.tolist(), parents.tolist()
    uniforms = [min(max(u, 0.0), 1.0) if u == u else 0.0 for u in uniforms.to(F64).tolist()]
    out = []
    for r in range(len(starts) - 1):
        s0, s1 = int(starts[r]), int(starts[r + 1])
        n = max(0, min(s1 - s0, max_new)) if s0 >= 0 and s1 <= T else 0
        heat = 1.0 if temperature is None else float(temperature[r])
        nodes, answer = ([0], []) if n else ([], [])
        while n:
            a = nodes[-1]
            row = logits[s0 + a]
            below = [i for i in range(a + 1, n) if parents[s0 + i] == a]
            P = probabilities(row, heat if heat > 0 else 1.0) if 0 <= heat < math.inf else None
            q = probabilities(draft[s0 + a], heat) if draft is not None and heat > 0 and below and P is not None else None
            if P is None or (q is None and draft is not None and heat > 0 and below):
                answer.append(-1)
                break
            taken = None
            if heat == 0:
                best = int(torch.nonzero(row == row.max())[0])
                taken = next((i for i in below if ids[s0 + i] == best), None)
            for i in below if heat > 0 else []:
                x, u = ids[s0 + i], uniforms[s0 + i]
                inside = 0 <= x < V
                if draft is None:
                    if inside and u < float(P[x]):
                        taken = i
                        break
                    rest = P.clone()
                    if inside:
                        rest[x] = 0
                else:
                    if inside and u * float(q[x]) < float(P[x]):
                        taken = i
                        break
                    rest = (P - q).clamp_min(0)
                if float(rest.sum()) > 2.0 ** -36:
                    P = rest / rest.sum()
            if taken is not None:
                nodes.append(taken)
                answer.append(ids[s0 + taken])
                continue
            if heat == 0:
                answer.append(best)
            else:
                sums = torch.cumsum(P, 0)
                v = int(torch.searchsorted(sums, uniforms[s0] * sums[-1:], right=True)[0])
                answer.append(min(v, int(torch.nonzero(P > 0)[-1])))
            break
        out.append((nodes, answer))
    pad = lambda x: x + [-1] * (max_new - len(x))
    return [len(n) for n, _ in out], [pad(n) for n, _ in out], [pad(a) for _, a in out]


def keep(cache, table, lens, starts, nodes, kept):
    """The cache's four tensors and the lengths after it."""
    arrays = [cache.k_codes.clone(), cache.k_scales.clone(), cache.v_codes.clone(), cache.v_scales.clone()]
    old = [x.clone() for x in arrays]
    page, cols, out = cache.page_size, nodes.shape[1], []

    def slot(r, token):
        if token < 0 or token // page >= table.shape[1]:
            return None
        p = int(table[r, token // page])
        return (p, token % page) if 0 <= p < cache.pages else None

    for r in range(table.shape[0]):
        count = int(starts[r + 1]) - int(starts[r])
        base = int(lens[r]) - count
        n = max(0, min(int(kept[r]), count, cols))
        for k in range(n):
            node = int(nodes[r, k])
            to, at = slot(r, base + k), slot(r, base + node)
            if 0 <= node < count and to and at:
                for x, o in zip(arrays, old):
                    x[to[0], :, to[1]] = o[at[0], :, at[1]]
        out.append(max(0, base + n))
    return arrays, out
