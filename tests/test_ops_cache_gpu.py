"""e2_cache_append and e2_cache_read: every bit against the header's roundings,
the values against 64 bits."""
import math

import pytest
import torch

import ops_reference as R

pytestmark = pytest.mark.gpu
HALF, BF = torch.float16, torch.bfloat16


def table(n, rot):
    ang = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * \
        10000.0 ** (-torch.arange(rot // 2, device="cuda", dtype=torch.float64) * 2 / max(rot, 1))
    return ang.cos().float(), ang.sin().float()


def randn(seed, *shape, dtype=BF):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def expect(cache, k, v, slots, positions, cos, sin, interleaved):
    """The cache's four tensors as they have to be afterwards."""
    want = [t.clone() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    n = cache.pages * cache.page_size
    ok = (slots >= 0) & (slots < n) & (positions >= 0) & (positions < cos.shape[0])
    at = positions[ok].long()
    p, o = slots[ok] // cache.page_size, slots[ok] % cache.page_size
    for i, x in ((0, R.rotate(k[ok], cos[at], sin[at], interleaved)), (2, v[ok].float())):
        codes, scales = R.cache_pack(x)
        want[i][p, :, o], want[i + 1][p, :, o] = codes, scales
    return want


def same(a, b):
    """Equal bit for bit, any NaN equal to any other."""
    if a.is_floating_point():
        assert torch.equal(torch.isnan(a), torch.isnan(b))
        a, b = torch.nan_to_num(a), torch.nan_to_num(b)
    assert torch.equal(a, b)


def check(cache, k, v, slots, positions, cos, sin, q=None, interleaved=False):
    from paper_2606_03770_gb300 import ops
    want = expect(cache, k, v, slots, positions, cos, sin, interleaved)
    qo = ops.cache_append(cache, k, v, slots, positions, cos, sin, q=q, interleaved=interleaved)
    for got, w in zip((cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), want):
        same(got, w)
    if q is not None:
        at = positions.long().clamp(0, cos.shape[0] - 1)
        r = R.rotate(q, cos[at], sin[at], interleaved).to(q.dtype)
        r[(positions < 0) | (positions >= cos.shape[0])] = math.nan
        same(qo.float(), r.float()) if q.dtype == BF else same(qo, r)
    return qo


@pytest.mark.parametrize("D,rot", [(64, 64), (64, 32), (64, 0), (128, 128), (128, 64), (128, 16), (128, 96)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [HALF, BF])
def test_append_bits(D, rot, interleaved, dtype):
    from paper_2606_03770_gb300 import ops
    for tokens, heads, hq, page in ((1, 1, 1, 16), (5, 3, 21, 32), (33, 8, 64, 256)):
        cache = ops.Cache.empty(4, page, heads, D)
        cos, sin = table(300, rot)
        slots = torch.randperm(4 * page, device="cuda")[:tokens]
        pos = torch.randint(0, 300, (tokens,), device="cuda", dtype=torch.int32)
        check(cache, randn(1, tokens, heads, D, dtype=dtype), randn(2, tokens, heads, D, dtype=dtype), slots, pos,
              cos, sin, randn(3, tokens, hq, D, dtype=dtype), interleaved)


def test_values_against_64_bits():
    from paper_2606_03770_gb300 import ops
    T, H, D = 50, 2, 128
    k, v = randn(4, T, H, D) + 5, randn(5, T, H, D) * 100
    cache = ops.Cache.empty(4, 16, H, D)
    slots = torch.arange(T, device="cuda")
    cos, sin = table(T, D)
    ops.cache_append(cache, k, v, slots, slots.int(), cos, sin)
    for dtype in (HALF, BF, torch.float32):
        rk, rv = ops.cache_read(cache, slots, dtype)
        c, s = cos.double()[:, None], sin.double()[:, None]
        a, b = k.double().split(64, 2)
        for got, x in ((rk, torch.cat([a * c - b * s, b * c + a * s], 2)), (rv, v.double())):
            g = x.unflatten(2, (-1, 64))
            lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
            step = (hi - lo) / 15
            # half a step; scale and minimum rounded to fp16; the turn in 32 bits; the read value rounded
            lim = step / 2 * 1.001 + 2.0 ** -11 * (lo.abs() + 16 * step) + 1e-6 * x.abs().max() + \
                (R.EPS[dtype] * (g.abs() + step))
            assert bool(((got.double().unflatten(2, (-1, 64)) - g).abs() <= lim).all())


def test_read_is_the_codes_values():
    from paper_2606_03770_gb300 import ops
    g = torch.Generator(device="cuda").manual_seed(9)
    for D, page in ((64, 16), (128, 64)):
        cache = ops.Cache.empty(5, page, 3, D)
        for c in (cache.k_codes, cache.v_codes):
            c.copy_(torch.randint(0, 256, c.shape, generator=g, device="cuda"))
        for s in (cache.k_scales, cache.v_scales):
            s.copy_(torch.randn(s.shape, generator=g, device="cuda"))
        slots = torch.tensor([0, 5 * page - 1, 17, -1, 3, 5 * page, 2 ** 40, -2 ** 40], device="cuda")
        ok = (slots >= 0) & (slots < 5 * page)
        at = torch.where(ok, slots, 0)
        for dtype in (HALF, BF, torch.float32):
            for got, codes, scales in zip(ops.cache_read(cache, slots, dtype), (cache.k_codes, cache.v_codes),
                                          (cache.k_scales, cache.v_scales)):
                w = R.cache_values(codes[at // page, :, at % page], scales[at // page, :, at % page])
                w = torch.where(ok[:, None, None], w, 0.0)
                R.close(got, w, R.EPS[dtype] * w.abs() + 4 * R.EPS32 * (w.abs() + 16) + R.TINY16)


def test_padding_bad_slots_and_bad_positions():
    from paper_2606_03770_gb300 import ops
    cache = ops.Cache.empty(2, 16, 2, 64)
    slots = torch.tensor([-1, 32, 5, 2 ** 41, -2 ** 41, 7, 31], device="cuda")
    pos = torch.tensor([0, 1, 9, 3, 4, -5, 10], device="cuda", dtype=torch.int32)   # a table of 10 rows
    cos, sin = table(10, 64)
    qo = check(cache, randn(1, 7, 2, 64), randn(2, 7, 2, 64), slots, pos, cos, sin, randn(3, 7, 4, 64))
    assert int((cache.k_codes != 0).any(-1).sum()) == 2          # one token, two heads
    assert torch.isnan(qo).flatten(1).any(1).tolist() == [False] * 5 + [True] * 2


def test_values_that_fp16_does_not_hold():
    from paper_2606_03770_gb300 import ops
    cache = ops.Cache.empty(1, 16, 1, 128)
    v = randn(7, 8, 1, 128)
    v[0, 0, 3] = math.nan
    v[1, 0, 70] = math.inf
    v[2, 0, 70], v[2, 0, 71] = -math.inf, math.inf
    v[3] = 1e30
    v[4] = -3.0                      # all equal: scale 0
    v[5] = 0
    v[6] *= 1e-7                     # below fp16's normal range
    v[7, 0, :64] = 65504
    k = v.clone()
    slots = torch.arange(8, device="cuda")
    cos, sin = table(8, 0)
    check(cache, k, v, slots, slots.int(), cos, sin)
    _, r = ops.cache_read(cache, slots, torch.float32)
    assert bool(torch.isnan(r[0, 0, :64]).all()) and bool(torch.isfinite(r[0, 0, 64:]).all())
    assert bool(torch.isfinite(r[1:]).all())
    assert bool((r[3] == 65504).all()) and bool((r[4] == -3).all()) and bool((r[5] == 0).all())


def test_strided_projection_rows_and_in_place_queries():
    """Queries, keys and values side by side in one projection's rows."""
    from paper_2606_03770_gb300 import ops
    T, H, Hq, D = 9, 2, 6, 64
    rows = randn(11, T, (Hq + 2 * H) * D + 8)
    q = rows[:, :Hq * D].unflatten(1, (Hq, D))
    k = rows[:, Hq * D:(Hq + H) * D].unflatten(1, (H, D))
    v = rows[:, (Hq + H) * D:(Hq + 2 * H) * D].unflatten(1, (H, D))
    kept = rows.clone()
    cache = ops.Cache.empty(1, 16, H, D)
    cos, sin = table(64, D)
    slots = torch.arange(T, device="cuda") + 3
    want = expect(cache, k, v, slots, slots.int(), cos, sin, False)
    qw = R.rotate(q, cos[slots], sin[slots], False).to(BF)
    ops.cache_append(cache, k, v, slots, slots.int(), cos, sin, q=q, q_out=q)
    for got, w in zip((cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), want):
        same(got, w)
    assert torch.equal(q, qw) and torch.equal(rows[:, Hq * D:], kept[:, Hq * D:])


def test_slots_beyond_31_bits_of_bytes():
    """A cache whose arrays pass 2^31 bytes: its last tokens."""
    from paper_2606_03770_gb300 import ops
    pages, page, H, D = 70000, 256, 2, 128            # 2.3 GB of codes each
    codes = [torch.empty(pages, H, page, D // 2, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.empty(pages, H, page, 2, 2, dtype=HALF, device="cuda") for _ in range(2)]
    cache = ops.Cache(codes[0], scales[0], codes[1], scales[1])
    n = pages * page
    slots = torch.tensor([n - 1, n - 300, 0, n // 2], device="cuda")
    cos, sin = table(4, D)
    k, v = randn(1, 4, H, D), randn(2, 4, H, D)
    ops.cache_append(cache, k, v, slots, torch.zeros(4, device="cuda", dtype=torch.int32), cos, sin)
    for x, c, s in ((k, codes[0], scales[0]), (v, codes[1], scales[1])):
        wc, ws = R.cache_pack(x.float())
        same(c[slots // page, :, slots % page], wc)
        same(s[slots // page, :, slots % page], ws)


def test_refusals():
    from paper_2606_03770_gb300 import e2ga, ops
    cache = ops.Cache.empty(1, 16, 2, 64)
    k = randn(1, 3, 2, 64)
    slots, pos = torch.arange(3, device="cuda"), torch.zeros(3, device="cuda", dtype=torch.int32)
    cos, sin = table(4, 64)
    ok = (k, k, slots, pos, cos, sin)
    for i, bad in ((0, k.float()), (0, k[:, :1]), (1, k.half()), (2, slots.int()), (3, pos.long()), (3, pos[:2]),
                   (4, cos.double()), (5, sin[:, :8]), (0, k.cpu())):
        a = list(ok)
        a[i] = bad
        with pytest.raises(ValueError):
            ops.cache_append(cache, *a)
    with pytest.raises(e2ga.E2Error, match="multiple of 16"):
        ops.cache_append(cache, k, k, slots, pos, *table(4, 24))
    with pytest.raises(e2ga.E2Error, match="up to head_dim"):
        ops.cache_append(cache, k, k, slots, pos, *table(4, 128))
    with pytest.raises(e2ga.E2Error, match="16-byte"):
        ops.cache_append(cache, randn(1, 3, 130)[:, 1:129].unflatten(1, (2, 64)), k, slots, pos, cos, sin)
    with pytest.raises(ValueError, match="side by side"):
        ops.cache_append(cache, randn(1, 3, 4, 64)[:, ::2], k, slots, pos, cos, sin)
    with pytest.raises(ValueError, match="page_size"):
        ops.Cache.empty(1, 24, 2, 64)
    with pytest.raises(ValueError, match="head_dim"):
        ops.Cache.empty(1, 16, 2, 96)
    with pytest.raises(ValueError):
        ops.cache_read(cache, slots.int())
    k0 = k[:0]
    assert ops.cache_append(cache, k0, k0, slots[:0], pos[:0], cos, sin, q=k0).shape == (0, 2, 64)


@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("unit", [1.0, 0.75, 3.0, 2.0 ** -14, 5.0 * 2.0 ** 8])
def test_quotients_at_and_beside_halves(dtype, unit):
    """Groups whose quotients are whole numbers, halves and the numbers next to them."""
    from paper_2606_03770_gb300 import ops
    g = torch.Generator(device="cuda").manual_seed(3)
    k = torch.randint(0, 31, (96, 2, 128), generator=g, device="cuda") * 0.5
    k[:, :, 0::64], k[:, :, 1::64] = 0.0, 15.0
    v = (k * unit).to(dtype)
    k = k.to(dtype)
    step = torch.randint(-1, 2, v.shape, generator=g, device="cuda").to(torch.int16)
    step[(v == 0) | (step < 0) & (v == v.amax())] = 0
    v = (v.view(torch.int16) + step).view(dtype)
    cache = ops.Cache.empty(3, 32, 2, 128)
    slots, pos = torch.arange(96, device="cuda"), torch.zeros(96, device="cuda", dtype=torch.int32)
    check(cache, k, v, slots, pos, *table(4, 128))


def test_a_cache_keeps_the_memory_it_points_at():
    from paper_2606_03770_gb300 import ops
    cache = ops.Cache.empty(2, 16, 2, 64)
    for name in ("k_codes", "k_scales", "v_codes", "v_scales", "pages", "kv_heads", "page_size", "head_dim", "device",
                 "struct", "ref"):
        with pytest.raises(AttributeError, match="Cache"):
            setattr(cache, name, getattr(cache, name))
    with pytest.raises(AttributeError, match="Cache"):
        del cache.v_scales
    given = [t.clone() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    other = ops.Cache(*given)
    for t in given:
        t.data = torch.ones_like(t)
    slots = torch.arange(32, device="cuda")
    k, v = randn(1, 32, 2, 64), randn(2, 32, 2, 64)
    for c in (cache, other):
        ops.cache_append(c, k, v, slots, torch.zeros(32, device="cuda", dtype=torch.int32), *table(4, 64))
    for a, b in zip(ops.cache_read(cache, slots), ops.cache_read(other, slots)):
        assert torch.equal(a, b)
    assert all(bool((t == 1).all()) for t in given)


def test_gradients_are_refused():
    from paper_2606_03770_gb300 import ops
    cache = ops.Cache.empty(1, 16, 2, 64)
    k, (cos, sin) = randn(1, 3, 2, 64), table(4, 64)
    slots, pos = torch.arange(3, device="cuda"), torch.zeros(3, device="cuda", dtype=torch.int32)
    ok = dict(k=k, v=k, cos=cos, sin=sin, q=k, q_out=k.clone())
    for name in ok:
        with pytest.raises(ValueError, match=f"{name} requires a gradient"):
            ops.cache_append(cache, slots=slots, positions=pos, **dict(ok, **{name: ok[name].clone().requires_grad_()}))
    other = ops.Cache(cache.k_codes, cache.k_scales.clone().requires_grad_(), cache.v_codes, cache.v_scales)
    with pytest.raises(ValueError, match="gradient"):
        ops.cache_read(other, slots)
    with torch.no_grad():
        ops.cache_append(cache, slots=slots, positions=pos, **{n: t.clone().requires_grad_() for n, t in ok.items()})
    assert bool((cache.k_codes[0, :, :3] != 0).any())
