"""e2_cache_attend against 64 bits: head layouts, lengths, windows, pages, empty
rows, and what is out of range."""
import math

import pytest
import torch

import ops_reference as R

pytestmark = pytest.mark.gpu
HALF, BF = torch.float16, torch.bfloat16


def setup(lens, news, Hkv, G, D, page, dtype=BF, seed=0, extra_cols=0, spread=False):
    from paper_2606_03770_gb300 import ops
    g = torch.Generator(device="cuda").manual_seed(seed)
    B, cols = len(lens), max(1, -(-max(lens + [1]) // page)) + extra_cols
    pages = B * cols + 2
    cache = ops.Cache.empty(pages, page, Hkv, D)
    for c in (cache.k_codes, cache.v_codes):
        c.copy_(torch.randint(0, 256, c.shape, generator=g, device="cuda"))
    for s in (cache.k_scales, cache.v_scales):
        d = 0.1 + 0.2 * torch.rand(s.shape[:-1], generator=g, device="cuda")
        if spread:                                   # values of very different sizes, some constant groups
            d = d * 10.0 ** torch.randint(-3, 3, s.shape[:-1], generator=g, device="cuda")
            d[torch.rand(d.shape, generator=g, device="cuda") < 0.1] = 0
        m = -7.5 * d + 0.3 * torch.randn(d.shape, generator=g, device="cuda")
        s.copy_(torch.stack([d, m], -1))
    if spread:
        cache.k_scales.mul_(0.05)
    table = torch.randperm(pages, generator=g, device="cuda")[:B * cols].reshape(B, cols).int()
    T = sum(news)
    q = torch.randn(T, Hkv * G, D, generator=g, device="cuda").to(dtype)
    starts = torch.tensor([0] + list(torch.tensor(news).cumsum(0)), dtype=torch.int32, device="cuda")
    return cache, q, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), starts


def check(lens, news, Hkv, G, D, page, dtype=BF, window=0, scale=None, **kw):
    from paper_2606_03770_gb300 import ops
    s = setup(lens, news, Hkv, G, D, page, dtype, **kw)
    out = ops.cache_attend(*s, max_new=max(news), max_len=max(lens), window=window, scale=scale)
    want, lim, _ = R.attend(*s, 1 / math.sqrt(D) if scale is None else scale, window)
    R.close(out, want, lim, "out")
    return s, out


@pytest.mark.parametrize("Hkv,G", [(1, 1), (2, 3), (1, 5), (3, 7), (8, 8), (1, 16), (2, 20), (1, 40), (32, 1)])
@pytest.mark.parametrize("D", [64, 128])
def test_heads(Hkv, G, D):
    check([37, 200], [1, 1], Hkv, G, D, 16)


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 255, 257, 1000])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_lengths_one_token(length, page):
    check([length], [1], 1, 8, 128, page)
    check([length], [1], 2, 3, 64, page, HALF)


@pytest.mark.parametrize("new", [2, 3, 4, 8, 9, 17, 40, 64, 100])
def test_several_queries(new):
    check([new], [new], 1, 4, 64, 32)                   # a prompt from its start
    check([new + 77], [new], 2, 8 if new < 20 else 2, 128, 16, HALF)


@pytest.mark.parametrize("window", [1, 5, 16, 128, 1000])
@pytest.mark.parametrize("dtype", [HALF, BF])
def test_windows(window, dtype):
    check([300, 40, 129], [1, 1, 1], 2, 4, 128, 32, dtype, window)
    check([300, 40, 129], [5, 40, 1], 1, 8, 64, 16, dtype, window)


def test_ragged_batches_with_empty_requests():
    check([0, 1, 500, 33, 0, 64], [0, 1, 3, 2, 0, 1], 3, 7, 64, 16, HALF, 128)
    check([0, 1, 500, 33, 0, 64, 7], [0, 1, 20, 33, 0, 1, 7], 2, 5, 128, 64)
    check([70, 3000, 1], [64, 1, 1], 1, 8, 128, 64)


def test_queries_before_the_first_key_are_zero():
    """More queries than cached tokens: the first of them see nothing."""
    s, out = check([3], [5], 2, 4, 128, 16)
    assert bool((out[:2] == 0).all()) and bool((out[2:] != 0).any())
    s, out = check([0], [2], 1, 2, 64, 16)
    assert bool((out == 0).all())
    s, out = check([4, 80], [20, 70], 1, 8, 64, 16)
    assert bool((out[:16] == 0).all())


@pytest.mark.parametrize("B,length", [(1, 20000), (3, 4097), (16, 700)])
def test_long_contexts_are_split(B, length):
    check([length - 3 * b for b in range(B)], [1] * B, 1, 8, 128, 64)
    check([length - 3 * b for b in range(B)], [1] * B, 2, 1, 64, 16)


@pytest.mark.parametrize("new", [1, 30])
def test_scores_of_all_sizes(new):
    check([200], [new], 2, 4, 128, 16, scale=0.0)
    check([200], [new], 2, 4, 128, 16, scale=-0.05)
    check([200], [new], 2, 4, 64, 16, scale=2.0)          # one key takes nearly all the weight


@pytest.mark.parametrize("new", [1, 4, 33])
def test_values_of_all_sizes(new):
    check([150, 400], [new, 1], 2, 4, 128, 16, spread=True)
    check([150, 400], [new, 1], 1, 3, 64, 16, HALF, spread=True)


@pytest.mark.parametrize("new", [1, 2, 40])
def test_queries_of_all_sizes(new):
    """bf16 queries beyond fp16's range, and far below it."""
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([90], [new], 1, 4, 128, 16)
    q[:, 0] *= 1e6
    q[:, 1] *= 1e-9
    q[:, 2] = 0
    for scale in (1e-6, 1e-3):
        out = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=90, scale=scale)
        R.close(out, *R.attend(cache, q, table, lens, starts, scale, 0)[:2])


@pytest.mark.parametrize("new", [1, 50])
def test_pages_outside_the_cache_are_not_seen(new):
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([200, 200], [new, 1], 2, 4, 128, 16)
    table[0, 2], table[0, 5], table[1, 0] = -1, cache.pages, 2 ** 31 - 1
    out = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=200)
    R.close(out, *R.attend(cache, q, table, lens, starts, 128 ** -0.5, 0)[:2])
    table[0] = -1
    out = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=200)
    assert bool((out[:new] == 0).all())


@pytest.mark.parametrize("new", [1, 24])
def test_hidden_keys_do_not_matter(new):
    """NaN and huge values in keys that the mask hides, and past the end."""
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([100], [new], 1, 8, 128, 16)
    a = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=100, window=20)
    for s in (cache.k_scales, cache.v_scales):
        page, at = table[0, 100 // 16].item(), 100 % 16
        s[page, :, at:] = math.nan
        for j in range(0, 100 - new - 20):                   # before every window
            s[table[0, j // 16].item(), :, j % 16] = math.nan if j % 2 else math.inf
    b = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=100, window=20)
    assert torch.equal(a, b)


@pytest.mark.parametrize("new", [1, 24])
def test_nan_in_a_seen_key_reaches_its_heads_only(new):
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([100], [new], 2, 4, 64, 16)
    a = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=100)
    cache.k_scales[table[0, 1], 0, 3] = math.nan
    b = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=100)
    assert bool(torch.isnan(b[:, :4]).all()) and torch.equal(a[:, 4:], b[:, 4:])


def test_hints_larger_lengths_and_tokens_outside_requests():
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([300, 120], [3, 40], 2, 4, 128, 16, extra_cols=2)
    want, lim, _ = R.attend(cache, q, table, lens, starts, 128 ** -0.5, 0)
    for new, length in ((40, 300), (1, 1), (43, 5000), (0, 0), (2, 40)):
        out = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=length)
        R.close(out, want, lim, (new, length))
    R.close(ops.cache_attend(cache, q, table, lens, starts), want, lim)        # read from the device
    part = torch.tensor([1, 3, 20], dtype=torch.int32, device="cuda")          # tokens 0 and 20.. belong to none
    want, lim, written = R.attend(cache, q, table, lens, part, 128 ** -0.5, 0)
    out = torch.full_like(q, 9.0)
    ops.cache_attend(cache, q, table, lens, part, max_new=17, max_len=300, out=out)
    R.close(out[written], want[written], lim[written])
    assert bool((out[~written] == 9).all())
    bad = torch.tensor([-5, 2, 4000], dtype=torch.int32, device="cuda")        # starts out of range
    want, lim, written = R.attend(cache, q, table, lens, bad, 128 ** -0.5, 0)
    out = ops.cache_attend(cache, q, table, lens, bad, max_new=40, max_len=300)
    R.close(out[written], want[written], lim[written])


def test_table_narrower_than_its_rows_and_strided_queries():
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([60, 50], [1, 2], 2, 4, 64, 16, extra_cols=3)
    wide = torch.zeros(3, 8 * 64 + 16, device="cuda", dtype=BF)
    qs = wide[:, 8:-8].unflatten(1, (8, 64))
    qs.copy_(q)
    want, lim, _ = R.attend(cache, q, table[:, :2], lens, starts, 0.125, 0)    # keys from 32 on are not there
    out = wide.clone()
    o = out[:, 8:-8].unflatten(1, (8, 64))
    ops.cache_attend(cache, qs, table[:, :2], lens, starts, max_new=2, max_len=60, out=o)
    R.close(o, want, lim)
    assert torch.equal(out[:, :8], wide[:, :8]) and torch.equal(out[:, -8:], wide[:, -8:])


@pytest.mark.parametrize("news", [[1, 1], [30, 1]])
def test_same_bits_again_on_another_stream_and_in_a_graph(news):
    from paper_2606_03770_gb300 import ops
    s = setup([5000, 3000], news, 2, 8, 128, 64)
    kw = dict(max_new=max(news), max_len=5000)
    a = ops.cache_attend(*s, **kw)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(a)
    with torch.cuda.stream(st):
        rest = [ops.cache_attend(*s, **kw) for _ in range(4)]
        graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ops.cache_attend(*s, out=out, **kw)
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for b in rest) and torch.equal(a, out)


def test_cache_beyond_31_bits_of_bytes():
    from paper_2606_03770_gb300 import ops
    pages, page, H, D = 70000, 256, 2, 128            # 2.3 GB of codes each
    codes = [torch.empty(pages, H, page, D // 2, dtype=torch.uint8, device="cuda") for _ in range(2)]
    scales = [torch.empty(pages, H, page, 2, 2, dtype=HALF, device="cuda") for _ in range(2)]
    cache = ops.Cache(codes[0], scales[0], codes[1], scales[1])
    g = torch.Generator(device="cuda").manual_seed(5)
    table = torch.tensor([[pages - 1, pages - 2, 0, pages // 2]], dtype=torch.int32, device="cuda")
    for c, s in zip(codes, scales):
        for p in table[0].tolist():
            c[p] = torch.randint(0, 256, c[p].shape, generator=g, device="cuda")
            s[p] = 0.1 * torch.randn(s[p].shape, generator=g, device="cuda")
    for new in (1, 40):
        q = torch.randn(new, 8, D, generator=g, device="cuda").to(BF)
        lens = torch.tensor([1000], dtype=torch.int32, device="cuda")
        starts = torch.tensor([0, new], dtype=torch.int32, device="cuda")
        out = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=1000)
        R.close(out, *R.attend(cache, q, table, lens, starts, D ** -0.5, 0)[:2])


def test_empty_and_refusals():
    from paper_2606_03770_gb300 import e2ga, ops
    cache, q, table, lens, starts = setup([20, 20], [1, 2], 2, 2, 64, 16)
    kw = dict(max_new=2, max_len=20)
    assert ops.cache_attend(cache, q[:0], table[:0], lens[:0], starts[:1]).shape == (0, 4, 64)
    for bad in ((q.float(), table, lens, starts), (q[..., :32], table, lens, starts), (q, table.long(), lens, starts),
                (q, table, lens[:1], starts), (q, table, lens, starts[:2]), (q.cpu(), table, lens, starts)):
        with pytest.raises(ValueError):
            ops.cache_attend(cache, *bad, **kw)
    with pytest.raises(e2ga.E2Error, match="multiple of kv_heads"):
        ops.cache_attend(cache, q[:, :3].contiguous(), table, lens, starts, **kw)
    with pytest.raises(e2ga.E2Error, match="finite"):
        ops.cache_attend(cache, q, table, lens, starts, scale=math.inf, **kw)
    with pytest.raises(e2ga.E2Error, match="window"):
        ops.cache_attend(cache, q, table, lens, starts, window=-1, **kw)
    with pytest.raises(e2ga.E2Error, match="table_cols"):
        ops.cache_attend(cache, q, table[:, :0], lens, starts, **kw)
    with pytest.raises(e2ga.E2Error, match="16-byte"):
        ops.cache_attend(cache, torch.zeros(3, 260, device="cuda", dtype=BF)[:, 1:257].unflatten(1, (4, 64)), table, lens,
                         starts, **kw)


@pytest.mark.parametrize("dtype", [HALF, BF])
def test_prompts_longer_than_the_launch_was_told(dtype):
    from paper_2606_03770_gb300 import ops
    s = setup([400, 90, 700], [130, 1, 300], 2, 8, 128, 64, dtype)
    want, lim, _ = R.attend(*s, 128 ** -0.5, 0)
    for new in (10, 33, 100):                        # several blocks of rows in turn
        R.close(ops.cache_attend(*s, max_new=new, max_len=700), want, lim, new)


@pytest.mark.parametrize("B,length,window", [(2, 2000, 0), (1, 900, 0), (6, 1100, 400), (9, 300, 0), (24, 257, 0)])
@pytest.mark.parametrize("new", [1, 2])
def test_parts_joined_in_a_cluster(B, length, window, new):
    lens = [length - 37 * b % length for b in range(B)]
    check(lens, [min(new, n) for n in lens], 4, 8, 128, 16, window=window)
    check(lens, [min(new, n) for n in lens], 3, 5, 64, 64, dtype=HALF, window=window)


@pytest.mark.parametrize("length", [700, 5000])
def test_nan_in_one_part_reaches_its_heads_only(length):
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([length, 40], [1, 1], 2, 4, 128, 64)
    a = ops.cache_attend(cache, q, table, lens, starts, max_new=1, max_len=length)
    cache.v_scales[int(table[0, length // 128]), 0, 5, :, 1] = math.nan     # a key near the middle, first KV head
    b = ops.cache_attend(cache, q, table, lens, starts, max_new=1, max_len=length)
    assert bool(torch.isnan(b[0, :4]).all())
    assert torch.equal(a[0, 4:], b[0, 4:]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("length", [331, 333, 340, 700])
@pytest.mark.parametrize("scale,size", [(0.0, 1.0), (1e-38, 1e-9)])
def test_scores_of_zero_with_windows(length, scale, size):
    """Scores that are 0, or too small for 32 bits: every key seen counts alike, also in rows to which
    a warp's first tile is hidden (a launch told of short contexts: several tiles a warp)."""
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([length], [16], 2, 1, 64, 16)
    q *= size
    for window in (270, 300, 316):
        out = ops.cache_attend(cache, q, table, lens, starts, max_new=16, max_len=1, scale=scale, window=window)
        R.close(out, *R.attend(cache, q, table, lens, starts, scale, window)[:2], window)


@pytest.mark.parametrize("new,G", [(1, 8), (2, 4), (16, 1), (40, 2)])
def test_scores_of_zero_with_pages_that_are_not_there(new, G):
    from paper_2606_03770_gb300 import ops
    for missing in (1, 4):
        cache, q, table, lens, starts = setup([700], [new], 2, G, 128, 32)
        table[0, :missing] = -1
        out = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=1, scale=0.0)
        R.close(out, *R.attend(cache, q, table, lens, starts, 0.0, 0)[:2], missing)


LOW, HIGH = -2 ** 31, 2 ** 31 - 1


@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("new", [3, 40, 100])
@pytest.mark.parametrize("length", [LOW, LOW + 1, -1, HIGH - 64, HIGH])
def test_lengths_at_the_ends_of_their_type(length, new, dtype):
    """Below 0 nothing is seen; beyond the table all that it has."""
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([150, 90], [new, 2], 2, 4, 64, 16, dtype, extra_cols=1)
    lens[0] = length
    for window in (0, 70):
        out = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=150, window=window)
        R.close(out, *R.attend(cache, q, table, lens, starts, 0.125, window)[:2], window)
        assert length > 0 or bool((out[:new] == 0).all())


@pytest.mark.parametrize("tokens", [2, 50, 200])
@pytest.mark.parametrize("starts", [(LOW, HIGH), (0, HIGH), (LOW, 30), (LOW, -5), (HIGH - 3, HIGH), (20, LOW), (HIGH, LOW), (-7, 13)])
def test_starts_at_the_ends_of_their_type(starts, tokens):
    """Queries outside q are none; those inside keep their positions."""
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, _ = setup([150], [tokens], 2, 4, 128, 16)
    starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
    for length in (150, HIGH, LOW):
        lens[0] = length
        want, lim, written = R.attend(cache, q, table, lens, starts, 128 ** -0.5, 0)
        for new in (1, 30, 120):
            out = torch.full_like(q, 9.0)
            ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=150, out=out)
            R.close(out[written], want[written], lim[written], (length, new))
            assert bool((out[~written] == 9).all())


def test_gradients_are_refused():
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([20], [3], 2, 2, 64, 16)
    kw = dict(max_new=3, max_len=20)
    out = ops.cache_attend(cache, q, table, lens, starts, **kw)
    grad = q.clone().requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        ops.cache_attend(cache, grad, table, lens, starts, **kw)
    with pytest.raises(ValueError, match="gradient"):
        ops.cache_attend(cache, q, table, lens, starts, out=grad, **kw)
    with torch.no_grad():
        assert torch.equal(out, ops.cache_attend(cache, grad, table, lens, starts, **kw))


@pytest.mark.parametrize("new", [1, 40])
def test_windows_and_hints_beyond_32_bits(new):
    """They are as large as any context, not what is left of them in 32 bits."""
    from paper_2606_03770_gb300 import e2ga, ops
    s = setup([300, 90], [new, 1], 2, 4, 64, 16)
    want = ops.cache_attend(*s, max_new=new, max_len=300)
    for big in (2 ** 31 - 1, 2 ** 31, 2 ** 32 + 5, 2 ** 40):
        assert torch.equal(want, ops.cache_attend(*s, max_new=new, max_len=300, window=big)), big
        R.close(ops.cache_attend(*s, max_new=big, max_len=big), *R.attend(*s, 0.125, 0)[:2], big)
    for small in (-1, -2 ** 31 - 1, -2 ** 32 + 7):
        with pytest.raises(e2ga.E2Error, match="window"):
            ops.cache_attend(*s, max_new=new, max_len=300, window=small)


@pytest.mark.parametrize("starts", [(1, 0), (LOW, HIGH), (7, 7)])
@pytest.mark.parametrize("length", [-20, 20])
def test_hints_are_read_from_any_lengths(starts, length):
    """Counts below 0 are none, those beyond 32 bits are not taken for such."""
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, _ = setup([20], [3], 2, 4, 64, 16)
    lens[0] = length
    starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 9.0)
    ops.cache_attend(cache, q, table, lens, starts, out=out)
    want, lim, written = R.attend(cache, q, table, lens, starts, 0.125, 0)
    R.close(out[written], want[written], lim[written])
    assert bool((out[~written] == 9).all())


def test_workspaces_that_are_given():
    from paper_2606_03770_gb300 import e2ga, ops
    s = setup([20000], [1], 1, 8, 128, 64)
    kw = dict(max_new=1, max_len=20000)
    want = ops.cache_attend(*s, **kw)
    one = torch.zeros(1, device="cuda")
    with pytest.raises(ValueError, match="contiguous"):
        ops.cache_attend(*s, workspace=one.expand(1 << 26), **kw)
    with pytest.raises(e2ga.E2Error, match="workspace"):
        ops.cache_attend(*s, workspace=one, **kw)
    assert torch.equal(want, ops.cache_attend(*s, workspace=torch.zeros(1 << 20, device="cuda"), **kw))


@pytest.mark.parametrize("d", [9000.0, -9000.0])
@pytest.mark.parametrize("new", [1, 40])
def test_values_beyond_fp16_in_a_cache(new, d):
    """A cache with larger scales than appended tokens have: as they are for a few rows, no larger
    than 65,504 from 65 rows of a request and KV head on."""
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([90], [new], 1, 4, 64, 16)
    cache.v_scales[..., 0], cache.v_scales[..., 1] = d, 500.0
    out = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=90)
    at = torch.arange(90, device="cuda")
    page = table[0].long()[at // 16]
    k, v = (R.cache_values(c[page, 0, at % 16], s[page, 0, at % 16]) for c, s in
            ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)))
    if 4 * new >= 65:
        v = v.clamp(-65504.0, 65504.0)
    seen = at[None] <= torch.arange(90 - new, 90, device="cuda")[:, None]
    a = (q.double() @ k.T / 8).masked_fill(~seen[:, None], -math.inf)
    p = torch.softmax(a, -1)
    _, lim, _ = R.attend(cache, q, table, lens, starts, 0.125, 0)      # (of the values as they are: larger ones)
    R.close(out, p @ v, lim)


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("new", [1, 2, 40])
def test_queries_that_are_not_finite_are_nan_where_they_see_keys(new, dtype, value):
    """Scores that are all -inf (keys of one sign) have no softmax, either."""
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([200, new - 1], [new, new], 2, 4, 64, 16, dtype)
    cache.k_scales[..., 1] = 0.5
    cache.k_codes.bitwise_or_(0x11)
    y0 = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=200)
    q[0, 1, 7] = value
    q[-1, 5, 0], q[-1, 6, 63] = value, -value
    if new > 1:
        q[new, 3] = value                              # a query that sees no key
    for window in (0, 30):
        out = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=200, window=window)
        R.close(out, *R.attend(cache, q, table, lens, starts, 0.125, window)[:2])
    assert bool(torch.isnan(out[0, 1]).all()) and bool((out[new, 3] == 0).all())
    y = ops.cache_attend(cache, q, table, lens, starts, max_new=new, max_len=200)
    assert torch.equal(y[0, 2:], y0[0, 2:]) and torch.equal(y[-1, :5], y0[-1, :5])


@pytest.mark.parametrize("new,window", [(1, 0), (1, 700), (3, 0), (40, 0), (40, 700)])
@pytest.mark.parametrize("B,length,D,page", [(1, 1000, 64, 16), (8, 2305, 128, 64), (1, 4097, 128, 64), (3, 9001, 64, 256),
                                             (1, 20000, 128, 64)])
@pytest.mark.parametrize("dtype", [HALF, BF])
def test_every_key_counts(B, length, D, page, new, window, dtype):
    """Each key has one element of its own that is not 0, so one that is lost, or seen twice, shows.

    Queries of ones and constant keys: a score is its key's level, exact in any form, levels by 64
    keys.  Weights and their products with values may be rounded to fp16 (2^-11 each), outputs to
    2^-8 or 2^-11; the rest is in 32 bits."""
    from paper_2606_03770_gb300 import ops
    H = 8
    cache, q, table, lens, starts = setup([length - 5 * b for b in range(B)], [new] * B, H, 2, D, page, dtype)
    q.fill_(1)
    g = torch.Generator(device="cuda").manual_seed(length)
    level = torch.randint(-4, 5, (length,), generator=g, device="cuda")[torch.arange(length, device="cuda") // 64] * 0.5
    key = torch.arange(length, device="cuda")
    for s in (cache.k_scales, cache.v_scales):
        s.zero_()
    cache.v_scales[..., 0] = 1
    for b in range(B):
        cache.k_scales[table[b].long()[key // page], :, key % page, :, 1] = level.half()[:, None, None]
    scale = 0.5 / D
    kw = dict(max_new=new, max_len=length, window=window, scale=scale)
    pos = torch.arange(-new, 0, device="cuda")[:, None]
    h, d = torch.meshgrid(torch.arange(H, device="cuda"), torch.arange(D, device="cuda"), indexing="ij")
    tol = 2.0 ** -9 + R.EPS[dtype] + (length + 64) * R.EPS32 / 16
    for first in range(0, length, H * D):
        own = (first + h * D + d) % length                                     # the key of element (h, d)
        cache.v_codes.zero_()
        for b in range(B):
            cache.v_codes[table[b].long()[own // page], h, own % page, d // 2] |= (15 << 4 * (d % 2)).byte()
        out = ops.cache_attend(cache, q, table, lens, starts, **kw).view(B, new, H, 2, D)
        for b in range(B):
            at = int(lens[b]) + pos
            seen = (key <= at) & ((key > at - window) if window else (key >= 0))
            p = torch.softmax((level.double() * 0.5).masked_fill(~seen, -math.inf), -1)
            want = (15 * p)[:, own][:, :, None]                                # [new][H][1][D]
            got = out[b].double()
            bad = (got - want).abs() > tol * want + R.TINY16
            assert not bool(bad.any()), (b, first, int(bad.sum()))


@pytest.mark.parametrize("lens,news", [([5000, 3000], [1, 1]), ([40000], [1]), ([700, 300], [40, 3])])
def test_two_streams_at_once(lens, news):
    """Each call with a workspace of its own, many of both in flight."""
    from paper_2606_03770_gb300 import ops
    kw = dict(max_new=max(news), max_len=max(lens))
    sets = [setup(lens, news, 2, 8, 128, 64, seed=seed) for seed in (1, 2)]
    want = [ops.cache_attend(*s, **kw) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(ops.cache_attend(*sets[i], **kw))
    torch.cuda.synchronize()
    for a, outs in zip(want, got):
        assert all(torch.equal(a, o) for o in outs)
