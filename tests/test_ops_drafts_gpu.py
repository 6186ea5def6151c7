"""The operators for drafted tokens against 64 bits: trees and their masks, decisions at their
borders, rows without a distribution, ways that move onto one another, and the run of them together."""
import math

import pytest
import torch

import drafts_reference as DR
import ops_reference as R
from test_ops_attend_gpu import setup

pytestmark = pytest.mark.gpu
HALF, BF, F32 = torch.float16, torch.bfloat16, torch.float32
I32 = dict(dtype=torch.int32, device="cuda")


def i32(x):
    return torch.tensor(x, **I32)


def random_tree(n, seed, chain=0.3):
    """Parents of n nodes: some chains, some bushes."""
    g = torch.Generator().manual_seed(seed)
    out = [-1]
    for i in range(1, n):
        far = torch.rand(1, generator=g).item() < chain
        out.append(i - 1 if far else int(torch.randint(0, i, (1,), generator=g)))
    return out


def trees(news, seed=0):
    return i32([p for r, n in enumerate(news) for p in (random_tree(n, seed + r) if n else [])])


# ---- attention --------------------------------------------------------------------------------------
def check_tree(lens, news, Hkv, G, D, page, dtype=BF, window=0, scale=None, parents=None, **kw):
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens_t, starts = setup(lens, news, Hkv, G, D, page, dtype, **kw)
    parents = trees(news) if parents is None else i32(parents)
    out = ops.cache_attend_tree(cache, q, parents, table, lens_t, starts, max_new=max(news), max_len=max(lens), window=window,
                                scale=scale)
    want, bound, _ = DR.attend_tree(cache, q, parents, table, lens_t, starts, D ** -0.5 if scale is None else scale, window)
    R.close(out, want, bound, f"{lens} {news} {Hkv}x{G} {D} {dtype} {window}")
    return cache, q, parents, table, lens_t, starts, out


@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 5, 8, 16])
@pytest.mark.parametrize("new", [1, 2, 7, 16, 64])
def test_heads_and_nodes(dtype, D, G, new):
    check_tree([new + 100, new, new + 1], [new, new, max(1, new - 1)], 2, G, D, 16, dtype, seed=new + G)


@pytest.mark.parametrize("new", [3, 9, 33])
@pytest.mark.parametrize("before", [0, 1, 13, 31, 32, 33, 63, 64, 65, 127, 129, 1000])
def test_trees_across_tiles_and_pages(new, before):
    """The tree's keys begin and end anywhere in a tile, and in a page."""
    for page, G in ((16, 8), (64, 3)):
        check_tree([before + new], [new], 1, G, 128, page, seed=before)


@pytest.mark.parametrize("window", [1, 2, 5, 40, 333, 5000])
@pytest.mark.parametrize("G", [1, 7, 16])
def test_windows(window, G):
    """A window ends within the tree, at its root, and before it."""
    check_tree([1500, 40, 64, 11], [20, 20, 64, 3], 3, G, 64, 16, HALF, window=window, seed=window)


def test_long_contexts():
    check_tree([9000, 4097], [7, 64], 2, 8, 128, 64, seed=3)
    check_tree([20000], [16], 1, 16, 128, 128, seed=4)
    check_tree([30011], [3], 1, 2, 64, 32, HALF, seed=5)


@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,G,new,ctx", [(8, 2, 16, 700), (8, 8, 16, 700), (4, 8, 16, 1100), (4, 3, 9, 1100), (3, 64, 3, 2000)])
def test_contexts_joined_in_clusters(dtype, D, B, G, new, ctx):
    """Parts of two and of four blocks, of a few rows and of many, some of them empty."""
    check_tree([ctx - 90 * r if r != 2 else new for r in range(B)], [new] * B, 8, G, D, 64, dtype, seed=B + G)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window", [0, 70])
def test_pages(page, D, window):
    """Copies of a tile in one piece, two and four."""
    check_tree([777, 64, 320], [20, 3, 64], 2, 4, D, page, window=window, seed=page)


def test_more_requests_than_multiprocessors():
    news = [1 + r % 5 for r in range(60)]
    check_tree([200 + 7 * r for r in range(60)], news, 4, 8, 64, 32, seed=15)
    check_tree([20 + r for r in range(60)], news, 4, 1, 128, 16, seed=16)


def test_tables_with_columns_to_spare():
    from paper_2606_03770_gb300 import ops
    for G in (1, 8):
        cache, q, table, lens, starts = setup([300, 90], [9, 4], 2, G, 128, 64, seed=17, extra_cols=3)
        parents = trees([9, 4])
        kw = dict(max_new=9, max_len=300)
        want = ops.cache_attend_tree(cache, q, parents, table.contiguous(), lens, starts, **kw)
        wide = torch.full((2, table.shape[1] + 5), 10 ** 6, **I32)
        wide[:, 2:2 + table.shape[1]] = table
        assert torch.equal(ops.cache_attend_tree(cache, q, parents, wide[:, 2:2 + table.shape[1]], lens, starts, **kw), want)
        # a table that ends within the context, and one that ends within the tree
        for cols in (1, 4):
            out = ops.cache_attend_tree(cache, q, parents, table[:, :cols], lens, starts, **kw)
            ref, bound, _ = DR.attend_tree(cache, q, parents, table[:, :cols], lens, starts, 128 ** -0.5, 0)
            R.close(out, ref, bound)


def test_ragged_batches_and_empty_requests():
    check_tree([0, 517, 1, 90, 64], [0, 12, 1, 64, 3], 3, 7, 64, 16, HALF, seed=6)
    check_tree([5, 700], [0, 1], 8, 1, 128, 64, seed=7)


def test_chains_are_what_cache_attend_computes():
    """Of a chain the tree's mask is the causal one: where the same kernel computes both, bit for bit."""
    from paper_2606_03770_gb300 import ops
    for G, new in ((1, 5), (4, 2)):                              # (up to eight rows)
        cache, q, table, lens, starts = setup([517, 90], [new, new], 4, G, 128, 64, HALF, seed=8)
        parents = i32([i - 1 for _ in range(2) for i in range(new)])
        kw = dict(max_new=new, max_len=517)
        for window in (0, 64):
            a = ops.cache_attend(cache, q, table, lens, starts, window=window, **kw)
            b = ops.cache_attend_tree(cache, q, parents, table, lens, starts, window=window, **kw)
            assert torch.equal(a, b)


@pytest.mark.parametrize("G", [1, 2, 16])
@pytest.mark.parametrize("new,before", [(5, 3), (16, 100), (64, 0), (64, 190), (37, 27)])
@pytest.mark.parametrize("window", [0, 1, 7, 60])
def test_each_node_sees_its_way_and_no_more(G, new, before, window):
    """Queries of 0 weigh all keys alike, and node a's value is 1 at element a: an output tells which nodes it is of."""
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([before + new], [new], 2, G, 64, 16, seed=14)
    q.zero_()
    cache.k_scales.zero_()
    cache.v_codes.zero_()
    cache.v_scales.zero_()
    cache.v_scales[..., 0] = 1.0 / 15
    for a in range(new):
        at = before + a
        cache.v_codes[int(table[0, at // 16]), :, at % 16, a // 2] = 15 << (4 * (a % 2))
    par = random_tree(new, new + before, 0.6)
    out = ops.cache_attend_tree(cache, q, i32(par), table, lens, starts, max_new=new, max_len=before + new, window=window).float()
    for i in range(new):
        up = DR.way(par, 0, i, new)
        nodes = [a for d, a in enumerate(up) if not window or d < window]
        context = before if not window else min(before, max(0, window - len(up)))
        want = torch.zeros(64, device="cuda")
        want[nodes] = 1.0 / (len(nodes) + context)
        # (1/15 in fp16 times 15, and the output's rounding)
        assert torch.allclose(out[i], want.expand_as(out[i]), rtol=2.0 ** -10 + 2.0 ** -8, atol=0), i


@pytest.mark.parametrize("G", [1, 4, 16])
def test_parents_out_of_range_count_as_none(G):
    new = 12
    given = [-1, 0, 1, 3, 9, 100, -7, 6, 2 ** 31 - 1, 8, -2 ** 31, 10]
    check_tree([200], [new], 2, G, 128, 16, parents=given, seed=9)


@pytest.mark.parametrize("G", [1, 16])
def test_more_nodes_than_a_tree_holds(G):
    """A request of 70 nodes where the launch was told of 64: the 65th on are NaN, the others as they are."""
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([200], [70], 2, G, 64, 16, seed=10)
    parents = i32(random_tree(70, 1))
    out = ops.cache_attend_tree(cache, q, parents, table, lens, starts, max_new=64, max_len=200)
    want, bound, _ = DR.attend_tree(cache, q, parents, table, lens, starts, 64 ** -0.5, 0)
    R.close(out[:64], want[:64], bound[:64])
    assert torch.isnan(out[64:]).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G,told,ctx", [(1, 2, 700), (8, 5, 300), (8, 5, 3000), (8, 9, 300), (4, 16, 5000)])
def test_more_nodes_and_keys_than_the_launch_was_told_of(G, told, ctx, D):
    """max_new and max_len choose the launch; what the device's arrays say is what is done."""
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([ctx, 70], [64, 37], 2, G, D, 16, seed=told)
    parents = trees([64, 37])
    out = ops.cache_attend_tree(cache, q, parents, table, lens, starts, max_new=told, max_len=ctx // 2)
    want, bound, _ = DR.attend_tree(cache, q, parents, table, lens, starts, D ** -0.5, 0)
    R.close(out, want, bound)


@pytest.mark.parametrize("G", [2, 16])
def test_starts_and_lengths_out_of_range(G):
    """Queries that are not tokens of q are left out; trees longer than what is cached see less; rows behind stay."""
    from paper_2606_03770_gb300 import ops
    cache, q, table, _, _ = setup([100, 100, 100], [9, 9, 9], 2, G, 64, 16, seed=11)
    parents = trees([27])
    for lens, starts in (([100, 5, 0], [0, 9, 18, 27]), ([50, 60, -5], [-3, 4, 30, 40]), ([2 ** 31 - 1, 7, 9], [5, 5, 2, 20])):
        lens, starts = i32(lens), i32(starts)
        out = torch.full_like(q, 7.0)
        ops.cache_attend_tree(cache, q, parents, table, lens, starts, max_new=20, max_len=100, out=out)
        want, bound, written = DR.attend_tree(cache, q, parents, table, lens, starts, 64 ** -0.5, 0)
        # (a token of two requests is either's)
        twice = [t for t in range(27) if sum(int(starts[r]) <= t < int(starts[r + 1]) for r in range(3)) > 1]
        written[twice] = False
        R.close(out[written], want[written], bound[written])
        written[twice] = True
        assert (out[~written] == 7.0).all()


@pytest.mark.parametrize("G", [1, 16])
def test_not_finite_in_hidden_places(G):
    """A NaN key or value of a node spoils the nodes below it only; a NaN query its own row."""
    from paper_2606_03770_gb300 import ops
    new, before = 12, 50
    par = random_tree(new, 3, 0.1)
    cache, q, table, lens, starts = setup([before + new], [new], 2, G, 128, 16, seed=12)
    kw = dict(max_new=new, max_len=before + new)
    clean = ops.cache_attend_tree(cache, q, i32(par), table, lens, starts, **kw)
    sick = 4
    at = before + sick
    for scales in (cache.k_scales, cache.v_scales):
        kept = scales.clone()
        scales[table[0, at // 16].long(), :, at % 16] = math.nan
        out = ops.cache_attend_tree(cache, q, i32(par), table, lens, starts, **kw)
        for i in range(new):
            if sick in DR.way(par, 0, i, new):
                assert torch.isnan(out[i]).all()
            else:
                assert torch.isfinite(out[i]).all()
                assert torch.allclose(out[i].float(), clean[i].float(), atol=2e-2)
        scales.copy_(kept)
    q[7, 3 % q.shape[1]] = math.nan
    out = ops.cache_attend_tree(cache, q, i32(par), table, lens, starts, **kw)
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[7, 3 % q.shape[1]] = True
    assert torch.isnan(out[bad]).all() and torch.isfinite(out[~bad]).all()


@pytest.mark.parametrize("B,G,new,ctx", [(2, 1, 12, 200), (2, 16, 12, 200), (2, 8, 7, 200), (8, 8, 16, 700), (4, 8, 7, 1100), (1, 8, 7, 20000),
                                         (1, 16, 12, 20000)])
@pytest.mark.parametrize("D", [64, 128])
def test_not_finite_far_below_the_largest_score(B, G, new, ctx, D):
    """A NaN among seen keys or values spoils every row, however little the tiles around it weigh beside the others."""
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([ctx] * B, [new] * B, 2, G, D, 16, seed=ctx)
    q *= 60                                                  # (scores hundreds apart: far tiles' factors are 0 in 32 bits)
    parents, kw = trees([new] * B), dict(max_new=new, max_len=ctx)
    assert torch.isfinite(ops.cache_attend_tree(cache, q, parents, table, lens, starts, **kw)).all()
    for at in (0, 5, 40, 64 + 3, 64 + 37, 130, ctx // 2, ctx - new - 1):
        for scales in (cache.k_scales, cache.v_scales):
            kept = scales.clone()
            scales[table[:, at // 16].long(), :, at % 16] = math.nan
            out = ops.cache_attend_tree(cache, q, parents, table, lens, starts, **kw)
            assert torch.isnan(out).all(), at
            scales.copy_(kept)


def test_windows_choose_the_launch():
    """What is chosen goes by the keys that are seen, not by a context that a window hides."""
    import ctypes
    from paper_2606_03770_gb300 import e2ga, ops
    cache = ops.Cache.empty(4, 16, 8, 128)

    def workspace(new, max_len, window, dtype):
        a = ops.e2_attend_args(new, dtype, 8, 1, None, 1, 1, None, None, new, max_len, 1.0, window)
        return e2ga.load().e2_cache_attend_tree_workspace(cache.ref, ctypes.byref(a))

    ops.load()
    for dtype in (ops.E2_F16, ops.E2_BF16):
        for new in (1, 8, 9, 16, 17, 64):
            for window in (100, 9000, 30000):
                assert workspace(new, 10 ** 6, window, dtype) == workspace(new, window + new, window, dtype)


def test_strided_queries_and_given_outputs():
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([300, 90], [9, 4], 2, 4, 128, 64, seed=13)
    parents = trees([9, 4])
    wide = torch.randn(13, 12, 128, device="cuda").to(BF)
    wide[:, 2:10] = q
    out = torch.full((13, 11, 128), 3.0, device="cuda", dtype=BF)
    kw = dict(max_new=9, max_len=300)
    want = ops.cache_attend_tree(cache, q, parents, table, lens, starts, **kw)
    got = ops.cache_attend_tree(cache, wide[:, 2:10], parents, table, lens, starts, out=out[:, 1:9], **kw)
    assert torch.equal(got, want) and (out[:, 0] == 3).all() and (out[:, 9:] == 3).all()
    assert torch.equal(ops.cache_attend_tree(cache, q, parents, table, lens, starts), want)      # sizes read from the device


# ---- verification -----------------------------------------------------------------------------------
def batch_of(news, V, dtype=F32, pad=0, seed=0, draft=True, std=3.0, near=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T = sum(news)
    x = std * torch.randn(T, V + pad, generator=g, device="cuda")
    y = x + near * torch.randn(T, V + pad, generator=g, device="cuda")
    parents, starts = trees(news, seed), i32([0] + torch.tensor(news).cumsum(0).tolist())
    ids = torch.zeros(T, **I32)
    s = 0
    for n in news:
        for i in range(n):
            if i:
                row = y[s + int(parents[s + i]), :V].to(dtype).float()
                ids[s + i] = torch.multinomial(torch.softmax(row, 0), 1, generator=g)[0].int()
        s += n
    u = torch.rand(T, generator=g, device="cuda")
    x, y = x.to(dtype)[:, :V], y.to(dtype)[:, :V]
    return [x, ids, parents, starts, u, y if draft else None]


def check_verify(x, ids, parents, starts, u, draft, temperature=None, max_new=None):
    from paper_2606_03770_gb300 import ops
    most = int((starts[1:] - starts[:-1]).max()) if max_new is None else max_new
    got = ops.verify_drafts(x, ids, parents, starts, u, draft=draft, temperature=temperature, max_new=most)
    want = DR.verify(x, ids, parents, starts, u, draft, temperature, most)
    for g, w, n in zip(got, want, ("kept", "nodes", "answer")):
        assert g.dtype is torch.int32 and g.tolist() == w, n
    return got


@pytest.mark.parametrize("dtype", [HALF, BF, F32])
@pytest.mark.parametrize("V", [1, 2, 31, 33, 500, 4097, 32000, 50001])
@pytest.mark.parametrize("draft", [True, False])
def test_vocabularies(dtype, V, draft):
    for B in (1, 9):
        news = [1 + (5 * r) % 8 for r in range(B)]
        s = batch_of(news, V, dtype, pad=(3 if V % 2 else 0), seed=V + B, draft=draft)
        check_verify(*s)
        check_verify(*s, temperature=torch.tensor([(0.0, 0.5, 1.7)[r % 3] for r in range(B)], device="cuda"))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_a_large_vocabulary(dtype):
    check_verify(*batch_of([8] * 8, 128256, dtype, seed=1))
    check_verify(*batch_of([64], 128256, dtype, seed=2, near=2.0))
    check_verify(*batch_of([4] * 40, 128256, dtype, seed=3, draft=False))


@pytest.mark.parametrize("near", [0.0, 0.3, 2.0, 6.0])
@pytest.mark.parametrize("draft", [True, False])
def test_bushes(near, draft):
    """Many children of one node, drafts far from the target: many rejections, one after the other, and
    the same token drafted again."""
    n = 40
    s = batch_of([n] * 6, 600, seed=int(10 * near), near=near, draft=draft, std=2.0)
    s[2] = i32(([-1] + [0] * (n - 1)) * 6)
    g = torch.Generator(device="cuda").manual_seed(5)
    for r in range(6):
        row = torch.softmax((s[0] if s[5] is None else s[5])[r * n].float(), 0)
        s[1][r * n + 1:(r + 1) * n] = torch.multinomial(row, n - 1, replacement=True, generator=g).int()
    s[4] = (1 - 0.2 * s[4]) if near else s[4]
    check_verify(*s)


def neighbours(x):
    """The 32-bit numbers next to a 64-bit one, below and above."""
    y = torch.tensor(x, dtype=torch.float64).float()
    lo = y if float(y) <= x else torch.nextafter(y, torch.tensor(0.0))
    return float(lo), float(torch.nextafter(lo, torch.tensor(2.0)))


@pytest.mark.parametrize("V", [300, 20000])
@pytest.mark.parametrize("heat", [1.0, 0.37])
def test_random_numbers_next_to_a_border(V, heat):
    """The first child's border p(x) / q(x) and the answer's, a sum of probabilities, by their 32-bit neighbours."""
    n = 24
    for draft in (True, False):
        s = batch_of([2] * n, V, seed=V, draft=draft, near=1.0)
        x, ids, parents, starts, u, y = s
        for r in range(n):
            p = DR.probabilities(x[2 * r], heat)
            if r % 2:
                # a token that may be rejected
                q = DR.probabilities(y[2 * r], heat) if draft else torch.ones_like(p)
                token = int(torch.topk(torch.where(p < q, p, 0.0), 8).indices[r % 8])
                ids[2 * r + 1] = token
                u[2 * r + 1] = neighbours(float(p[token] / q[token]))[r // 2 % 2]
            else:
                parents[2 * r + 1] = -1                      # (no child: the answer is drawn from p)
                v = int(torch.topk(p, 16).indices[r % 16])
                u[2 * r] = neighbours(float(torch.cumsum(p, 0)[v]))[r // 2 % 2]
        check_verify(*s, temperature=torch.full((n,), heat, device="cuda"))


def test_flat_and_peaked_rows():
    V = 40000
    for draft in (True, False):
        s = batch_of([3] * 12, V, seed=4, draft=draft)
        for x in [s[0]] + ([s[5]] if draft else []):
            x[0:3] = 0.0
            x[3:6] = torch.finfo(F32).min
            x[6:9] = 1e30
            x[9:12, 7] = 200.0
            x[12:15] *= 1e-20
            x[15:18] = torch.arange(V, device="cuda") * 1e-3
            x[18:21] = -torch.arange(V, device="cuda") * 1.0
        check_verify(*s)
        check_verify(*s, temperature=torch.tensor([1e-30, 1e30, 3e-39, 0.0, 1e4, 0.01] * 2, device="cuda"))


@pytest.mark.parametrize("dtype", [HALF, BF, F32])
@pytest.mark.parametrize("V", [40, 30000])
def test_forbidden_tokens(dtype, V):
    g = torch.Generator(device="cuda").manual_seed(6)
    s = batch_of([4] * 9, V, dtype, seed=6)
    for r, share in enumerate((0.1, 0.5, 0.9, 0.999)):
        s[0][4 * r:4 * r + 4].masked_fill_(torch.rand(4, V, generator=g, device="cuda") < share, -math.inf)
        s[5][4 * r:4 * r + 4].masked_fill_(torch.rand(4, V, generator=g, device="cuda") < share, -math.inf)
    for x in (s[0], s[5]):
        x[:, V // 3] = 0.0                                   # (every row has a token)
    s[0][16:20] = -math.inf                                  # one token left, which is drafted or is not
    s[0][16:20, 5] = -80.0
    s[1][17] = 5
    check_verify(*s)
    s[5] = None
    check_verify(*s)
    check_verify(*s, temperature=torch.zeros(9, device="cuda"))


@pytest.mark.parametrize("dtype", [HALF, BF, F32])
@pytest.mark.parametrize("V", [50, 20000])
def test_rows_without_a_distribution(dtype, V):
    """NaN, +inf or nothing, in the target's rows or the draft's, at node 0 and below it."""
    for draft in (True, False):
        for heat in (1.0, 0.0):
            s = batch_of([3] * 10, V, dtype, seed=7, draft=draft)
            s[2] = i32([-1, 0, 1] * 10)
            s[4][1::3] = 0.0                                 # (node 1 is accepted where it can be)
            s[1][1::3] = s[0][0::3].float().argmax(1).int()
            s[0][0, 3] = math.nan
            s[0][3, V - 1] = math.inf
            s[0][6] = -math.inf
            s[0][10, 1] = math.nan
            s[0][13] = math.inf
            s[0][16] = -math.inf
            if draft:
                s[5][18, 2] = math.nan
                s[5][22, 2] = math.inf
                s[5][24] = -math.inf
                s[5][29, 2] = math.nan                       # (a leaf's draft is not asked for)
            check_verify(*s, temperature=torch.full((10,), heat, device="cuda"))


def test_random_numbers_temperatures_and_ids_out_of_range():
    s = batch_of([4] * 12, 1000, seed=8)
    s[4][0:24:2] = torch.tensor([-1.0, math.nan, math.inf, -math.inf, 1.0, 2.0] * 2, device="cuda")
    s[1][1:20:3] = i32([-1, 1000, 2 ** 31 - 1, -2 ** 31, 5, 1000, -1])
    check_verify(*s)
    check_verify(*s[:5], None)
    heat = torch.tensor([1.0, -1.0, math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-45, 3e38, 0.5, 0.5, 0.5], device="cuda")
    got = check_verify(*s, temperature=heat)
    assert got[2][1:5, 0].tolist() == [-1] * 4


def test_ties_go_to_the_first():
    s = batch_of([3] * 3, 5000, seed=9)
    s[0].zero_()
    s[0][3:6, 77::100] = 2.0
    s[0][6:9, 4999] = 1.0
    s[1][:] = i32([0, 0, 0, 0, 77, 177, 0, 4998, 4999])
    check_verify(*s, temperature=torch.zeros(3, device="cuda"))


@pytest.mark.parametrize("dtype", [HALF, BF, F32])
def test_rows_where_they_lie(dtype):
    """Rows of other strides and alignments than one another's, and of a call with a single row."""
    V = 6001
    for seed, (a, b) in enumerate(((0, 3), (8, 0), (5, 1), (16, 16))):
        s = batch_of([5, 3, 8], V, dtype, seed=seed)
        x, y = (torch.full((16, V + 2 * k + 1), math.nan, device="cuda", dtype=dtype) for k in (a, b))
        x[:, a:a + V], y[:, b:b + V] = s[0], s[5]
        check_verify(x[:, a:a + V], *s[1:5], y[:, b:b + V])
    s = batch_of([1], V, dtype, seed=5)
    wide = torch.full((3, V + 3), math.nan, device="cuda", dtype=dtype)
    for at in (0, 1, 2):
        wide[1, at:at + V] = s[0][0]
        check_verify(wide[1:2, at:at + V], *s[1:5], None)


def test_many_requests():
    s = batch_of([2] * 400, 3000, BF, seed=13)
    check_verify(*s)
    check_verify(*batch_of([1, 0, 3] * 100, 9001, F32, seed=14, draft=False))


def test_starts_out_of_range():
    s = batch_of([4] * 4, 300, seed=10)
    for starts in ([0, 0, 16, 16, 16], [-4, 4, 8, 12, 20], [8, 4, 0, 16, 12], [0, 4, 8, 2 ** 31 - 1, 16]):
        s[3] = i32(starts)
        check_verify(*s, max_new=5)
    s[3] = i32([0, 4, 8, 12, 16])
    check_verify(*s, max_new=2)                               # nodes beyond are not looked at
    check_verify(*s, max_new=64)
    check_verify(*s, max_new=0)


def test_the_same_rows_for_draft_and_target():
    """p = q: every drafted token is accepted, or has no probability in both; what is left of P then counts as nothing."""
    s = batch_of([6] * 8, 9000, seed=11)
    s[0][:, :4000] = -math.inf
    s[5] = s[0]
    s[1][1::6] = 17
    check_verify(*s)


def test_a_token_is_the_same_however_rows_are_split():
    """One request alone, in a small batch and in a large one: other clusters, the same decisions."""
    V = 128256
    s = batch_of([5], V, BF, seed=12)
    one = [x.tolist() for x in check_verify(*s)]
    for B in (20, 80, 160):
        rows = torch.arange(5, device="cuda").repeat(B)
        from paper_2606_03770_gb300 import ops
        got = ops.verify_drafts(s[0][rows], s[1][rows], s[2][rows], torch.arange(B + 1, **I32) * 5, s[4][rows], draft=s[5][rows],
                                max_new=5)
        for g, w in zip(got, one):
            assert g.tolist() == w * B


def only(V, tokens, logits):
    """A row in which all but these are forbidden."""
    row = torch.full((V,), -math.inf, device="cuda")
    row[tokens] = logits
    return row


@pytest.mark.parametrize("dtype", [HALF, BF, F32])
@pytest.mark.parametrize("V", [700, 20000])
@pytest.mark.parametrize("u0", [0.0, 1.0])
def test_rejected_tokens_alone_in_their_part_of_a_row(dtype, V, u0):
    """Rejected tokens leave nothing where nothing else is allowed: the answer is the first token that is left, or the last."""
    n, B = 6, 40
    g = torch.Generator(device="cuda").manual_seed(20)
    s = batch_of([n] * B, V, F32, seed=20, draft=False)
    s[2] = i32(([-1] + [0] * (n - 1)) * B)
    s[4][:] = 1.0
    s[4][::n] = u0
    for r in range(B):
        far = 60 + 3 * r % 40
        drafted = torch.randperm(60, generator=g, device="cuda")[:n - 1 - r % 3]
        left = far + torch.randperm(V - 160, generator=g, device="cuda")[:2 + r % 9]
        if u0:
            drafted, left = V - 1 - drafted, V - 1 - left
        tokens = torch.cat([drafted, left])
        s[0][r * n] = only(V, tokens, 2 * torch.randn(len(tokens), generator=g, device="cuda"))
        s[1][r * n + 1:(r + 1) * n] = drafted[torch.arange(n - 1, device="cuda") % len(drafted)].int()
    s[0] = s[0].to(dtype)
    kept, _, answer = check_verify(*s)
    assert kept.tolist() == [1] * B and (answer[:, 0] >= 0).all()
    check_verify(*s, temperature=torch.full((B,), 0.7, device="cuda"))


@pytest.mark.parametrize("V", [300, 20000])
def test_what_is_left_beside_a_rejected_token_of_nearly_all(V):
    """The others' shares, and the next child's, next to their borders after a token of 1 - 2^-10 to 1 - 2^-33 was rejected."""
    n, B = 3, 96
    g = torch.Generator(device="cuda").manual_seed(21)
    s = batch_of([n] * B, V, F32, seed=21, draft=False)
    x, ids, _, _, u, _ = s
    s[2] = i32([-1, 0, 0] * B)
    for r in range(B):
        tokens = torch.randperm(V, generator=g, device="cuda")[:40]
        logits = torch.randn(40, generator=g, device="cuda")
        logits[0] = torch.logsumexp(logits[1:], 0) + (10 + r % 24) * math.log(2.0)
        x[n * r] = only(V, tokens, logits)
        p = DR.probabilities(x[n * r], 1.0)
        p[tokens[0]] = 0
        p /= p.sum()
        ids[n * r + 1], u[n * r + 1] = tokens[0].int(), 1.0
        ids[n * r + 2] = tokens[1].int()
        if r % 2:
            u[n * r + 2] = neighbours(float(p[tokens[1]]))[r // 2 % 2]
        else:
            # (the second is rejected, too)
            u[n * r + 2] = 1.0
            p[tokens[1]] = 0
            border = torch.cumsum(p / p.sum(), 0)[tokens[2 + r // 2 % 30]]
            u[n * r] = neighbours(float(border))[r // 2 % 2]
    check_verify(*s)


@pytest.mark.parametrize("V", [1000, 20000])
@pytest.mark.parametrize("u0", [0.0, 1.0])
def test_parts_of_a_row_that_draft_and_target_share(V, u0):
    """The same logits in both rows where nothing is left of P, and others elsewhere that sum to the same."""
    n, B = 2, 120
    g = torch.Generator(device="cuda").manual_seed(22)
    s = batch_of([n] * B, V, F32, seed=22)
    x, ids, _, _, u, y = s
    s[2] = i32([-1, 0] * B)
    at = torch.arange(V, device="cuda") if u0 == 0 else torch.arange(V - 1, -1, -1, device="cuda")
    for r in range(B):
        # light and shared; heavy in pairs that change places
        x[n * r] = -math.inf
        light, heavy = at[:V // 4], at[V // 2:V // 2 + 2 + 2 * (r % 3)]
        x[n * r, light] = -25.0 + torch.randn(len(light), generator=g, device="cuda")
        x[n * r, heavy] = torch.randn(len(heavy), generator=g, device="cuda")
        y[n * r] = x[n * r]
        y[n * r, heavy] = x[n * r, heavy.view(-1, 2).flip(1).flatten()]
        ids[n * r + 1] = heavy[int(x[n * r, heavy[0]] > x[n * r, heavy[1]])].int()          # (of less in the target)
    u[1::2] = 1.0
    u[::2] = u0
    from paper_2606_03770_gb300 import ops
    kept, _, answer = ops.verify_drafts(*s[:5], draft=y, max_new=n)
    assert kept.tolist() == [1] * B
    # (of tokens that have as much in both rows 64 bits, too, may leave their rounding)
    for r in range(B):
        p, q = (DR.probabilities(z[n * r], 1.0) for z in (x, y))
        clear = torch.nonzero(p - q > 2.0 ** -36)[0 if u0 == 0 else -1]
        got = int(answer[r, 0])
        assert got >= 0 and (got == int(clear) or abs(float(p[got] - q[got])) < 2.0 ** -36), (r, got, int(clear))


@pytest.mark.parametrize("u0", [0.0, 1.0])
def test_long_parts_of_a_row_that_draft_and_target_share(u0):
    """As above for parts of 192 equal tokens a lane, the draft's logits all a little higher: sums of the two round apart."""
    n, B, V = 2, 160, 65536
    g = torch.Generator(device="cuda").manual_seed(24)
    s = batch_of([n] * B, 8, F32, seed=24)
    s[0], s[5] = torch.full((n * B, V), -math.inf, device="cuda"), torch.full((n * B, V), -math.inf, device="cuda")
    x, ids, _, _, u, y = s
    s[2] = i32([-1, 0] * B)
    sixteenths = lambda *size: torch.randint(-16, 17, size, generator=g, device="cuda") / 16
    at = torch.arange(V, device="cuda") if u0 == 0 else torch.arange(V - 1, -1, -1, device="cuda")
    for r in range(B):
        x[n * r, at[:3 * V // 4]] = -25.0 + sixteenths(1)
        heavy = at[-2:]
        x[n * r, heavy[0]], x[n * r, heavy[1]] = 0.0, 1.0 + r % 3
        y[n * r] = x[n * r]
        y[n * r, heavy] = x[n * r, heavy.flip(0)]
        y[n * r] += sixteenths(1)
        ids[n * r + 1] = heavy[0].int()                      # (of less in the target)
    u[1::2] = 1.0
    u[::2] = u0
    from paper_2606_03770_gb300 import ops
    kept, _, answer = ops.verify_drafts(*s[:5], draft=y, max_new=n)
    assert kept.tolist() == [1] * B
    # (the equal tokens, or the one that has more in the target)
    for r in range(B):
        got = int(answer[r, 0])
        assert got >= 0 and (got == int(at[-1]) or float(x[n * r, got]) < -20), (r, got)


@pytest.mark.parametrize("V", [7, 900, 20000])
def test_rejections_that_leave_next_to_nothing(V):
    """A token of the draft that the target forbids, again and again, where both agree on the rest: each rejection leaves some
    5e-4 of P and P as it was, until what is left is rounding's."""
    n, B = 9, 100
    g = torch.Generator(device="cuda").manual_seed(25)
    rand = lambda: torch.rand(1, generator=g, device="cuda")
    x, y = torch.full((n * B, V), -math.inf, device="cuda"), torch.full((n * B, V), -math.inf, device="cuda")
    ids, u = torch.zeros(n * B, **I32), torch.rand(n * B, generator=g, device="cuda")
    for r in range(B):
        a, b, out = torch.randperm(V, generator=g, device="cuda")[:3]
        x[n * r, a], x[n * r, b] = rand(), -11 + 2 * rand()
        y[n * r] = x[n * r]
        y[n * r, out] = -8 + rand()
        ids[n * r + 1:n * (r + 1)] = out
        # (token a has all but e^-9 at most, and is the answer but for what that leaves)
        u[n * r] = 0.01 + 0.98 * u[n * r]
    parents, starts = i32(([-1] + [0] * (n - 1)) * B), i32(range(0, n * B + 1, n))
    from paper_2606_03770_gb300 import ops
    for children in range(1, n):
        par = torch.where(torch.arange(n * B, device="cuda") % n <= children, parents, -1).int()
        kept, _, answer = ops.verify_drafts(x, ids, par, starts, u, draft=y, max_new=n)
        assert kept.tolist() == [1] * B
        assert answer[:, 0].tolist() == x[::n].argmax(1).tolist(), children


@pytest.mark.parametrize("B,V,dtype", [(160, 1 << 22, BF), (160, 65536, BF), (160, 262144, F32), (2, (1 << 26) + 1357, HALF)])
@pytest.mark.parametrize("draft", [False, True])
def test_long_rows_of_equal_logits(B, V, dtype, draft):
    """The rows whose sums lose most, long ones in one block: random numbers by 2^-13.5 and less beside a child's border, the
    nearest to it, and answers."""
    if draft:
        V //= 2
    g = torch.Generator(device="cuda").manual_seed(23)
    far = [-2 ** -13.5, 2 ** -13.5, -2 ** -14.5, 2 ** -14.5, -2 ** -17, 2 ** -17, -2 ** -20, 2 ** -20, 0.0, 0.0]
    rounds = 1 if B > 2 else 6
    for k in range(rounds):
        s = [torch.empty(2 * B, V, dtype=dtype, device="cuda"), torch.zeros(2 * B, **I32), i32([-1, 0] * B), i32(range(0, 2 * B + 1, 2)),
             torch.rand(2 * B, generator=g, device="cuda"), torch.empty(2 * B, V, dtype=dtype, device="cuda") if draft else None]
        for r in range(B):
            for z in s[0::5] if draft else s[:1]:
                z[2 * r:2 * r + 2] = -3 * torch.rand(2, 1, generator=g, device="cuda")
                z[2 * r:2 * r + 2, 0] = 0.0
            if draft:
                s[5][2 * r, V // 2:] = -math.inf             # (so that q is some 2 p)
            token = 1 + (7919 * r + 31 * k) % (V // 3)
            p = DR.probabilities(s[0][2 * r], 1.0)[token]
            if draft:
                p /= DR.probabilities(s[5][2 * r], 1.0)[token]
            s[1][2 * r + 1] = token
            s[4][2 * r + 1] = float(p) * (1 + far[(r + 2 * k) % len(far)])
        check_verify(*s)


# ---- keeping ----------------------------------------------------------------------------------------
def a_way(parents, n, g):
    path = [0] if n else []
    while path:
        below = [i for i in range(path[-1] + 1, n) if parents[i] == path[-1]]
        if not below:
            break
        path.append(below[int(torch.randint(0, len(below), (1,), generator=g))])
    return path


def check_keep(caches, table, lens, starts, nodes, kept, **kw):
    from paper_2606_03770_gb300 import ops
    want = [DR.keep(c, table, lens, starts, nodes, kept) for c in caches]
    got = ops.cache_keep(ops.CacheLayers(caches), table, lens, starts, nodes, kept, **kw)
    for c, (arrays, out) in zip(caches, want):
        assert got.tolist() == out
        for a, b in zip((c.k_codes, c.k_scales, c.v_codes, c.v_scales), arrays):
            assert torch.equal(a, b)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads", [1, 3, 8])
@pytest.mark.parametrize("page", [16, 64])
def test_keep(D, heads, page):
    g = torch.Generator().manual_seed(D + heads)
    news = [7, 1, 0, 64, 20]
    lens = [90, 1, 0, 64, 31]
    caches = [setup(lens, news, heads, 1, D, page, seed=i)[0] for i in range(3)]
    _, _, table, lens_t, starts = setup(lens, news, heads, 1, D, page, seed=0)
    par = [random_tree(n, r) for r, n in enumerate(news)]
    ways = [a_way(par[r], n, g) for r, n in enumerate(news)]
    nodes = i32([w + [-1] * (64 - len(w)) for w in ways])
    check_keep(caches, table, lens_t, starts, nodes, i32([len(w) for w in ways]))


def test_nodes_that_go_where_others_come_from():
    """Every node to another's place: a rotation, a mirror, the same node everywhere; whole trees of 64."""
    news, lens = [64, 64, 64, 5], [100, 64, 300, 9]
    for D in (64, 128):
        cache, _, table, lens_t, starts = setup(lens, news, 2, 1, D, 16, seed=1)
        nodes = i32([[(k + 1) % 64 for k in range(64)], [63 - k for k in range(64)], [9] * 64, [4, 3, 2, 1, 0] + [77] * 59])
        check_keep([cache], table, lens_t, starts, nodes, i32([64, 64, 64, 5]))


def test_keep_out_of_range():
    """Nodes, counts, lengths and pages out of range: nothing else is moved, the rest is."""
    news, lens = [8, 8, 8, 8, 8], [40, 3, 40, 40, 40]
    cache, _, table, lens_t, starts = setup(lens, news, 2, 1, 128, 16, seed=2)
    table[2] = i32([3, -1, 10 ** 6][:table.shape[1]])
    lens_t[3] = 49
    lens_t[4] = -20
    nodes = i32([[0, -3, 8, 5, 2 ** 31 - 1, -2 ** 31, 7, 1], [0, 2, 4, 6, 7, 5, 3, 1], [7, 6, 5, 4, 3, 2, 1, 0], [2, 1, 0, 7, 6, 5, 4, 3],
                 [1, 2, 3, 4, 5, 6, 7, 0]])
    for kept in ([8, 8, 8, 8, 8], [100, -1, 2 ** 31 - 1, -2 ** 31, 3]):
        check_keep([cache], table, lens_t, starts, nodes, i32(kept))
    check_keep([cache], table, lens_t, i32([8, 4, 100, 3, 3, 12]), nodes, i32([8] * 5))
    check_keep([cache], table, lens_t, starts, nodes[:, :3], i32([8] * 5))
    check_keep([cache], table, lens_t, starts, nodes[:, :0], i32([8] * 5))


# ---- refusals, streams, graphs ------------------------------------------------------------------------
def test_refusals():
    from paper_2606_03770_gb300 import e2ga, ops
    cache, q, table, lens, starts = setup([40, 30], [3, 2], 2, 2, 64, 16)
    parents = trees([3, 2])
    tree = lambda **kw: ops.cache_attend_tree(**{**dict(cache=cache, q=q, parents=parents, table=table, lens=lens, starts=starts,
                                                        max_new=3, max_len=40), **kw})
    tree()
    for kw in (dict(parents=parents.long()), dict(parents=parents[:4]), dict(parents=parents.cpu()), dict(q=q.float()),
               dict(parents=torch.zeros(10, **I32)[::2]), dict(q=q[:, :, :32]), dict(lens=lens[:1]), dict(starts=starts.long())):
        with pytest.raises(ValueError):
            tree(**kw)
    for kw in (dict(max_new=65), dict(max_new=-1), dict(window=-1), dict(scale=math.nan), dict(q=q[:, :3])):
        with pytest.raises(e2ga.E2Error):
            tree(**kw)
    s = batch_of([3, 2], 100, seed=0)
    verify = lambda **kw: ops.verify_drafts(**{**dict(logits=s[0], ids=s[1], parents=s[2], starts=s[3], uniforms=s[4], draft=s[5],
                                                      max_new=3), **kw})
    verify()
    for kw in (dict(logits=s[0].double()), dict(draft=s[5].half()), dict(draft=s[5][:, :99]), dict(ids=s[1].long()), dict(uniforms=s[4][:4]),
               dict(parents=s[2].cpu()), dict(starts=s[3][None]), dict(starts=s[3][:0]), dict(temperature=torch.ones(3, device="cuda")),
               dict(temperature=torch.ones(2, device="cuda").double()), dict(max_new=65), dict(max_new=-1),
               dict(logits=s[0].clone().requires_grad_()), dict(uniforms=s[4].clone().requires_grad_()),
               dict(draft=s[5].clone().requires_grad_()), dict(temperature=torch.ones(2, device="cuda", requires_grad=True))):
        with pytest.raises(ValueError):
            verify(**kw)
    layers = ops.CacheLayers([cache])
    nodes, kept = i32([[0, 2], [0, 1]]), i32([2, 2])
    keep = lambda **kw: ops.cache_keep(**{**dict(layers=layers, table=table, lens=lens, starts=starts, nodes=nodes, kept=kept), **kw})
    assert keep().tolist() == [39, 30]
    for kw in (dict(layers=cache), dict(layers=[cache]), dict(nodes=nodes.long()), dict(nodes=nodes[:1]), dict(kept=kept[:1]),
               dict(nodes=torch.zeros(2, 65, **I32)), dict(lens_out=kept.long()), dict(table=table.long())):
        with pytest.raises(ValueError):
            keep(**kw)
    with pytest.raises(e2ga.E2Error):
        keep(lens_out=lens)
    for shared in (kept, starts[:-1], starts[1:], nodes.view(-1)[1:3], table.view(-1)[:2], table.view(-1)[-2:]):
        with pytest.raises(e2ga.E2Error, match="lens_out"):
            keep(lens_out=shared)
    big = setup([9000], [9], 2, 4, 64, 16)
    with pytest.raises(e2ga.E2Error, match="workspace"):
        ops.cache_attend_tree(*big[:2], trees([9]), *big[2:], max_new=9, max_len=9000, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    with pytest.raises(AttributeError):
        layers.arrays = None
    other = ops.Cache.empty(4, 16, 1, 64)
    half = ops.Cache(cache.k_codes, cache.k_scales, cache.k_codes, cache.v_scales)
    for caches in ([cache, other], [cache, cache], [half]):
        with pytest.raises(ValueError):
            ops.CacheLayers(caches)
    grad = ops.Cache(cache.k_codes, cache.k_scales.clone().requires_grad_(), cache.v_codes, cache.v_scales)
    with pytest.raises(ValueError, match="gradient"):
        keep(layers=ops.CacheLayers([grad]))
    with pytest.raises(ValueError, match="gradient"):
        tree(cache=grad)


def test_layers_that_share_memory_are_refused():
    """Codes or scales, of two layers or within one, whole or in part."""
    from paper_2606_03770_gb300 import ops
    shape = (6, 2, 16)
    codes = lambda: torch.zeros(*shape, 64, dtype=torch.uint8, device="cuda")
    scales = lambda: torch.zeros(*shape, 2, 2, dtype=torch.float16, device="cuda")
    a = (codes(), scales(), codes(), scales())
    assert len(ops.CacheLayers([ops.Cache(*a), ops.Cache(codes(), scales(), codes(), scales())])) == 2
    inside = a[0].view(-1)[256:256 + scales().nbytes].view(torch.float16).view(*shape, 2, 2)
    longer = torch.zeros(2 * scales().numel() - 8, dtype=torch.float16, device="cuda")
    first, second = longer[:scales().numel()].view(*shape, 2, 2), longer[scales().numel() - 8:].view(*shape, 2, 2)
    for caches in ([a, (codes(), a[1], codes(), scales())], [a, (codes(), scales(), codes(), a[3])], [a, (codes(), a[3], codes(), scales())],
                   [(codes(), a[1], codes(), a[1])], [a, (codes(), inside, codes(), scales())], [(codes(), first, codes(), second)],
                   [a, (codes(), scales(), codes(), scales()), (codes(), scales(), a[0], scales())], [a, (codes(), first, codes(), scales()),
                                                                                                     (codes(), second, codes(), scales())]):
        with pytest.raises(ValueError, match="share memory"):
            ops.CacheLayers([ops.Cache(*c) for c in caches])
    # (next to one another is apart)
    whole = torch.zeros(4, scales().numel(), dtype=torch.float16, device="cuda")
    s = [whole[i].view(*shape, 2, 2) for i in range(4)]
    assert len(ops.CacheLayers([ops.Cache(codes(), s[2], codes(), s[0]), ops.Cache(codes(), s[1], codes(), s[3])])) == 2


class NoBinding:
    """The compiled binding, going by."""
    attend_tree = verify = keep = staticmethod(lambda *a: None)


@pytest.mark.parametrize("G", [1, 8])
def test_the_binding_in_python_is_the_same(G, monkeypatch):
    from paper_2606_03770_gb300 import ops
    s, run = step(3, 9, 70, 2, G, 500, 4)
    want = run()
    heat = torch.tensor([0.0, 0.5, 1.0], device="cuda")
    x = s["x"]
    more = lambda: (ops.verify_drafts(x[0], x[1], x[2], s["starts"], x[4], draft=x[5], temperature=heat, max_new=20)
                    + (ops.cache_attend_tree(s["cache"], s["q"], s["parents"], s["table"], s["lens"], s["starts"], max_new=9, max_len=79,
                                             scale=0.3, window=50, out=torch.empty_like(s["q"])),
                       ops.cache_attend_tree(s["cache"], s["q"], s["parents"], s["table"], s["lens"], s["starts"], max_new=9, max_len=79,
                                             workspace=torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))))
    want += more()
    assert ops.binding().verify(x[0], x[1], x[2], s["starts"], x[4], x[5], None, 9) is not None
    assert ops.binding().attend_tree(s["cache"].fast, s["q"], s["parents"], s["table"], s["lens"], s["starts"], 9, 79, None, 0, None, None) is not None
    assert ops.binding().keep(s["layers"].fast, s["table"], s["lens"], s["starts"], want[3][:, :0].new_zeros(3, 2), s["lens"].new_zeros(3), None) is not None
    monkeypatch.setattr(ops, "_binding", NoBinding)
    got = run() + more()
    for a, b in zip(got, want):
        assert a.dtype is b.dtype and torch.equal(a, b)


def test_refusals_without_the_binding(monkeypatch):
    from paper_2606_03770_gb300 import ops
    monkeypatch.setattr(ops, "_binding", NoBinding)
    test_refusals()


def test_empty_calls():
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([40], [3], 2, 2, 64, 16)
    none = torch.zeros(0, **I32)
    out = ops.cache_attend_tree(cache, q[:0], none, table, lens, i32([0, 0]))
    assert out.shape == (0, 4, 64)
    got = ops.verify_drafts(torch.zeros(0, 10, device="cuda"), none, none, i32([0]), torch.zeros(0, device="cuda"))
    assert [x.shape for x in got] == [(0,), (0, 0), (0, 0)]
    got = ops.verify_drafts(torch.zeros(0, 10, device="cuda"), none, none, i32([0, 0, 0]), torch.zeros(0, device="cuda"), max_new=2)
    assert [x.tolist() for x in got] == [[0, 0], [[-1, -1]] * 2, [[-1, -1]] * 2]
    assert ops.cache_keep(ops.CacheLayers([cache]), table[:0], lens[:0], i32([0]), torch.zeros(0, 4, **I32), none).shape == (0,)


def step(B, new, before, Hkv, G, V, seed):
    """A step's operators over one state: what a program keeps, and what a step does."""
    from paper_2606_03770_gb300 import ops
    D, page = 128, 16
    cache, q, table, lens, starts = setup([before + new] * B, [new] * B, Hkv, G, D, page, seed=seed, extra_cols=1)
    g = torch.Generator(device="cuda").manual_seed(seed)
    par = random_tree(new, seed)
    depth = [len(DR.way(par, 0, i, new)) - 1 for i in range(new)]
    s = dict(cache=cache, layers=ops.CacheLayers([cache]), table=table, lens=lens, starts=starts, parents=i32(par * B), new=new,
             k=torch.randn(B * new, Hkv, D, generator=g, device="cuda").to(BF),
             v=torch.randn(B * new, Hkv, D, generator=g, device="cuda").to(BF), q=q, max_len=before + new)
    pos = torch.tensor([before + d for d in depth] * B, **I32)
    at = before + torch.arange(new, device="cuda").repeat(B)
    req = torch.arange(B, device="cuda").repeat_interleave(new)
    angle = torch.arange(before + new, device="cuda")[:, None] * 0.01 * torch.arange(1, 65, device="cuda")
    s.update(positions=pos, slots=table.long()[req, at // page] * page + at % page, cos=angle.cos().float(), sin=angle.sin().float())
    s["w"] = torch.randn(Hkv * G * D, V, generator=g, device="cuda") * 0.5
    s["x"] = batch_of([new] * B, V, seed=seed)
    s["x"][2] = s["parents"]

    def run():
        q = ops.cache_append(cache, s["k"], s["v"], s["slots"], pos, s["cos"], s["sin"], q=s["q"])
        a = ops.cache_attend_tree(cache, q, s["parents"], table, lens, starts, max_new=new, max_len=s["max_len"])
        logits = a.flatten(1).float() @ s["w"]
        kept, nodes, answer = ops.verify_drafts(logits, s["x"][1], s["parents"], starts, s["x"][4], draft=s["x"][5], max_new=new)
        return a, logits, kept, nodes, answer, ops.cache_keep(s["layers"], table, lens, starts, nodes, kept)

    return s, run


@pytest.mark.parametrize("G", [1, 8])
def test_a_whole_step(G):
    """Append, attend, verify, keep, each against its formula on what the one before gave."""
    s, run = step(3, 9, 70, 2, G, 500, 3)
    cache = s["cache"]
    s["x"][4] *= 0.3                                             # (most are accepted)
    a, logits, kept, nodes, answer, lens = run()
    # the cache before the move: appended again, on a copy
    from paper_2606_03770_gb300 import ops
    copy = ops.Cache(*(x.clone() for x in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)))
    q = ops.cache_append(copy, s["k"], s["v"], s["slots"], s["positions"], s["cos"], s["sin"], q=s["q"])
    want, bound, _ = DR.attend_tree(copy, q, s["parents"], s["table"], s["lens"], s["starts"], 128 ** -0.5, 0)
    R.close(a, want, bound)
    ref = DR.verify(logits, s["x"][1], s["parents"], s["starts"], s["x"][4], s["x"][5], None, 9)
    assert [kept.tolist(), nodes.tolist(), answer.tolist()] == list(ref)
    arrays, out = DR.keep(copy, s["table"], s["lens"], s["starts"], nodes, kept)
    assert lens.tolist() == out and max(out) > 70 + 1
    for x, y in zip((cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), arrays):
        assert torch.equal(x, y)
    # the next token sees the kept ones where a chain would have put them
    for r in range(3):
        path = nodes[r, :int(kept[r])].tolist()
        at = torch.arange(70, 70 + len(path), device="cuda")
        slots = s["table"].long()[r, at // 16] * 16 + at % 16
        got = ops.cache_read(cache, slots, torch.float32)
        old = torch.tensor([70 + i for i in path], device="cuda")
        was = ops.cache_read(copy, s["table"].long()[r, old // 16] * 16 + old % 16, torch.float32)
        assert torch.equal(got[0], was[0]) and torch.equal(got[1], was[1])


def test_captured_steps_replay():
    """A step in a graph, replayed on other contents of the same tensors, next to another graph's."""
    s, run = step(2, 7, 40, 2, 4, 3000, 5)
    t, other = step(4, 3, 90, 1, 16, 700, 6)
    run(), other()
    graphs = []
    for f in (run, other):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = f()
        graphs.append((g, out))
    torch.cuda.synchronize()
    for seed in (1, 2, 3):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for x in (s, t):
            x["q"].copy_(torch.randn(x["q"].shape, generator=gen, device="cuda"))
            x["x"][4].copy_(torch.rand(x["x"][4].shape, generator=gen, device="cuda"))
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (_, got), f in zip(graphs, (run, other)):
            got = [x.clone() for x in got]
            for x, y in zip(got, f()):
                assert torch.equal(x, y)


@pytest.mark.parametrize("G", [1, 8])
def test_captured_between_other_work(G):
    """Calls whose graph nodes follow copies, fills and another stream's work."""
    from paper_2606_03770_gb300 import ops
    cache, q, table, lens, starts = setup([300, 90], [9, 4], 2, G, 64, 64, seed=18)
    layers = ops.CacheLayers([cache])
    parents, s = trees([9, 4]), batch_of([9, 4], 9001, BF, seed=18)
    here, there = torch.empty_like(q), torch.zeros_like(s[0])
    side = torch.cuda.Stream()

    def step():
        main = torch.cuda.current_stream()
        here.copy_(q)
        side.wait_stream(main)
        with torch.cuda.stream(side):
            there.copy_(s[0])
            there.mul_(1)
        out = ops.cache_attend_tree(cache, here, parents, table, lens, starts, max_new=9, max_len=300)
        main.wait_stream(side)
        kept, nodes, answer = ops.verify_drafts(there, *s[1:5], draft=s[5], max_new=9)
        there.zero_()
        return out, kept, nodes, answer, ops.cache_keep(layers, table, lens, starts, nodes.clone(), kept)

    before = {k: getattr(cache, k).clone() for k in ("k_codes", "k_scales", "v_codes", "v_scales")}
    restore = lambda: [getattr(cache, k).copy_(v) for k, v in before.items()]
    want = [x.clone() for x in step()]
    torch.cuda.synchronize()
    restore()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        restore()
        here.zero_(), there.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    s, run = step(2, 12, 300, 2, 8, 30000, 7)
    t, other = step(1, 30, 500, 4, 2, 9000, 8)
    want, want_other = run(), other()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        with torch.cuda.stream(a):
            got = run()
        with torch.cuda.stream(b):
            got_other = other()
        torch.cuda.synchronize()
        for x, y in zip(got + got_other, want + want_other):
            assert torch.equal(x, y)
