"""e2_token_logprobs against 64 bits: types, odd rows, ties, forbidden tokens,
rows without a distribution."""
import math

import pytest
import torch

import ops_reference as R

pytestmark = pytest.mark.gpu
HALF, BF, F32 = torch.float16, torch.bfloat16, torch.float32


def check(x, tokens, top):
    from paper_2606_03770_gb300 import ops
    lp, ent, vals, ids = ops.token_logprobs(x, tokens, top=top)
    wlp, went, wvals, wids, dl, de = R.logprobs(x, tokens, top)
    R.close(lp, wlp, dl, "logprob")
    R.close(ent, went, de, "entropy")
    R.close(vals, wvals, dl[:, None], "values")
    assert torch.equal(ids, wids)


def logits(rows, vocab, dtype, seed=0, std=3.0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = (std * torch.randn(rows, vocab + pad, generator=g, device="cuda")).to(dtype)[:, :vocab]
    return x, torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("dtype", [HALF, BF, F32])
@pytest.mark.parametrize("vocab", [1, 2, 31, 33, 255, 1000, 4097, 32000, 128256])
@pytest.mark.parametrize("rows", [1, 3, 9])
def test_sizes(dtype, vocab, rows):
    check(*logits(rows, vocab, dtype, vocab), top=5)


@pytest.mark.parametrize("top", [0, 1, 2, 20, 31, 32])
@pytest.mark.parametrize("rows", [2, 700])
def test_alternatives(top, rows):
    check(*logits(rows, 5003, F32, top, pad=5), top=top)
    check(*logits(rows, 5003, BF, top, pad=2), top=top)     # many equal values


def test_many_rows_of_a_large_vocabulary():
    check(*logits(300, 128256, BF, 1), top=20)
    check(*logits(200, 50001, HALF, 1, pad=1), top=8)


@pytest.mark.parametrize("dtype", [HALF, BF, F32])
def test_ties_go_to_the_lowest_index(dtype):
    x = torch.zeros(3, 4000, device="cuda", dtype=dtype)
    x[1, ::7] = 1
    x[2] = torch.arange(4000, device="cuda").flip(0) // 500
    tokens = torch.tensor([0, 7, 3999], device="cuda", dtype=torch.int32)
    check(x, tokens, 32)
    x = (-torch.arange(4000, device="cuda", dtype=F32) // 100).flip(0)[None].to(dtype)     # rising
    check(x, tokens[:1], 32)


@pytest.mark.parametrize("dtype", [HALF, BF, F32])
@pytest.mark.parametrize("vocab", [40, 3001, 100000])
def test_forbidden_tokens(dtype, vocab):
    x, tokens = logits(6, vocab, dtype, 2)
    g = torch.Generator(device="cuda").manual_seed(1)
    for r, share in enumerate((0.1, 0.9, 0.999)):
        x[r, torch.rand(vocab, generator=g, device="cuda") < share] = -math.inf
    x[3] = -math.inf                                   # nothing left
    x[4] = -math.inf
    x[4, vocab // 2] = -70.0 if dtype != F32 else -1e30     # one left
    x[5] = torch.finfo(dtype).min                        # all at the lowest value: a uniform distribution
    check(x, tokens, 10)


@pytest.mark.parametrize("dtype", [HALF, BF, F32])
@pytest.mark.parametrize("vocab", [50, 20000])
def test_rows_without_a_distribution(dtype, vocab):
    x, tokens = logits(6, vocab, dtype, 3)
    x[0, 7] = math.nan
    x[1, vocab - 1] = math.inf
    x[2] = math.nan
    x[3, 5], x[3, 6] = math.inf, -math.inf
    x[4, :] = -math.inf
    x[4, 1] = math.nan
    check(x, tokens, 4)


def test_large_and_small_logits():
    for std in (1e-3, 30.0, 1e4, 1e30):
        check(*logits(4, 9000, F32, 5, std), top=8)
    check(*logits(4, 9000, BF, 5, 1e30), top=8)


def test_token_ids_outside_the_vocabulary():
    x, tokens = logits(5, 777, BF)
    tokens[0], tokens[1], tokens[2], tokens[3] = -1, 777, 2 ** 31 - 1, -2 ** 31
    check(x, tokens, 3)


def test_parts_left_out_strides_streams():
    from paper_2606_03770_gb300 import ops
    x, tokens = logits(4, 3000, F32)
    full = ops.token_logprobs(x, tokens, top=3)
    a, b, v, i = ops.token_logprobs(x, None, top=3, entropy=False)
    assert a is None and b is None and torch.equal(v, full[2]) and torch.equal(i, full[3])
    y = torch.empty(4, 9001, device="cuda")[:, 5:3005]       # rows at odd addresses
    y.copy_(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        z = ops.token_logprobs(y, tokens, top=3)
    s.synchronize()
    assert torch.equal(full[3], z[3]) and torch.allclose(full[0], z[0], rtol=0, atol=1e-5)


def test_rows_beyond_31_bits():
    from paper_2606_03770_gb300 import ops
    big = torch.zeros(3, 1 << 30, device="cuda", dtype=BF)
    x = big[:, :1003]                                       # rows 2 GB apart
    y, tokens = logits(3, 1003, BF)
    x.copy_(y)
    check(x, tokens, 5)


def test_empty_and_refusals():
    from paper_2606_03770_gb300 import e2ga, ops
    x, tokens = logits(2, 100, F32)
    lp, ent, vals, ids = ops.token_logprobs(x[:0], tokens[:0], top=2)
    assert lp.shape == (0,) and vals.shape == (0, 2)
    for bad in ((x.double(), tokens), (x, tokens.long()), (x, tokens[:1]), (x[0], tokens), (x.cpu(), tokens),
                (x.T, tokens)):
        with pytest.raises(ValueError):
            ops.token_logprobs(*bad)
    with pytest.raises(ValueError, match="top"):
        ops.token_logprobs(x, tokens, top=33)
    with pytest.raises(e2ga.E2Error, match="vocab"):
        ops.token_logprobs(x[:, :0], tokens)
    with pytest.raises(e2ga.E2Error, match="stride"):
        ops.token_logprobs(x[:1].expand(2, 100), tokens)


def test_gradients_are_refused():
    from paper_2606_03770_gb300 import ops
    x, tokens = logits(4, 300, F32)
    lp = ops.token_logprobs(x, tokens)[0]
    grad = x.clone().requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        ops.token_logprobs(grad, tokens)
    with torch.no_grad():
        assert torch.equal(lp, ops.token_logprobs(grad, tokens)[0])


@pytest.mark.parametrize("at", [64.0, -64.0, 256.0, 65536.0, -65536.0])
def test_logits_on_both_sides_of_a_power_of_two(at):
    """Where a row's maxima, in different lanes, are on both sides of what sums are kept apart by."""
    x = torch.full((5, 3000), -math.inf, device="cuda")
    x[0, 5], x[0, 700] = at - 0.5, at + 0.25
    x[1, 5], x[1, 6], x[1, 2900] = at - 0.25, at + 0.25, at
    x[2, ::3], x[2, 1::3] = at - 0.125, at + 0.5
    x[3, 0], x[3, 2999] = at + 0.5, at - 0.125
    x[4] = at + torch.randn(3000, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    check(x, torch.tensor([5, 6, 0, 0, 17], device="cuda", dtype=torch.int32), 4)


@pytest.mark.parametrize("vocab", [2 ** 31 - 1, 2 ** 31 - 8])
def test_a_vocabulary_at_the_end_of_its_type(vocab):
    """A row of 4.3 GB: its first and last elements, and what lies behind it, which is not its own."""
    from paper_2606_03770_gb300 import ops
    row = torch.full((1, 2 ** 31 + 64), -math.inf, device="cuda", dtype=BF)
    row[:, vocab:] = 5.0
    for at, value in ((0, 1.0), (3, 2.0), (vocab - 1, 3.0), (vocab - 2, 2.0), (vocab - 9, 0.5)):
        row[0, at] = value
    lp, ent, vals, ids = ops.token_logprobs(row[:, :vocab], torch.tensor([vocab - 1], device="cuda", dtype=torch.int32), top=6)
    z = torch.tensor([3.0, 2.0, 2.0, 1.0, 0.5], dtype=torch.float64)
    want = z - torch.logsumexp(z, 0)
    assert ids[0].tolist() == [vocab - 1, 3, vocab - 2, 0, vocab - 9, -1]
    # a handful of terms, each rounded a few times
    assert torch.allclose(vals[0, :5].double().cpu(), want, rtol=0, atol=64 * R.EPS32) and float(vals[0, 5]) == -math.inf
    assert abs(float(lp) - float(want[0])) < 64 * R.EPS32
    assert abs(float(ent) + float((want.exp() * want).sum())) < 64 * R.EPS32


def test_sizes_beyond_32_bits_are_refused():
    """They would lose their high bits: 2^32 + 5 logits taken for 5."""
    from paper_2606_03770_gb300 import ops
    x = torch.zeros(2 ** 32 + 5, device="cuda", dtype=HALF)
    for shape in ((1, -1), (-1, 1)):
        with pytest.raises(ValueError, match="2\\^31"):
            ops.token_logprobs(x.view(shape))
    with pytest.raises(ValueError, match="2\\^31"):
        ops.QuantWeight(torch.zeros(1, 1, device="cuda", dtype=torch.uint8).expand(2 ** 32 + 1, 1), x[:1].expand(2 ** 32 + 1, 1))
