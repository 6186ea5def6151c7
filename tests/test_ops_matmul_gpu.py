"""e2_quant_matmul against 64 bits: types, groups, odd sizes, strides, refusals."""
import math

import pytest
import torch

import ops_reference as R

pytestmark = pytest.mark.gpu
HALF, BF = torch.float16, torch.bfloat16


def make(rows, cols, group, mins, seed=0):
    from paper_2606_03770_gb300 import ops
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 256, (rows, cols // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = ((0.5 + torch.rand(rows, cols // group, generator=g, device="cuda")) * (0.2 / math.sqrt(cols))).half()
    m = (-(5 + 5 * torch.rand(s.shape, generator=g, device="cuda")) * s).half() if mins else None
    return ops.QuantWeight(codes, s, m), g


def randn(g, *shape, dtype=BF):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def check(tokens, rows, cols, group=64, dtype=BF, mins=False, gated=False, residual=False, spread=False):
    from paper_2606_03770_gb300 import ops
    w, g = make(rows, cols, group, mins, tokens + rows + cols)
    x = randn(g, tokens, cols, dtype=dtype)
    if spread:                 # rows of very different sizes, columns too
        x *= (10.0 ** torch.linspace(-4, 3, tokens, device="cuda"))[:, None].to(dtype)
        x[:, ::17] *= 30
    r = randn(g, tokens, rows // 2 if gated else rows, dtype=dtype) if residual else None
    y = ops.quant_matmul(x, w, residual=r, gated=gated)
    assert y.dtype == dtype
    R.close(y, *R.matmul(x, w, r, gated), "y")


@pytest.mark.parametrize("tokens", [1, 2, 7, 8, 9, 16, 17, 31, 33, 64, 65, 127, 130, 300])
@pytest.mark.parametrize("rows,cols,group", [(96, 512, 64), (257, 1376, 32), (33, 128, 128)])
def test_tokens(tokens, rows, cols, group):
    check(tokens, rows, cols, group, mins=tokens % 2 == 0)


@pytest.mark.parametrize("rows", [1, 15, 16, 17, 127, 128, 129, 1001])
@pytest.mark.parametrize("cols", [32, 64, 96, 992, 2080])
def test_rows_and_columns(rows, cols):
    check(3, rows, cols, 32, dtype=HALF, mins=True)
    check(140, rows, cols, 32, dtype=HALF)


@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("mins", [False, True])
@pytest.mark.parametrize("tokens", [1, 5, 40, 200])
def test_forms(dtype, group, mins, tokens):
    check(tokens, 320, 1280, group, dtype, mins, residual=True)
    check(tokens, 2 * 161, 1280, group, dtype, mins, gated=True)
    check(tokens, 2 * 161, 1280, group, dtype, mins, gated=True, residual=True)


@pytest.mark.parametrize("tokens", [1, 8, 24, 150])
def test_workload_widths(tokens):
    check(tokens, 4096, 11008)                       # the 4096-wide model's way back down
    check(tokens, 8192 + 2 * 1024, 8192, mins=True)   # queries, keys and values of the 8192-wide model


@pytest.mark.parametrize("tokens", [1, 6, 20, 129])
def test_rows_of_different_magnitude(tokens):
    check(tokens, 200, 2048, spread=True)
    check(tokens, 200, 2048, mins=True, spread=True)


@pytest.mark.parametrize("tokens", [3, 70])
def test_strides_outputs_and_in_place_residual(tokens):
    from paper_2606_03770_gb300 import ops
    w, g = make(100, 256, 64, False)
    wide = randn(g, tokens, 256 + 24)
    x = wide[:, 8:264]
    buf = torch.full((tokens, 111), 7.0, device="cuda", dtype=BF)
    r = randn(g, tokens, 100)
    buf[:, 5:105] = r
    ops.quant_matmul(x, w, residual=buf[:, 5:105], out=buf[:, 5:105])
    R.close(buf[:, 5:105], *R.matmul(x, w, r))
    assert bool((buf[:, :5] == 7).all()) and bool((buf[:, 105:] == 7).all())


@pytest.mark.parametrize("tokens", [2, 100])
def test_values_that_are_not_finite_stay_in_their_rows(tokens):
    from paper_2606_03770_gb300 import ops
    w, g = make(64, 256, 64, True)
    x = randn(g, tokens, 256)
    y0 = ops.quant_matmul(x, w)
    x[0, 3], x[1, 200] = math.nan, math.inf
    y = ops.quant_matmul(x, w)
    assert bool(torch.isnan(y[0]).all())
    assert not bool(torch.isfinite(y[1]).any())
    assert torch.equal(y[2:], y0[2:])


@pytest.mark.parametrize("tokens", [1, 8, 200])
def test_same_inputs_same_bits_also_on_another_stream(tokens):
    from paper_2606_03770_gb300 import ops
    w, g = make(512, 4096, 64, False)
    x = randn(g, tokens, 4096)
    y = ops.quant_matmul(x, w)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        z = [ops.quant_matmul(x, w) for _ in range(3)]
    s.synchronize()
    assert all(torch.equal(y, v) for v in z)


def test_captured_in_a_graph():
    from paper_2606_03770_gb300 import ops
    w, g = make(512, 1024, 64, False)
    for tokens in (4, 150):
        x = randn(g, tokens, 1024)
        out = torch.empty(tokens, 512, device="cuda", dtype=BF)
        ws = torch.empty(ops.load().e2_quant_matmul_workspace(512, 1024, tokens) + 1, device="cuda", dtype=torch.uint8)
        ops.quant_matmul(x, w, out=out, workspace=ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ops.quant_matmul(x, w, out=out, workspace=ws)
        x.copy_(randn(g, tokens, 1024))
        graph.replay()
        R.close(out, *R.matmul(x, w))


def test_quantize_weight_rounds_to_the_nearest_code():
    from paper_2606_03770_gb300 import ops
    g = torch.Generator(device="cuda").manual_seed(3)
    a = torch.randn(40, 256, generator=g, device="cuda")
    a[5] = 0
    for symmetric in (True, False):
        w = ops.quantize_weight(a, 64, symmetric)
        step = w.scales.double().repeat_interleave(64, 1)
        # half a step, and the roundings of scale and minimum to fp16
        lim = step / 2 + 2.0 ** -11 * (16 * step + a.abs().amax(1, keepdim=True)) + 1e-7
        assert bool(((R.weight(w) - a.double()).abs() <= lim).all())


def test_empty_and_refusals():
    from paper_2606_03770_gb300 import e2ga, ops
    w, g = make(64, 256, 64, False)
    assert ops.quant_matmul(torch.empty(0, 256, device="cuda", dtype=BF), w).shape == (0, 64)
    x = randn(g, 2, 256)
    for bad in (x.float(), x[:, :128], x.cpu()):
        with pytest.raises(ValueError):
            ops.quant_matmul(bad, w)
    with pytest.raises(ValueError):
        ops.quant_matmul(x, w, residual=randn(g, 2, 63))
    with pytest.raises(e2ga.E2Error, match="16-byte"):
        ops.quant_matmul(randn(g, 2, 264)[:, 1:257], w)
    with pytest.raises(e2ga.E2Error, match="16-byte"):
        ops.quant_matmul(randn(g, 2, 260)[:, :256], w)
    with pytest.raises(e2ga.E2Error, match="16-byte"):
        ops.quant_matmul(randn(g, 1, 256).expand(2, 256), w)
    odd, _ = make(33, 256, 64, False)
    with pytest.raises(e2ga.E2Error, match="even"):
        ops.quant_matmul(x, odd, gated=True)
    with pytest.raises(ValueError, match="one column per"):
        ops.QuantWeight(w.codes, torch.ones(64, 16, device="cuda", dtype=HALF))


@pytest.mark.parametrize("tokens,rows,cols,form", [(1150, 4001, 4096, {}), (250, 20000, 4096, dict(residual=True)),
                                                   (230, 2 * 10100, 4096, dict(gated=True, mins=True))])
def test_a_few_blocks_more_than_multiprocessors(tokens, rows, cols, form):
    check(tokens, rows, cols, **form)
    check(tokens, rows, cols, dtype=HALF, **form)


@pytest.mark.parametrize("tokens", [3, 16, 17, 40, 200])
@pytest.mark.parametrize("mins", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_weights_beyond_fp16(tokens, mins, group):
    """Scales and minima whose weights pass 65,504: as they are for a few tokens, no larger than
    that from 17 on."""
    from paper_2606_03770_gb300 import ops
    w, g = make(130, 512, group, mins)
    w.scales[::3] = 9000.0
    w.scales[1::5] = -12000.0
    if mins:
        w.mins[::2], w.mins[1::2] = 60000.0, -65504.0
    x = randn(g, tokens, 512)
    x[0, :7] = 0
    W, X = R.weight(w), x.double()
    if tokens >= 17:
        W = W.clamp(-65504.0, 65504.0)
    want = X @ W.T
    off = (2.0 ** -11 + 512 * R.EPS32) * (X.abs() @ W.abs().T)
    R.close(ops.quant_matmul(x, w), want, off + R.EPS[BF] * (want.abs() + off))


@pytest.mark.parametrize("tokens", [2, 30])
@pytest.mark.parametrize("value", [math.inf, math.nan])
def test_scales_that_are_not_finite_stay_in_their_rows(tokens, value):
    from paper_2606_03770_gb300 import ops
    for mins in (False, True):
        w, g = make(70, 256, 64, mins)
        x = randn(g, tokens, 256)
        y0 = ops.quant_matmul(x, w)
        (w.mins if mins else w.scales)[3, 1] = value
        y = ops.quant_matmul(x, w)
        assert not bool(torch.isfinite(y[:, 3]).any())
        rest = torch.arange(70, device="cuda") != 3
        assert torch.equal(y[:, rest], y0[:, rest])


@pytest.mark.parametrize("tokens", [1, 8, 16, 17, 200])
@pytest.mark.parametrize("mins", [False, True])
@pytest.mark.parametrize("dtype", [HALF, BF])
@pytest.mark.parametrize("rows,cols,gated", [(70, 512, False), (33, 8192, False), (66, 1088, True), (8000, 4096, False)])
def test_infinities_of_x_are_the_formulas(tokens, mins, dtype, rows, cols, gated):
    """Signed infinities, and NaN where signs meet or a weight is 0, whatever the tokens."""
    from paper_2606_03770_gb300 import ops
    w, g = make(rows, cols, 64, mins)
    if mins:
        w.mins[:, 0] = -4 * w.scales[:, 0]             # weights of 0
    x = randn(g, tokens, cols, dtype=dtype)
    x[0, 5] = math.inf
    if tokens > 4:
        x[1, cols - 1] = -math.inf
        x[2, 40], x[2, 41] = math.inf, -math.inf
        x[3, 9], x[3, 10] = math.inf, math.nan
        x[4, 9], x[4, cols // 2] = math.inf, math.inf
    r = randn(g, tokens, rows // 2 if gated else rows, dtype=dtype)
    want, lim = R.matmul(x, w, r, gated)
    assert bool((want[0] == math.inf).any()) and bool(torch.isnan(want[0]).any())
    assert gated or bool((want[0] == -math.inf).any())
    R.close(ops.quant_matmul(x, w, residual=r, gated=gated), want, lim)


def test_weights_keep_the_memory_they_point_at():
    """Nothing is assigned once they are made; other tensors behind the given ones do not matter."""
    from paper_2606_03770_gb300 import ops
    w, g = make(64, 256, 64, True)
    x = randn(g, 3, 256)
    y = ops.quant_matmul(x, w)
    for name in ("codes", "scales", "mins", "rows", "cols", "group", "device", "struct", "ref"):
        with pytest.raises(AttributeError, match="QuantWeight"):
            setattr(w, name, getattr(w, name, None))
    with pytest.raises(AttributeError, match="QuantWeight"):
        del w.codes
    w.name = "down"                                   # a program's own
    w.name = w.name + "_proj"
    del w.name
    given = [t.clone() for t in (w.codes, w.scales, w.mins)]
    v = ops.QuantWeight(*given)
    for t in given + [v.scales]:
        t.data = torch.zeros_like(t)
    del given
    filler = [torch.full((64, 128), 7, dtype=torch.uint8, device="cuda") for _ in range(64)]
    assert torch.equal(y, ops.quant_matmul(x, v)) and len(filler) == 64
    w.scales.mul_(2)                                  # written in place: counts
    w.mins.mul_(2)
    R.close(ops.quant_matmul(x, w), *R.matmul(x, w))


def test_gradients_are_refused():
    from paper_2606_03770_gb300 import ops
    w, g = make(64, 256, 64, False)
    x, r = randn(g, 2, 256), randn(g, 2, 64)
    y = ops.quant_matmul(x, w, residual=r)
    v = ops.QuantWeight(w.codes, w.scales.clone().requires_grad_())
    xg, rg = x.clone().requires_grad_(), r.clone().requires_grad_()
    for args, kw in (((xg, w), {}), ((x, w), dict(residual=rg)), ((x, w), dict(out=rg)), ((x, v), {})):
        with pytest.raises(ValueError, match="gradient"):
            ops.quant_matmul(*args, **kw)
    with torch.no_grad():
        assert torch.equal(y, ops.quant_matmul(xg, v, residual=rg))
    with torch.inference_mode():
        assert torch.equal(y, ops.quant_matmul(x.clone(), w, residual=r.clone()))


def test_rows_and_tokens_at_the_end_of_their_type_are_refused():
    import ctypes as C

    from paper_2606_03770_gb300 import e2ga, ops
    lib = ops.load()
    w, g = make(64, 64, 64, False)
    x, y = randn(g, 64, 64), torch.empty(64, 64, device="cuda", dtype=BF)
    for rows, tokens in ((2 ** 31 - 1, 1), (2 ** 31 - 1023, 40), (64, 2 ** 31 - 1), (0, 1), (64, -1)):
        s = ops.e2_quant_weight(rows, 64, 64, w.codes.data_ptr(), w.scales.data_ptr(), None)
        a = ops.e2_matmul_args(tokens, ops.E2_BF16, 0, x.data_ptr(), 64, None, 0, y.data_ptr(), 2 ** 31)
        assert lib.e2_quant_matmul_workspace(rows, 64, tokens) == 0
        assert lib.e2_quant_matmul(C.byref(s), C.byref(a), None, 0, None) == e2ga.E2_EINVAL
        assert b"rows" in lib.e2_ops_error() or b"tokens" in lib.e2_ops_error()


def test_workspaces_that_are_given():
    """Any type, as many bytes as are there: one byte repeated is one."""
    from paper_2606_03770_gb300 import e2ga, ops
    w, g = make(64, 256, 64, False)
    x = randn(g, 40, 256)
    y = ops.quant_matmul(x, w)
    need = ops.load().e2_quant_matmul_workspace(64, 256, 40)
    one = torch.zeros(1, dtype=torch.uint8, device="cuda")
    for view in (one.expand(need), torch.zeros(2 * need, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError, match="contiguous"):
            ops.quant_matmul(x, w, workspace=view)
    for short in (one, torch.zeros(need // 4 - 1, device="cuda")):
        with pytest.raises(e2ga.E2Error, match="workspace"):
            ops.quant_matmul(x, w, workspace=short)
    assert torch.equal(y, ops.quant_matmul(x, w, workspace=torch.zeros(-(-need // 4), device="cuda")))


@pytest.mark.parametrize("tokens", [1, 5, 40])
def test_outputs_over_x_are_refused(tokens):
    """Blocks that start later would read outputs; side by side in one buffer they do not meet."""
    from paper_2606_03770_gb300 import e2ga, ops
    w, g = make(128, 128, 64, False)
    buf = randn(g, 2 * tokens, 3 * 128 + 8)
    kept = buf.clone()
    x = buf[:tokens, 128:256]
    flat = buf.view(-1)
    for out in (x, buf[:tokens, 120:248], buf[:tokens, 255:383], flat[128:].as_strided((tokens, 128), (400, 1)),
                buf[tokens // 2:][:tokens, 128:256] if tokens > 1 else x):
        with pytest.raises(e2ga.E2Error, match="overlap"):
            ops.quant_matmul(x, w, out=out)
    assert torch.equal(buf, kept)
    want = R.matmul(x, w)
    for out in (buf[:tokens, :128], buf[:tokens, 256:384], buf[tokens:, 128:256]):
        R.close(ops.quant_matmul(x, w, out=out), *want)
        assert torch.equal(x, kept[:tokens, 128:256])
    v, _ = make(30, 128, 64, False)
    for at in (98, 256, 300, 380):                     # close beside x, and across a row's end
        out = flat[at:].as_strided((tokens, 30), (392, 1))
        R.close(ops.quant_matmul(x, v, out=out), *R.matmul(x, v))
        assert torch.equal(x, kept[:tokens, 128:256])


def test_quantize_weight_beyond_fp16():
    """Finite weights have finite codes' values: the nearest there are."""
    from paper_2606_03770_gb300 import ops
    g = torch.Generator(device="cuda").manual_seed(4)
    a = torch.randn(6, 256, generator=g, device="cuda")
    a[0, 3], a[1, 70], a[2, 5], a[3] = 1e6, -1e7, math.inf, 2e5
    a[4, :64] = torch.linspace(-9e4, 8e5, 64, device="cuda")
    for symmetric in (True, False):
        w = ops.quantize_weight(a, 64, symmetric)
        W, most = R.weight(w), 65504.0
        assert bool(torch.isfinite(W).all())
        top = 7 * most if symmetric else (w.mins.double() + 15 * most).repeat_interleave(64, 1)
        want = a.double().clamp(min=-8 * most if symmetric else -most)
        want = torch.minimum(want, torch.as_tensor(top, device="cuda", dtype=torch.float64))
        step = w.scales.double().repeat_interleave(64, 1)
        # half a step, and the roundings of scale and minimum to fp16
        lim = step / 2 + 2.0 ** -11 * (16 * step + want.abs().amax(1, keepdim=True)) + 1e-7
        assert bool(((W - want).abs() <= lim).all())


@pytest.mark.parametrize("tokens", [1, 8, 40])
def test_widths_of_the_largest_workload_and_its_head(tokens):
    check(tokens, 512, 53248)                        # the 16384-wide model's way back down
    check(tokens, 2 * 1000, 16384, gated=True, residual=True)
    check(tokens, 128256, 1024)                      # a head's rows


@pytest.mark.parametrize("tokens", [1, 16, 200])
def test_two_streams_at_once(tokens):
    """Each call with a workspace of its own, many of both in flight."""
    from paper_2606_03770_gb300 import ops
    pairs = []
    for seed in (1, 2):
        w, g = make(1024, 4096, 64, seed == 2, seed)
        x = randn(g, tokens, 4096)
        pairs.append((x, w, ops.quant_matmul(x, w)))
    streams = [torch.cuda.Stream() for _ in pairs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(ops.quant_matmul(*pairs[i][:2]))
    torch.cuda.synchronize()
    for (_, _, want), outs in zip(pairs, got):
        assert all(torch.equal(want, y) for y in outs)
