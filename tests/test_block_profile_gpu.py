"""The block that block_profile measures: against plain products and attention,
and prefill against decode."""
import pytest
import torch

import ops_reference as R

pytestmark = pytest.mark.gpu


def make(d=512, ffn=1376, kv=2, vocab=1000, D=64, dtype=torch.bfloat16, group=32):
    from paper_2606_03770_gb300.block_profile import Block
    return Block(d, ffn, kv, vocab, 256, head_dim=D, dtype=dtype, group=group)


def cache_for(block, requests, page=16, length=128):
    from paper_2606_03770_gb300 import ops
    pages = length // page
    table = torch.randperm(requests * pages, device="cuda").int().view(requests, pages)
    return ops.Cache.empty(requests * pages, page, block.kv_heads, block.D), table


def plain_norm(x, w):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w


def plain_forward(block, x, cache, batch, window):
    """The block in 64 bits on the cache's contents after the pass."""
    T, kv, D = x.shape[0], block.kv_heads, block.D
    x = x.double()
    qkv = (plain_norm(x, block.norms[0]) @ R.weight(block.w_qkv).T).view(T, -1, D)
    at = batch.positions.long()
    q = R.rotate(qkv[:, :block.heads].float(), block.cos[at], block.sin[at], False)
    a, _, _ = R.attend(cache, q, batch.table, batch.lens, batch.starts, D ** -0.5, window)
    x = x + a.reshape(T, -1) @ R.weight(block.w_out).T
    gu = plain_norm(x, block.norms[1]) @ R.weight(block.w_gate_up).T
    n = gu.shape[1] // 2
    return x + (torch.nn.functional.silu(gu[:, :n]) * gu[:, n:]) @ R.weight(block.w_down).T


@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("requests,new", [(1, 60), (3, 1), (2, 9)])
def test_block_against_plain(requests, new, window):
    from paper_2606_03770_gb300.block_profile import Batch
    block = make()
    cache, table = cache_for(block, requests)
    g = torch.Generator(device="cuda").manual_seed(1)
    before = 50
    first = torch.randn(requests * before, block.d, generator=g, device="cuda").bfloat16()
    block.forward(first, cache, Batch.of(table, 0, before, 16), window)
    x = torch.randn(requests * new, block.d, generator=g, device="cuda").bfloat16()
    batch = Batch.of(table, before, new, 16)
    y = block.forward(x, cache, batch, window)
    want = plain_forward(block, x, cache, batch, window)
    # eight roundings of the stream to bf16 (2^-9 each on average), and their way through the products
    assert float((y.double() - want).norm() / want.norm()) < 8 * 2.0 ** -9


def test_decode_continues_prefill():
    """The last token of a prompt, prefilled with it or decoded after it."""
    from paper_2606_03770_gb300.block_profile import Batch
    block = make(dtype=torch.float16)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(70, block.d, generator=g, device="cuda").half()
    cache, table = cache_for(block, 1)
    whole = block.forward(x, cache, Batch.of(table, 0, 70, 16))
    other, table2 = cache_for(block, 1)
    block.forward(x[:69], other, Batch.of(table2, 0, 69, 16))
    last = block.forward(x[69:], other, Batch.of(table2, 69, 1, 16))
    # the two go through other kernels: codes at a rounding's edge may differ by one (a 15th of a range)
    assert float((last - whole[69:]).float().norm() / whole[69:].float().norm()) < 0.02
    lp, ent, vals, ids = block.head(last, torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert vals.shape == (1, 5) and bool((vals.diff() <= 0).all()) and 0 < float(ent) < 7


def test_measure_and_plan(capsys):
    """A small model's profile, and the rates that reproduce it in the planner's cost."""
    from paper_2606_03770_gb300 import block_profile as P
    from paper_2606_03770_gb300 import workloads as W
    prob = W.make_config("c1_tiny")
    m = P.measure(dict(d=512, ffn=1024, kv_heads=2, vocab=1000), 64, 64, 2, repeats=2)
    assert len(m.block) == len(m.head) == 3 and all(t > 0 for t in m.block + m.head)
    prob.blk_flops, prob.blk_bytes = prob.blk_flops[:3], prob.blk_bytes[:3]
    rate, bw = P.as_device(prob, m)
    assert abs(float(prob.blk_flops[0]) / rate - m.block[0]) < 1e-9
    assert abs(float(prob.blk_bytes[2]) / bw - m.block[2]) < 1e-9


def test_plan_with_this_device(monkeypatch, capsys):
    """Measured and planned with from the command line: the fleet's first device has the measured
    rates and all memory that is free."""
    from paper_2606_03770_gb300 import block_profile as P
    from paper_2606_03770_gb300 import e2ga
    from paper_2606_03770_gb300 import workloads as W
    seen = []

    class Engine(e2ga.Engine):
        def __init__(self, prob, *args, **kw):
            torch.cuda.empty_cache()
            seen.append((prob, torch.cuda.mem_get_info()[0]))
            super().__init__(prob, *args, **kw)

    monkeypatch.setattr(e2ga, "Engine", Engine)
    P.main(["--config", "c2", "--plan", "--generations", "2"])
    out = capsys.readouterr().out
    prob, free = seen[0]
    assert f"{prob.rate[0] / 1e12:.1f} TFLOP/s, {prob.bw[0] / 1e9:.0f} GB/s" in out
    assert (prob.rate[1:] == W.make_config("c2").rate[1:]).all()
    assert free - int(prob.mem[0]) < 1 << 26
    assert "best plan after 2 generations" in out and "inf" not in out and "nan" not in out


def test_planned_bytes_are_the_blocks():
    from paper_2606_03770_gb300 import block_profile as P
    from paper_2606_03770_gb300 import ops
    from paper_2606_03770_gb300 import workloads as W
    prob, model = W.make_config("c2"), W.CONFIGS["c2"]["model"]
    block = P.Block(model["d"], model["ffn"], model["kv_heads"], 64, 8)
    held = sum(t.numel() * t.element_size() for w in (block.w_qkv, block.w_out, block.w_gate_up, block.w_down)
               for t in (w.codes, w.scales))
    cache = ops.Cache.empty(1, 16, block.kv_heads, block.D)
    token = sum(t.numel() * t.element_size() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)) // 16
    got = P.planned(prob, model)
    assert int(got.blk_bytes[0]) == held + prob.NP * token
    assert int(got.blk_bytes[5]) == held + 5 * (prob.NP + prob.ND) * token
