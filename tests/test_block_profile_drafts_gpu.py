"""A decode step with drafted tokens through the block that block_profile measures."""
import dataclasses

import pytest
import torch

import drafts_reference as DR
import ops_reference as R
from test_block_profile_gpu import cache_for, make, plain_norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tree", ["1.1.1", "3.2", "2.2.2"])
@pytest.mark.parametrize("requests", [1, 3])
def test_a_tree_through_the_block(tree, requests):
    """Against plain products, and attention in which a node sees its own way."""
    from paper_2606_03770_gb300.block_profile import Batch, branching
    block, parents = make(), branching(tree)
    cache, table = cache_for(block, requests)
    g = torch.Generator(device="cuda").manual_seed(1)
    before, n = 50, len(parents)
    block.forward(torch.randn(requests * before, block.d, generator=g, device="cuda").bfloat16(), cache, Batch.of(table, 0, before, 16))
    x = torch.randn(requests * n, block.d, generator=g, device="cuda").bfloat16()
    batch = Batch.of_trees(table, before, parents, 16)
    y = block.forward(x, cache, batch)
    s = x.double()
    qkv = (plain_norm(s, block.norms[0]) @ R.weight(block.w_qkv).T).view(requests * n, -1, block.D)
    at = batch.positions.long()
    q = R.rotate(qkv[:, :block.heads].float(), block.cos[at], block.sin[at], False)
    a, _, _ = DR.attend_tree(cache, q, batch.parents, batch.table, batch.lens, batch.starts, block.D ** -0.5, 0)
    s = s + a.reshape(requests * n, -1) @ R.weight(block.w_out).T
    gu = plain_norm(s, block.norms[1]) @ R.weight(block.w_gate_up).T
    m = gu.shape[1] // 2
    want = s + (torch.nn.functional.silu(gu[:, :m]) * gu[:, m:]) @ R.weight(block.w_down).T
    # eight roundings of the stream to bf16 (2^-9 each on average), and their way through the products
    assert float((y.double() - want).norm() / want.norm()) < 8 * 2.0 ** -9


def test_steps_one_after_another():
    """Two steps with drafts against decoding the same tokens one by one: the kept tokens' keys and values are where, and
    what, decoding would have left."""
    from paper_2606_03770_gb300 import ops
    from paper_2606_03770_gb300.block_profile import Batch, branching
    block = make(dtype=torch.float16)
    g = torch.Generator(device="cuda").manual_seed(2)
    embed = torch.randn(1000, block.d, generator=g, device="cuda").half()
    cache, table = cache_for(block, 1)
    prompt = embed[torch.randint(0, 1000, (40,), generator=g, device="cuda")]
    block.forward(prompt, cache, Batch.of(table, 0, 40, 16))
    other = ops.Cache(*(x.clone() for x in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)))
    parents, layers, last, before, text = branching("3.2"), ops.CacheLayers([cache]), 7, 40, []
    for _ in range(2):
        ids = torch.randint(0, 1000, (len(parents),), generator=g, device="cuda", dtype=torch.int32)
        ids[0] = last
        batch = Batch.of_trees(table, before, parents, 16)
        y = block.forward(embed[ids.long()], cache, batch)
        # (greedy: what the target answers is drafted as the last child's, so that ways move)
        heat = torch.zeros(1, device="cuda")
        _, _, answer = ops.verify_drafts(ops.quant_matmul(plain_half(block, y), block.w_head), ids, batch.parents, batch.starts,
                                         torch.zeros(len(ids), device="cuda"), temperature=heat)
        ids[3] = answer[0, 0]
        y = block.forward(embed[ids.long()], cache, batch)
        kept, nodes, answer, lens = block.accept(y, ids, batch, torch.zeros(len(ids), device="cuda"), None, layers, temperature=heat)
        n = int(kept[0])
        assert nodes[0, :2].tolist() == [0, 3] and n >= 2 and lens.tolist() == [before + n]
        text += ids[nodes[0, :n].long()].tolist()
        before, last = before + n, int(answer[0, n - 1])
    for i, token in enumerate(text):
        block.forward(embed[token][None], other, Batch.of(table, 40 + i, 1, 16))
    at = torch.arange(40, before, device="cuda")
    slots = table.long()[0, at // 16] * 16 + at % 16
    for a, b in zip(ops.cache_read(cache, slots, torch.float32), ops.cache_read(other, slots, torch.float32)):
        # other kernels on the way: codes at a rounding's edge may differ by one (a 15th of a range)
        assert float((a - b).norm() / b.norm()) < 0.02


def plain_half(block, y):
    from paper_2606_03770_gb300.block_profile import norm
    return norm(y, block.norms[2])


def test_measured_drafts(capsys, monkeypatch):
    from paper_2606_03770_gb300 import block_profile as P
    model = dict(N=2, d=512, ffn=1408, kv_heads=2, vocab=1000, wbits=4)
    m = P.measure_drafts(model, 40, 24, 2, P.branching("2.1"), page=16, repeats=2)
    assert len(m.block) == len(m.head) == 2 and all(t > 0 for t in m.block + m.head)
    real = P.measure_drafts
    monkeypatch.setattr(P, "measure_drafts", lambda model, NP, ND, b_max, parents, window=0: real(
        dict(model, d=512, ffn=1408, kv_heads=2, vocab=1000), 40, 24, 2, parents, repeats=2))
    monkeypatch.setattr(P, "measure", lambda model, NP, ND, b_max, window=0: P.Measured([1e-3] * 9, [1e-4] * 9, NP, ND))
    P.main(["--config", "c2", "--draft", "2.1"])
    out = capsys.readouterr().out
    assert "trees of 5 nodes" in out and out.count("decode 2") == 2


@pytest.mark.parametrize("tree", ["1.1.1", "3.2.1"])
def test_measured_steps_are_accepted(tree):
    """The head that is timed verifies ways, and moves them: nearly all of a tree's depth."""
    from paper_2606_03770_gb300 import block_profile as P
    model = dict(N=2, d=512, ffn=1408, kv_heads=2, vocab=1000, wbits=4)
    m = P.measure_drafts(model, 40, 24, 8, P.branching(tree), page=16, repeats=2)
    assert len(m.given) == 8 and all(1 <= g <= 4 for g in m.given)
    # (a node's first child is accepted but in the draft's distance from the target, some 1%; 36 requests)
    assert sum(g * (b + 1) for b, g in enumerate(m.given)) / 36 > 3.5


def test_batches_without_trees_are_as_they_were():
    from paper_2606_03770_gb300.block_profile import Batch
    table = torch.arange(4, device="cuda").int().view(1, 4)
    assert Batch.of(table, 5, 2, 16).parents is None
    assert [f.name for f in dataclasses.fields(Batch)][:7] == ["table", "lens", "starts", "positions", "slots", "max_new", "max_len"]
