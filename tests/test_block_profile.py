"""block_profile without a GPU: what it refuses, and what it gives the planner."""
import pytest

from paper_2606_03770_gb300 import block_profile as P
from paper_2606_03770_gb300 import workloads as W


def test_models_with_other_weights_are_refused(capsys):
    """The block's weights have 4 bits: no rates of it for a model whose weights have 16."""
    with pytest.raises(ValueError, match="4-bit"):
        P.measure(W.CONFIGS["c1_tiny"]["model"], 64, 64, 2)
    with pytest.raises(SystemExit):
        P.main(["--config", "c1_tiny"])
    assert "c1_tiny" in capsys.readouterr().err


@pytest.mark.parametrize("config", ["c2", "c4"])
def test_the_plan_counts_the_work_that_is_timed(config):
    """Bytes of the block's tensors and of the cache's tokens, as the operators lay them out."""
    prob, model = W.make_config(config), W.CONFIGS[config]["model"]
    got = P.planned(prob, model)
    d, ffn, kv = model["d"], model["ffn"], model["kv_heads"] * W.HEAD_DIM
    weights = sum(rows * (cols // 2 + cols // 64 * 2) for rows, cols in ((d + 2 * kv, d), (d, d), (2 * ffn, d), (d, ffn)))
    token = 2 * model["kv_heads"] * (W.HEAD_DIM // 2 + W.HEAD_DIM // 64 * 4)
    ctx = prob.NP + prob.ND
    assert int(got.blk_bytes[0]) == weights + prob.NP * token
    for b in range(1, prob.V):
        assert int(got.blk_bytes[b]) == int(got.blk_mem[b]) == weights + b * ctx * token
    assert (got.blk_flops == prob.blk_flops).all() and got.PF is None
    assert (prob.blk_bytes == W.make_config(config).blk_bytes).all()          # (a copy)
    # a window: what the workloads with two types of blocks count for the sliding one
    few = P.planned(prob, model, window=128)
    two = W.make_config(config, layered="alternate")
    assert [int(f) for f in few.blk_flops] == [int(f) for f in two.PF[:, 1]]
    assert int(few.blk_bytes[3]) == weights + 3 * 128 * token and int(few.blk_bytes[0]) == weights + 128 * token


def test_main_plans_with_the_work_that_is_timed(monkeypatch, capsys):
    """The printed bandwidth is bytes that the measured block moves over its time."""
    monkeypatch.setattr(P, "measure", lambda model, NP, ND, b_max, window=0: P.Measured([1e-3] * 9, [1e-4] * 9, NP, ND))
    for window in (0, 128):
        P.main(["--config", "c2", "--window", str(window)])
        prob = P.planned(W.make_config("c2"), W.CONFIGS["c2"]["model"], window)
        assert f"{float(prob.blk_bytes[8]) / 1e-3 / 1e9:.0f} GB/s" in capsys.readouterr().out


@pytest.mark.parametrize("prefill,decode,said", [(2e-3, 2e-4, []), (1e-4, 2e-4, ["the prefill"]), (2e-3, 2.5e-1, ["the prefill"]),
                                                 (9.0, 1e-6, ["decode 8"])])
def test_what_the_planner_makes_of_the_rates(prefill, decode, said, monkeypatch, capsys):
    """Measured times come back where their own term is the larger; where the other one is, it is said."""
    prob = P.planned(W.make_config("c2"), W.CONFIGS["c2"]["model"])
    block = [prefill] + [decode * b / 8 for b in range(1, 9)]
    monkeypatch.setattr(P, "measure", lambda model, NP, ND, b_max, window=0: P.Measured(block, [1e-4] * 9, NP, ND))
    rate, bw = P.as_device(prob, P.measure(None, prob.NP, prob.ND, 8))
    times = P.planner_times(prob, rate, bw)
    assert times[0] == pytest.approx(max(prefill, float(prob.blk_bytes[0]) / bw))
    assert times[8] == pytest.approx(max(decode, float(prob.blk_flops[8]) / rate))
    assert (times[0] == pytest.approx(prefill)) == ("the prefill" not in said)
    assert (times[8] == pytest.approx(decode)) == ("decode 8" not in said)
    P.main(["--config", "c2"])
    out = capsys.readouterr().out
    assert [w for w in ("the prefill", "decode 8") if f"us for {w}" in out] == said
