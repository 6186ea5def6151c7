"""Measure one decoder block on this GPU, and plan with it.

The paper's planner takes per-block latencies that are measured by loading a
reduced number of blocks on each device (Sec. 3.1); the workloads here derive
them from work and rates instead.  This module runs the block itself, with the
operators of ``ops``: 4-bit weights, a paged 4-bit cache, the head's output layer
(workloads with 16-bit weights are refused).  It times the prefill of one prompt (l_P)
and the decode of b requests (l_D(b)), and turns the prefill into a compute rate and the
largest batch into a memory bandwidth, for the block's own flops and bytes; the planner
takes those two.  The other batches' and the head's times are shown, not planned with.
The two norms are plain torch: some 28 us of every decode (146 us with one request of
the 32-device workload).

    python -m paper_2606_03770_gb300.block_profile --config c2          # the table
    python -m paper_2606_03770_gb300.block_profile --config c2 --plan   # and a search
"""
from __future__ import annotations

import argparse
import dataclasses

import numpy as np
import torch

from . import ops
from . import workloads as W

EPS = 1e-6


def norm(x, weight):
    """Root-mean-square norm over the last axis, in 32 bits."""
    y = x.float()
    y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS)
    return (y * weight).to(x.dtype)


def random_weight(rows, cols, generator, group=64):
    """Random 4-bit weights that keep the size of what they are applied to."""
    codes = torch.randint(0, 256, (rows, cols // 2), generator=generator, device="cuda", dtype=torch.uint8)
    scales = (torch.rand(rows, cols // group, generator=generator, device="cuda") + 0.5) * (0.2 / cols ** 0.5)
    return ops.QuantWeight(codes, scales.half())


@dataclasses.dataclass
class Batch:
    """The requests of one forward pass: where their new tokens stand and go."""

    table: torch.Tensor      # int32 [requests, pages]
    lens: torch.Tensor       # int32 [requests] tokens cached after the pass
    starts: torch.Tensor     # int32 [requests + 1] first new token of each
    positions: torch.Tensor  # int32 [tokens]
    slots: torch.Tensor      # int64 [tokens]
    max_new: int
    max_len: int

    @classmethod
    def of(cls, table, before, new, page):
        """`new` tokens (each request the same) after `before` cached ones."""
        B = table.shape[0]
        pos = torch.arange(before, before + new, device="cuda").repeat(B)
        req = torch.arange(B, device="cuda").repeat_interleave(new)
        slots = table.long()[req, pos // page] * page + pos % page
        i32 = dict(dtype=torch.int32, device="cuda")
        return cls(table, torch.full((B,), before + new, **i32), torch.arange(B + 1, **i32) * new, pos.int(), slots, new,
                   before + new)


class Block:
    """One decoder block (attention and gated MLP, a norm before each) and the
    head, with random weights."""

    def __init__(self, d, ffn, kv_heads, vocab, positions, head_dim=W.HEAD_DIM, dtype=torch.bfloat16, seed=0, group=64):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.d, self.D, self.dtype = d, head_dim, dtype
        self.heads = d // head_dim
        self.kv_heads = self.heads if kv_heads is None else kv_heads
        self.w_qkv = random_weight((self.heads + 2 * self.kv_heads) * head_dim, d, g, group)
        self.w_out = random_weight(d, self.heads * head_dim, g, group)
        self.w_gate_up = random_weight(2 * ffn, d, g, group)
        self.w_down = random_weight(d, ffn, g, group)
        self.w_head = random_weight(vocab, d, g, group)
        self.norms = [1 + 0.1 * torch.randn(d, generator=g, device="cuda") for _ in range(3)]
        inv = 10000.0 ** (-torch.arange(head_dim // 2, device="cuda", dtype=torch.float64) * 2 / head_dim)
        angle = torch.arange(positions, device="cuda", dtype=torch.float64)[:, None] * inv
        self.cos, self.sin = angle.cos().float(), angle.sin().float()

    def forward(self, x, cache, batch, window=0):
        """x [tokens, d] through the block; keys and values go to the cache."""
        T, kv = x.shape[0], self.kv_heads
        qkv = ops.quant_matmul(norm(x, self.norms[0]), self.w_qkv).view(T, -1, self.D)
        q, k, v = qkv[:, :self.heads], qkv[:, self.heads:self.heads + kv], qkv[:, self.heads + kv:]
        ops.cache_append(cache, k, v, batch.slots, batch.positions, self.cos, self.sin, q=q, q_out=q)
        a = ops.cache_attend(cache, q, batch.table, batch.lens, batch.starts, max_new=batch.max_new,
                             max_len=batch.max_len, window=window)
        x = ops.quant_matmul(a.view(T, -1), self.w_out, residual=x)
        h = ops.quant_matmul(norm(x, self.norms[1]), self.w_gate_up, gated=True)
        return ops.quant_matmul(h, self.w_down, residual=x)

    def head(self, x, tokens, top=5):
        """The output layer on the last tokens' rows: log probabilities of
        `tokens`, entropy, alternatives."""
        logits = ops.quant_matmul(norm(x, self.norms[2]), self.w_head)
        return ops.token_logprobs(logits, tokens, top=top)


def time_graph(f, repeats=20):
    """Seconds per call of f, captured and replayed on the device."""
    f()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(4):
            f()
    graph.replay()
    start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    torch.cuda.synchronize()
    start.record()
    for _ in range(repeats):
        graph.replay()
    stop.record()
    torch.cuda.synchronize()
    return start.elapsed_time(stop) * 1e-3 / (4 * repeats)


@dataclasses.dataclass
class Measured:
    """Seconds of one block and of the head: index 0 the prefill of NP tokens,
    b the decode of b requests at a context of NP + ND tokens."""

    block: list
    head: list
    NP: int
    ND: int


def measure(model, NP, ND, b_max, page=64, window=0, repeats=20):
    """Run and time the block of `model` (a ``workloads.CONFIGS`` entry's, with 4-bit weights)."""
    if model.get("wbits", 4) != 4:
        raise ValueError(f"the block has 4-bit weights, the model {model['wbits']}-bit ones")
    block = Block(model["d"], model["ffn"], model["kv_heads"], model["vocab"], NP + ND + 1)
    pages = -(-(NP + ND) // page)
    cache = ops.Cache.empty(b_max * pages, page, block.kv_heads, block.D)
    table = torch.randperm(b_max * pages, device="cuda").int().view(b_max, pages)
    x = torch.randn(max(NP, b_max), block.d, device="cuda").to(block.dtype)
    tokens = torch.zeros(b_max, dtype=torch.int32, device="cuda")
    # every request's context, so that decode reads what prompts and tokens left
    for r in range(b_max):
        block.forward(torch.randn(NP + ND - 1, block.d, device="cuda").to(block.dtype), cache,
                      Batch.of(table[r:r + 1], 0, NP + ND - 1, page), window)
    out = Measured([], [], NP, ND)
    prompt = Batch.of(table[:1], 0, NP, page)
    out.block.append(time_graph(lambda: block.forward(x[:NP], cache, prompt, window), max(1, repeats // 4)))
    out.head.append(time_graph(lambda: block.head(x[:1], tokens[:1]), repeats))
    for b in range(1, b_max + 1):
        step = Batch.of(table[:b], NP + ND - 1, 1, page)
        out.block.append(time_graph(lambda: block.forward(x[:b], cache, step, window), repeats))
        out.head.append(time_graph(lambda: block.head(x[:b], tokens[:b]), repeats))
    return out


def planned(prob, model, window=0, group=64):
    """`prob` with the work of the block that `measure` runs in place of its own: 4-bit weights
    and a 4-bit cache, each with its scales, and at most `window` keys a token (0: all).  The
    workloads count 4-bit weights without scales and an fp16 cache."""
    d = model["d"]
    d_kv = d if model["kv_heads"] is None else model["kv_heads"] * W.HEAD_DIM
    params = 2 * d * d + 2 * d * d_kv + 3 * d * model["ffn"]
    weights = params // 2 + params // group * 2
    token = 2 * d_kv * (ops.E2_CACHE_GROUP // 2 + 4) // ops.E2_CACHE_GROUP       # keys and values
    flops, moved = [], []
    for v in range(prob.V):
        tokens, length, requests = (prob.NP, prob.NP, 1) if v == 0 else (v, prob.NP + prob.ND, v)
        seen = min(length, window) if window else length
        flops.append(2 * params * tokens + 4 * tokens * seen * d)
        moved.append(weights + requests * seen * token)
    u64 = lambda x: np.array(x, dtype=np.uint64)
    return dataclasses.replace(prob, blk_flops=u64(flops), blk_bytes=u64(moved), blk_mem=u64(moved))


def as_device(prob, measured):
    """(rate, bandwidth) of the device: the flops of a prefill over its measured
    time, the bytes of the largest decode batch over its.  ``planner_times`` has
    what the planner makes of them."""
    b = prob.b_max
    return float(prob.blk_flops[0]) / measured.block[0], float(prob.blk_bytes[b]) / measured.block[b]


def planner_times(prob, rate, bw):
    """The planner's stage time of one block, max(flops / rate, bytes / bandwidth), per
    variant.  With ``as_device``'s rates it is the measured one of the prefill and of the
    largest batch unless the other term is the larger there; the batches between
    follow from the bandwidth alone."""
    return [max(float(f) / rate, float(y) / bw) for f, y in zip(prob.blk_flops, prob.blk_bytes)]


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--config", default="c2", choices=[c for c, w in W.CONFIGS.items() if w["model"]["wbits"] == 4],
                    help="a workload with 4-bit weights")
    ap.add_argument("--window", type=int, default=0, help="sliding window of the block (0: full attention)")
    ap.add_argument("--plan", action="store_true", help="search with this GPU in the place of the fleet's first device")
    ap.add_argument("--generations", type=int, default=10)
    a = ap.parse_args(argv)
    prob = planned(W.make_config(a.config), W.CONFIGS[a.config]["model"], a.window)
    m = measure(W.CONFIGS[a.config]["model"], prob.NP, prob.ND, prob.b_max, window=a.window)
    rate, bw = as_device(prob, m)
    print(f"{a.config}: block of width {W.CONFIGS[a.config]['model']['d']}, prompt {prob.NP}, context {prob.NP + prob.ND}")
    times = planner_times(prob, rate, bw)
    print(f"{'':12s}{'block us':>10s}{'planner':>10s}{'head us':>10s}")
    for v, (t, s, h) in enumerate(zip(m.block, times, m.head)):
        print(f"{'prefill' if v == 0 else f'decode {v}':12s}{t * 1e6:10.1f}{s * 1e6:10.1f}{h * 1e6:10.1f}")
    for v in (0, prob.b_max):
        if times[v] > 1.01 * m.block[v]:
            print(f"no rate and bandwidth give both measured times: the planner takes {times[v] * 1e6:.1f} us for "
                  f"{'the prefill' if v == 0 else f'decode {v}'}")
    print(f"as a device of the planner: {rate / 1e12:.1f} TFLOP/s, {bw / 1e9:.0f} GB/s")
    if a.plan:
        from .e2ga import Engine
        prob.rate[0], prob.bw[0] = rate, bw
        torch.cuda.empty_cache()             # (the measured block's memory is free again)
        prob.mem[0] = torch.cuda.mem_get_info()[0]
        eng = Engine(prob)
        eng.init_population(seed=2026)
        for gen in range(1, a.generations + 1):
            eng.run_generation(2026, gen)
        _, fit = eng.elites()
        print(f"best plan after {a.generations} generations: waiting time {fit[0][0]:.3f} s, "
              f"prefill {fit[0][2]:.1f} tokens/s, decode {fit[0][3]:.1f} tokens/s")
        eng.close()


if __name__ == "__main__":
    main()
