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
    python -m paper_2606_03770_gb300.block_profile --config c2 --draft 2.1.1   # and steps with drafted tokens

``--draft`` also times a decode step with a tree of drafted tokens for each request, given by its
branching level by level (2.1.1: two children of a request's last token, one of each of these, one of
each of those): the block on all nodes, then the head, the verification and the move of the accepted
way's keys and values.  How many drafted tokens a model accepts is not known here.  The head's steps
are those of a draft that is nearly the target, whose ways are accepted to their ends as a rule (how many tokens
they gave is shown), and what a block's step has to give to be worth its time is shown.
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
    parents: torch.Tensor | None = None      # int32 [tokens] where the new tokens are trees

    @classmethod
    def of_trees(cls, table, before, parents, page):
        """The same tree of drafted tokens, by its nodes' parents (-1: none), for each request."""
        batch = cls.of(table, before, len(parents), page)
        depth = []
        for p in parents:
            depth.append(depth[p] + 1 if p >= 0 else 0)
        i32 = dict(dtype=torch.int32, device="cuda")
        batch.positions = (before + torch.tensor(depth, **i32)).repeat(table.shape[0])
        batch.parents = torch.tensor(list(parents), **i32).repeat(table.shape[0])
        return batch

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
        if batch.parents is None:
            a = ops.cache_attend(cache, q, batch.table, batch.lens, batch.starts, max_new=batch.max_new,
                                 max_len=batch.max_len, window=window)
        else:
            a = ops.cache_attend_tree(cache, q, batch.parents, batch.table, batch.lens, batch.starts,
                                      max_new=batch.max_new, max_len=batch.max_len, window=window)
        x = ops.quant_matmul(a.view(T, -1), self.w_out, residual=x)
        h = ops.quant_matmul(norm(x, self.norms[1]), self.w_gate_up, gated=True)
        return ops.quant_matmul(h, self.w_down, residual=x)

    def head(self, x, tokens, top=5):
        """The output layer on the last tokens' rows: log probabilities of
        `tokens`, entropy, alternatives."""
        logits = ops.quant_matmul(norm(x, self.norms[2]), self.w_head)
        return ops.token_logprobs(logits, tokens, top=top)

    def accept(self, x, ids, batch, uniforms, draft, layers, temperature=None):
        """The output layer on all nodes' rows of a batch of trees: which drafted tokens are accepted
        (``ops.verify_drafts``); their keys and values, in the caches of ``layers``, go to where they
        belong.  Returns (kept, nodes, answer, cached tokens of each request)."""
        logits = ops.quant_matmul(norm(x, self.norms[2]), self.w_head)
        kept, nodes, answer = ops.verify_drafts(logits, ids, batch.parents, batch.starts, uniforms, draft=draft,
                                                temperature=temperature, max_new=batch.max_new)
        return kept, nodes, answer, ops.cache_keep(layers, batch.table, batch.lens, batch.starts, nodes, kept)


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
    given: list = dataclasses.field(default_factory=list)     # tokens a request and step, of steps with drafts


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


def branching(text):
    """The parents of a tree's nodes, numbered level by level, from its branching ("2.1.1")."""
    parents, level = [-1], [0]
    for b in text.split("."):
        if not b.isdigit() or int(b) < 1:
            raise ValueError(f"{text!r}: a tree is positive numbers with dots between them")
        if len(parents) + len(level) * int(b) > ops.E2_MAX_DRAFT:
            raise ValueError(f"{text!r} has more than {ops.E2_MAX_DRAFT} nodes")
        below = range(len(parents), len(parents) + len(level) * int(b))
        parents += [p for p in level for _ in range(int(b))]
        level = below
    return parents


def measure_drafts(model, NP, ND, b_max, parents, page=64, window=0, repeats=20):
    """Run and time decode steps with a tree of drafted tokens for each request, at the context of
    `measure`'s: ``block`` and ``head`` (with verification and move) of b requests at index b - 1, and
    ``given``, the tokens that such a step gave a request.  Drafted tokens are drawn, each by itself, from a
    draft whose logits are the target's and a little noise."""
    n = len(parents)
    block = Block(model["d"], model["ffn"], model["kv_heads"], model["vocab"], NP + ND + n)
    pages = -(-(NP + ND - 1 + n) // page)
    cache = ops.Cache.empty(b_max * pages, page, block.kv_heads, block.D)
    layers = ops.CacheLayers([cache])
    table = torch.randperm(b_max * pages, device="cuda").int().view(b_max, pages)
    for r in range(b_max):
        block.forward(torch.randn(NP + ND - 1, block.d, device="cuda").to(block.dtype), cache,
                      Batch.of(table[r:r + 1], 0, NP + ND - 1, page), window)
    out = Measured([], [], NP, ND)
    for b in range(1, b_max + 1):
        step = Batch.of_trees(table[:b], NP + ND - 1, parents, page)
        x = torch.randn(b * n, block.d, device="cuda").to(block.dtype)
        logits = ops.quant_matmul(norm(x, block.norms[2]), block.w_head)
        draft = logits + 0.01 * logits.float().std().to(block.dtype) * torch.randn_like(logits)
        ids, uniforms = torch.empty(b * n, dtype=torch.int32, device="cuda"), torch.rand(b * n, device="cuda")
        for t in range(b * n):
            p = torch.softmax(draft[t // n * n + max(parents[t % n], 0)].float(), 0)
            ids[t] = torch.multinomial(p, 1)[0]
        out.block.append(time_graph(lambda: block.forward(x, cache, step, window), repeats))
        out.head.append(time_graph(lambda: block.accept(x, ids, step, uniforms, draft, layers), repeats))
        out.given.append(float(block.accept(x, ids, step, uniforms, draft, layers)[0].float().mean()))
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
    ap.add_argument("--draft", type=branching, metavar="TREE",
                    help="also a decode step with a tree of drafted tokens for each request, by its branching (2.1.1)")
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
    if a.draft:
        d = measure_drafts(W.CONFIGS[a.config]["model"], prob.NP, prob.ND, prob.b_max, a.draft, window=a.window)
        print(f"trees of {len(a.draft)} nodes: {'block us':>10s}{'head us':>10s}  (giving)  tokens a block's step has to give")
        for b, (t, h, g) in enumerate(zip(d.block, d.head, d.given), 1):
            print(f"{f'decode {b}':16s}{t * 1e6:10.1f}{h * 1e6:10.1f}{g:10.2f}{t / m.block[b]:10.2f}")
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
