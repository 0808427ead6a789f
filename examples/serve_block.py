"""Serving pruned Transformer blocks: prompts and decoding steps of several requests, each with its own adapter.

A block is the LLaMA-2 / Qwen2.5 one whose projections the pruning replaces:

    h, y   = norm(x + residual)                       add_rms_norm
    q, k, v = projections of y (+ adapters)           linear_batched_into, adapters_batched_into
    q       = rotary(q); k, v into the pages          cache_append
    a       = attention over the pages                paged_attention
    x       = output projection of a (+ adapters)     linear_into, adapters_into
    h, y   = norm(x + h);  x = down(silu(gate(y)) up(y))

Every step (a prompt's chunk, a token, any mix) is the same call.  Decoding steps are captured into a CUDA graph once and
replayed with new lengths.  Weights and inputs are random (`python examples/serve_block.py`, one GPU).
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

import torch

ROOT = Path(__file__).resolve().parent.parent
if str(ROOT) not in sys.path:
    sys.path.insert(0, str(ROOT))

from paper_2609_33977_gb300 import groupsparse as gs  # noqa: E402

NAMES = ("q", "k", "v", "o", "gate", "up", "down")


def random_block(hidden, inter, heads, kv_heads, density, n_adapters, rank, seed):
    """Dense weights, group masks (1 x 256), norm weights and adapters of one block."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    d = hidden // heads
    shapes = {"q": (hidden, hidden), "k": (kv_heads * d, hidden), "v": (kv_heads * d, hidden), "o": (hidden, hidden),
              "gate": (inter, hidden), "up": (inter, hidden), "down": (hidden, inter)}

    def randn(*shape, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(torch.bfloat16)
    W = {n: randn(*s, scale=(s[1] * density) ** -0.5) for n, s in shapes.items()}
    M = {n: (torch.rand((s[0], s[1] // 256), generator=g, device="cuda") < density).to(torch.uint8) for n, s in shapes.items()}
    A = {n: randn(n_adapters, rank, s[1], scale=s[1] ** -0.5) for n, s in shapes.items()}
    B = {n: randn(n_adapters, s[0], rank, scale=0.3 * rank ** -0.5) for n, s in shapes.items()}
    norms = [1.0 + randn(hidden, scale=0.1) for _ in range(2)]
    return {"W": W, "M": M, "A": A, "B": B, "norms": norms, "scale": torch.full((n_adapters,), 2.0, device="cuda")}


class Block:
    """One block's packed projections, adapters and cache."""

    def __init__(self, weights, heads, kv_heads, pages, page_size):
        self.heads, self.kv_heads = heads, kv_heads
        self.p = {n: gs.pack(weights["W"][n], weights["M"][n]) for n in NAMES}
        self.ad = {n: gs.Adapters(weights["A"][n], weights["B"][n], weights["scale"]) for n in NAMES}
        self.norms = weights["norms"]
        self.d = self.p["q"].out // heads
        k = torch.zeros((pages, kv_heads, page_size, self.d), dtype=torch.bfloat16, device="cuda")
        self.cache = gs.PagedCache(k, torch.zeros_like(k))

    def _project(self, x, names, step):
        ys = [torch.empty((x.shape[0], self.p[n].out), dtype=torch.bfloat16, device="cuda") for n in names]
        xs = [x] * len(names)
        gs.linear_batched_into(xs, [self.p[n] for n in names], ys)
        gs.adapters_batched_into(xs, ys, [self.ad[n] for n in names], step.batch.offsets, step.ids, ys)
        return ys

    def __call__(self, x, h, step):
        """x: what the block before added to the residual stream h (None: the first block); returns the same pair."""
        y, h2 = gs.add_rms_norm(x, self.norms[0], h)
        h = x if h2 is None else h2
        q, k, v = self._project(y, ("q", "k", "v"), step)
        split = lambda t, n: t.view(-1, n, self.d)  # noqa: E731
        q = split(q, self.heads)
        gs.cache_append(self.cache, step.batch, q, split(k, self.kv_heads), split(v, self.kv_heads), step.cos, step.sin, q_out=q)
        a = gs.paged_attention(q, self.cache, step.batch)
        x, = self._project(a.flatten(1), ("o",), step)
        y, h = gs.add_rms_norm(x, self.norms[1], h)
        gate, up = self._project(y, ("gate", "up"), step)
        x, = self._project(torch.nn.functional.silu(gate) * up, ("down",), step)
        return x, h


class Step:
    """The tensors of one step's requests; the same ones may be refilled and a captured graph replayed."""

    def __init__(self, new, lens, ids, table, cos, sin):
        offsets = [0]
        for n in new:
            offsets.append(offsets[-1] + n)
        dev = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        self.lens, self.ids, self.cos, self.sin = dev(lens), dev(ids), cos, sin
        self.batch = gs.Batch(dev(offsets), self.lens, table, max(new))


def angles(n, d, base=10000.0):
    a = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * base ** (
        -torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
    return a.cos().float(), a.sin().float()


def run(blocks, prompts, decode_inputs, ids, table, max_len):
    """Prompts (a list of [n_i, hidden]) through the blocks, then a decoding step for each [requests, hidden] of
    decode_inputs: the residual stream after every step."""
    d = blocks[0].d
    cos, sin = angles(max_len, d)

    def through(x, step):
        h = None
        for b in blocks:
            x, h = b(x, h, step)
        return x + h
    lens = [p.shape[0] for p in prompts]
    outs = [through(torch.cat(prompts), Step(lens, lens, ids, table, cos, sin))]
    if not len(decode_inputs):
        return outs
    step = Step([1] * len(prompts), lens, ids, table, cos, sin)
    x = torch.zeros_like(decode_inputs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):       # once outside the graph: scratch of this stream is made here
        step.lens += 1
        through(x, step)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = through(x, step)
    for i, t in enumerate(decode_inputs):
        x.copy_(t)
        if i:
            step.lens += 1
        graph.replay()
        outs.append(out.clone())
    return outs


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--requests", type=int, default=16)
    ap.add_argument("--steps", type=int, default=50)
    a = ap.parse_args()
    hidden, inter, heads, page = 4096, 11008, 32, 64            # LLaMA-2-7B
    g = torch.Generator().manual_seed(0)
    lens = [int(v) for v in torch.randint(20, 1000, (a.requests,), generator=g)]
    ids = [i % 9 - 1 for i in range(a.requests)]                # eight adapters; -1: none
    per = -(-(max(lens) + a.steps + 1) // page)
    table = torch.randperm(per * a.requests, generator=g).to(torch.int32).view(a.requests, per).cuda()
    blocks = [Block(random_block(hidden, inter, heads, heads, 0.5, 8, 16, seed), heads, heads, per * a.requests, page)
              for seed in range(a.layers)]
    prompts = [torch.randn((n, hidden), device="cuda").to(torch.bfloat16) for n in lens]
    tokens = torch.randn((a.steps, a.requests, hidden), device="cuda").to(torch.bfloat16)
    run(blocks, prompts, tokens[:2], ids, table, per * page)    # kernels and scratch are loaded
    ev = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    ev[0].record()
    run(blocks, prompts, tokens[:0], ids, table, per * page)
    ev[1].record()
    outs = run(blocks, prompts, tokens, ids, table, per * page)
    ev[2].record()
    torch.cuda.synchronize()
    assert gs.device_status() == gs.GS_OK and all(o.isfinite().all() for o in outs)
    first, both = ev[0].elapsed_time(ev[1]), ev[1].elapsed_time(ev[2])
    print(f"{a.layers} pruned 7B blocks, {a.requests} requests, {sum(lens)} prompt tokens: prompts {first:.2f} ms, "
          f"{a.steps} decoding steps {max(0.0, both - first) / a.steps:.3f} ms each (capture included)")


if __name__ == "__main__":
    main()
