"""Decode steps of a stack of decoder blocks stored as additive codebooks (random weights of the
Llama-3-8B block's shapes), over a paged key-value cache: a few sequences share a prompt, and every
step reserves a token for each, writes its keys and values and attends over the cache.

    python examples/decode.py [--blocks 2] [--prefix 2] [--beams 4] [--context 512] [--steps 16]
                              [--cache bf16|e4m3] [--graph]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import workloads  # noqa: E402
from paper_2606_12876_gb300.block import AQDecoderBlock, rope_angles  # noqa: E402
from paper_2606_12876_gb300.kv import PagedKVCache  # noqa: E402
from paper_2606_12876_gb300.linear import AQLinear  # noqa: E402

HEADS, KV_HEADS, HEAD_DIM, HIDDEN, PAGE = 32, 8, 128, 4096, 64


def build(blocks):
    names = {"q_proj": "q", "k_proj": "k", "v_proj": "v", "o_proj": "o", "gate_proj": "gate", "up_proj": "up",
             "down_proj": "down"}
    layers = {names[n]: AQLinear.from_layer(layer) for n, layer in workloads.config_layers("llama8b_block")}
    w = torch.ones(HIDDEN, dtype=torch.bfloat16, device="cuda")
    # (every block has the same random weights: one copy in memory)
    return [AQDecoderBlock(layers, w, w, HEADS, KV_HEADS, layer=i) for i in range(blocks)]


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--prefix", type=int, default=2, help="codebooks used, m")
    ap.add_argument("--beams", type=int, default=4)
    ap.add_argument("--context", type=int, default=512)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--cache", choices=("bf16", "e4m3"), default="bf16")
    ap.add_argument("--graph", action="store_true", help="capture a step in a CUDA graph and replay it")
    a = ap.parse_args()
    torch.manual_seed(0)
    blocks = build(a.blocks)
    per_seq = -(-(a.context + a.steps + 8) // PAGE)   # (8: warm-up)
    cache = PagedKVCache((a.beams + 1) * per_seq, PAGE, KV_HEADS, HEAD_DIM, a.beams + 1, per_seq, layers=a.blocks,
                         dtype=a.cache)
    ints = lambda v: torch.as_tensor(list(v), dtype=torch.int32, device="cuda")

    # a prompt (random keys and values) in sequence 0, which the beams share
    cache.reserve(ints([0]), ints([a.context]))
    for i in range(a.blocks):
        k, v = (torch.randn(a.context, KV_HEADS, HEAD_DIM, device="cuda").bfloat16() for _ in range(2))
        cache.write(k, v, ints([0] * a.context), ints(range(a.context)), layer=i)
    beams = ints(range(1, a.beams + 1))
    cache.fork(ints([0] * a.beams), beams)
    cache.free(ints([0]))

    x0 = torch.randn(a.beams, HIDDEN, device="cuda").bfloat16()

    def step(x):
        cache.reserve(beams)
        rope = rope_angles(cache.lens[1:] - 1, HEAD_DIM)
        residual = None
        for b in blocks:
            x, residual = b.step(x, residual, a.prefix, cache, beams, rope)
        return x + residual

    run = lambda: step(x0)
    for _ in range(3):                               # warm-up; allocates the workspaces
        out = run()
    if a.graph:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = run()
        run = graph.replay
    t0, t1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    torch.cuda.synchronize()
    t0.record()
    for _ in range(a.steps):
        run()
    t1.record()
    cache.check()
    print("%d blocks, %d beams, m = %d, cache %s: %.3f ms a step; lengths now %s, finite: %s" % (
        a.blocks, a.beams, a.prefix, a.cache, t0.elapsed_time(t1) / a.steps, cache.lens[1:].tolist(),
        bool(torch.isfinite(out).all())))


if __name__ == "__main__":
    main()
