"""examples/decode.py as a user runs it, and the captured step of AQDecoderBlock, which its --graph replays."""
import gc
import importlib.util
import os
import re
import sys

import pytest
import torch

import aq_testutil as U
import workloads
from paper_2606_12876_gb300.block import AQDecoderBlock, rope_angles
from paper_2606_12876_gb300.kv import PagedKVCache
from paper_2606_12876_gb300.linear import AQLinear

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode.py")


@pytest.fixture(autouse=True)
def collected():
    """(Destroying a graph invalidates a capture that is under way.)"""
    gc.collect()
    yield
    gc.collect()


@pytest.mark.parametrize("args,length", [("--blocks 1 --context 70 --steps 5 --beams 3", 78),
                                         ("--blocks 2 --context 64 --steps 4 --beams 2 --cache e4m3 --graph", 71)])
def test_example(monkeypatch, capsys, args, length):
    """Three warm-up steps and the timed ones lengthen every beam; all outputs are finite."""
    U.require_gpu()
    spec = importlib.util.spec_from_file_location("decode_example", PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    monkeypatch.setattr(sys, "argv", [PATH] + args.split())
    example.main()
    out = capsys.readouterr().out
    beams = int(re.search(r"--beams (\d+)", args).group(1))
    assert "lengths now %s, finite: True" % ([length] * beams) in out, out


@pytest.mark.parametrize("n", [3, 20])
def test_captured_block_steps_equal_eager_ones(n):
    """Products by GEMV (3 sequences) and by GEMM (20), two blocks, a graph replayed 12 times: bit for bit
    what eager steps give, and the caches' contents with them."""
    U.require_gpu()
    hid, qh, kh, hd, ffn = 256, 4, 2, 64, 512
    shapes = {"q": (qh * hd, hid), "k": (kh * hd, hid), "v": (kh * hd, hid), "o": (hid, qh * hd),
              "gate": (ffn, hid), "up": (ffn, hid), "down": (hid, ffn)}
    lins = [{k: AQLinear.from_layer(workloads.make_layer(o, i, M=3, book_std=0.03, seed=10 * b + j))
             for j, (k, (o, i)) in enumerate(shapes.items())} for b in range(2)]
    w = torch.ones(hid, device="cuda", dtype=torch.float16)
    blocks = [AQDecoderBlock(p, w, w, qh, kh, layer=b) for b, p in enumerate(lins)]
    caches = [PagedKVCache(4 * n, 8, kh, hd, n, 4, layers=2, dtype="f16") for _ in range(2)]
    for c in caches:
        for t in (c.k, c.v):
            t.zero_()
    seqs = torch.arange(n, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    xs = torch.randn(14, n, hid, device="cuda", generator=g).half()
    x = xs[0].clone()

    def step(cache, x):
        cache.reserve(seqs)
        rope = rope_angles(cache.lens - 1, hd)
        residual = None
        for b in blocks:
            x, residual = b.step(x, residual, 2, cache, seqs, rope)
        return x + residual

    for c in caches:
        step(c, x)                                   # warm-up
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(caches[1], x)
    for i in range(1, 13):
        want = step(caches[0], xs[i])
        x.copy_(xs[i])
        graph.replay()
        assert torch.equal(out, want), i
    for c in caches:
        c.check()
    assert caches[0].lens.tolist() == caches[1].lens.tolist() == [13] * n
    assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v, caches[1].v)
