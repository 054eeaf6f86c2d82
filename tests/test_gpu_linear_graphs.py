"""Captured calls of AQLinear and gemv_group: their workspaces (partial sums, counters) belong to the capture,
as its graph may be replayed on any stream; and the captured step of AQDecoderBlock."""
import gc

import pytest
import torch

import aq_testutil as U
import workloads
from paper_2606_12876_gb300 import linear
from paper_2606_12876_gb300.linear import AQLinear, gemv_group

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def collected():
    """Destroying a graph invalidates a capture that is under way: none of an earlier test's is left for the
    collector to find then."""
    gc.collect()
    yield
    gc.collect()


def layers(shapes, M=3):
    return [AQLinear.from_layer(workloads.make_layer(o, i, M=M, book_std=0.05, seed=o + i)) for o, i in shapes]


def activations(n, inp, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(n, inp, device="cuda", generator=g).half()


def record(monkeypatch, name, at):
    """The addresses that the binding hands to a call as its workspace (positional argument `at`)."""
    call, seen = getattr(linear, name), []

    def spy(*args):
        seen.append(args[at].data_ptr())
        return call(*args)
    monkeypatch.setattr(linear, name, spy)
    return seen


def capture(stream, fn, times=2):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        for _ in range(times):
            fn()
    return graph


@pytest.mark.parametrize("what,n", [("aq_gemv", 1), ("aq_gemv", 7), ("aq_gemm", 40), ("aq_gemv_group", 1),
                                    ("aq_gemv_refine", 2)])
def test_a_capture_has_workspaces_of_its_own(monkeypatch, what, n):
    U.require_gpu()
    lins = layers([(512, 1024), (300, 1024)])
    x = activations(n, 1024, 1)
    y = torch.empty(n, 512, dtype=torch.float16, device="cuda")
    ys = [y, torch.empty(n, 300, dtype=torch.float16, device="cuda")]
    prev = torch.zeros(n, 512, dtype=torch.float16, device="cuda")
    call, at = {"aq_gemv": (lambda: lins[0].gemv(x, 2, y=y), 10), "aq_gemm": (lambda: lins[0].gemm(x, 2, y=y), 10),
                "aq_gemv_group": (lambda: gemv_group(lins, x, 2, ys=ys), 10),
                "aq_gemv_refine": (lambda: lins[0].refine(x, 2, prev, y=y), 11)}[what]
    seen = record(monkeypatch, what, at)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graphs = [capture(side, call) for _ in range(2)]
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    assert seen[0] == seen[5] and seen[1] == seen[2] and seen[3] == seen[4]
    assert len(set(seen)) == 3 and len(graphs) == 2


def test_equal_layers_share_a_workspace_within_a_capture(monkeypatch):
    """The blocks of a model have equal layers: a capture holds one workspace for each kind of them."""
    U.require_gpu()
    lins = layers([(512, 1024)]) + layers([(512, 1024)])
    x = activations(1, 1024, 2)
    want = [lin.gemv(x, 2) for lin in lins]
    ys = [torch.empty_like(w) for w in want]
    seen = record(monkeypatch, "aq_gemv", 10)
    torch.cuda.synchronize()
    graph = capture(None, lambda: [lin.gemv(x, 2, y=y) for lin, y in zip(lins, ys)])
    assert len(set(seen)) == 1
    graph.replay()
    assert all(torch.equal(y, w) for y, w in zip(ys, want))


def test_eager_calls_after_a_capture_without_a_warm_up():
    """A capture as a stream's first use leaves nothing behind that an eager call there would take: its
    workspace has to be zero, and nothing of the graph has run."""
    U.require_gpu()
    lins = layers([(512, 1024), (300, 1024)])
    x = activations(1, 1024, 3)
    want = [lin.gemv(x, 3) for lin in lins]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    junk = lambda: [torch.full((1 << 20,), -1, dtype=torch.int32, device="cuda") for _ in range(4)]

    def step():
        junk()                                   # freed blocks of the graph's pool, full of ones
        return gemv_group(lins, x, 3) + [lin.gemv(x, 3) for lin in lins]

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        outs = step()
    with torch.cuda.stream(side):
        eager = step()
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for y, w in zip(eager, want + want))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for y, w in zip(outs, want + want))


def test_graphs_replayed_at_once():
    """Graphs captured on one stream, replayed on streams of their own beside each other and beside eager
    calls on the capture stream."""
    U.require_gpu()
    lins = layers([(2048, 4096), (1024, 4096)], M=4)
    xs = [activations(n, 4096, n) for n in (1, 1, 6, 1)]
    want = [gemv_group(lins, x, 4) + [lins[0].gemv(x, 4)] for x in xs]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [[[torch.empty_like(w) for w in ws] for _ in range(8)] for ws in want]

    def step(x, o):
        gemv_group(lins, x, 4, ys=o[:2])
        lins[0].gemv(x, 4, y=o[2])

    with torch.cuda.stream(side):
        step(xs[0], outs[0][0])
    torch.cuda.synchronize()
    graphs = []
    for x, o in zip(xs[:3], outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            for t in o:
                step(x, t)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(10):
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        with torch.cuda.stream(side):
            for t in outs[3]:
                step(xs[3], t)
        torch.cuda.synchronize()
        for o, ws in zip(outs, want):
            for t in o:
                assert all(torch.equal(a, b) for a, b in zip(t, ws))
                for a in t:
                    a.zero_()
