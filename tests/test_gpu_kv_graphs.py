"""Captured calls of a PagedKVCache: what a graph records and where it may be replayed."""
import gc

import pytest
import torch

import aq_testutil as U
import kv_testutil as K
from paper_2606_12876_gb300 import AQ_ERR_INVALID_ARG, AQError
from paper_2606_12876_gb300.kv import PagedKVCache

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def collected():
    """Destroying a graph invalidates a capture that is under way: none of an earlier test's is left for the
    collector to find then."""
    gc.collect()
    yield
    gc.collect()


def query(n, heads, dim, dtype, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(n, heads, dim, device="cuda", generator=g).to(dtype)


def test_check_waits_for_replays_on_any_stream():
    """A graph captured on one stream is replayed on another, behind work of its own: check() reports what
    the replay records."""
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [50, 20], 16, 2, 64, "f16", seed=1)
    q, out = query(2, 4, 64, torch.float16), torch.empty(2, 4, 64, dtype=torch.float16, device="cuda")
    seqs = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    side, other, graph = torch.cuda.Stream(), torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        cache.attend(q, seqs, out=out)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        cache.attend(q, seqs, out=out)
    seqs.fill_(2)                                   # no such sequence: recorded by the replay
    torch.cuda.synchronize()
    with torch.cuda.stream(other):
        torch.cuda._sleep(500_000_000)              # about a quarter of a second
        graph.replay()
    with pytest.raises(AQError) as e:
        cache.check()
    assert e.value.status == AQ_ERR_INVALID_ARG
    cache.check()                                   # cleared


def record_workspaces(monkeypatch, name, at):
    """The addresses that the binding hands to a call as its workspace (argument `at`)."""
    from paper_2606_12876_gb300 import kv
    call, seen = getattr(kv, name), []

    def spy(*args):
        seen.append(args[at])
        return call(*args)
    monkeypatch.setattr(kv, name, spy)
    return seen


def test_a_capture_has_workspaces_of_its_own(monkeypatch):
    """Two captures on one stream, a third on torch's own, and eager calls there share no workspace; the calls
    of one capture on one stream do, and so do eager calls of one stream."""
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [50, 20], 16, 2, 64, "f16", seed=2)
    q, out = query(2, 4, 64, torch.float16), torch.empty(2, 4, 64, dtype=torch.float16, device="cuda")
    seen = record_workspaces(monkeypatch, "aq_kv_attend", 12)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        cache.attend(q, out=out)
        cache.attend(q, out=out)
    torch.cuda.synchronize()
    graphs = []
    for stream in (side, side, None):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            cache.attend(q, out=out)
            cache.attend(q, out=out)
    with torch.cuda.stream(side):
        cache.attend(q, out=out)
    torch.cuda.synchronize()
    assert all(seen)
    assert seen[0] == seen[1] == seen[8]
    assert all(seen[2 * i] == seen[2 * i + 1] for i in range(4))
    assert len(set(seen)) == 4


def test_branches_of_a_capture_have_workspaces_of_their_own(monkeypatch):
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [50, 20], 16, 2, 64, "f16", seed=3)
    q = query(2, 4, 64, torch.float16)
    outs = [torch.empty_like(q) for _ in range(2)]
    want = cache.attend(q)
    seen = record_workspaces(monkeypatch, "aq_kv_attend", 12)
    branch, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        branch.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(branch):
            cache.attend(q, out=outs[0])
        cache.attend(q, out=outs[1])
        torch.cuda.current_stream().wait_stream(branch)
    assert len(set(seen)) == 2
    for _ in range(20):
        for t in outs:
            t.zero_()
        graph.replay()
        assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
    cache.check()


def test_capture_on_a_stream_that_no_call_has_used():
    """torch.cuda.graph without a stream captures on one of its own: a warm-up on another is enough."""
    U.require_gpu()
    page, heads, dim, n = 8, 2, 64, 3
    caches = [PagedKVCache(32, page, heads, dim, n, 10, dtype="bf16") for _ in range(2)]
    seqs = torch.arange(n, dtype=torch.int32, device="cuda")
    rows = query(20 * n, 3 * heads, dim, torch.bfloat16).view(20, n, 3 * heads, dim)
    x = rows[0].clone()

    def step(cache, t):
        cache.reserve(seqs)
        cache.write(t[:, :heads], t[:, heads:2 * heads], seqs)
        return cache.attend(t[:, 2 * heads:])

    step(caches[1], x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(caches[1], x)
    for i in range(20):
        want = step(caches[0], rows[i])
        if i > 0:
            x.copy_(rows[i])
            graph.replay()
            assert torch.equal(out, want), i
    for c in caches:
        c.check()
    assert torch.equal(caches[0].tables, caches[1].tables) and caches[0].lens.tolist() == [20] * n


def test_a_condition_of_a_replay_is_reported_though_later_replays_are_well():
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [50, 20], 16, 2, 64, "f16", seed=4)
    q, out = query(2, 4, 64, torch.float16), torch.empty(2, 4, 64, dtype=torch.float16, device="cuda")
    seqs = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    cache.attend(q, seqs, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.attend(q, seqs, out=out)
    cache.check()
    for s in (1, -1, 1, 0):
        seqs.fill_(s)
        graph.replay()
    with pytest.raises(AQError):
        cache.check()
    cache.check()


def test_graphs_replayed_at_once():
    """Graphs captured on one stream (long sequences of one kv head, whose pieces cross all CTAs, so that
    every call counts arrivals), replayed on streams of their own beside each other and beside eager calls
    on the capture stream: each gives its own result every time."""
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [9000, 20000, 31, 70000], 64, 1, 128, "bf16", seed=5)
    side = torch.cuda.Stream()
    lists = [torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 1], [3], [2, 1, 0, 3], [1])]
    qs = [query(len(v), 8, 128, torch.bfloat16, seed=i) for i, v in enumerate(lists)]
    want = [cache.attend(q, v) for q, v in zip(qs, lists)]
    outs = [[torch.empty_like(q) for _ in range(16)] for q in qs]
    torch.cuda.synchronize()
    graphs = []
    with torch.cuda.stream(side):
        cache.attend(qs[0], lists[0])
    for q, v, o in zip(qs[:3], lists, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            for t in o:
                cache.attend(q, v, out=t)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(10):
        for o in outs:
            for t in o:
                t.zero_()
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        with torch.cuda.stream(side):
            for t in outs[3]:
                cache.attend(qs[3], lists[3], out=t)
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(t, w) for t in o)
    cache.check()


def test_a_cache_may_go_while_another_captures():
    """The garbage collector may drop a cache with captured calls at any time, in the middle of a capture
    too: releasing its workspaces must not disturb that."""
    U.require_gpu()
    q = query(1, 4, 64, torch.float16)

    def used():
        cache = PagedKVCache(4, 16, 1, 64, 1, dtype="f16")
        cache.attend(q)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            cache.attend(q)
        return cache, graph

    old, old_graph = used()
    old_graph.replay()
    torch.cuda.synchronize()
    del old_graph
    cache, x, graph = used()[0], torch.zeros(4, device="cuda"), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x.add_(1)
        del old
        out = cache.attend(q)
    graph.replay()
    assert x.tolist() == [1] * 4 and not bool(out.any())


def test_workspaces_go_with_their_cache():
    """Device memory of a capture's workspaces is released with the cache."""
    U.require_gpu()
    q = query(1, 16, 256, torch.float16)

    def use():
        cache = PagedKVCache(4, 16, 1, 256, 1, dtype="f16")
        cache.attend(q)
        torch.cuda.synchronize()
        for _ in range(8):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                cache.attend(q)
            graph.replay()
        cache.check()

    use()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    free = torch.cuda.mem_get_info()[0]
    for _ in range(5):
        use()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    # (eight of them hold about 40 MB; the driver keeps memory in pieces of a few MB)
    assert torch.cuda.mem_get_info()[0] >= free - (20 << 20)
