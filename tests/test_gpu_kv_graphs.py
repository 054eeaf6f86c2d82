"""Captured calls of a PagedKVCache: what a graph records and where it may be replayed."""
import pytest
import torch

import aq_testutil as U
import kv_testutil as K
from paper_2606_12876_gb300 import AQ_ERR_INVALID_ARG, AQError
from paper_2606_12876_gb300.kv import PagedKVCache

pytestmark = pytest.mark.gpu


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
