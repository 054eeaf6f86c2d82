"""Attention of one new token over the paged cache (aq_kv_attend) against fp64, within bounds
derived from its arithmetic (kv_testutil.attend_exact). Everything that is not cached (free pages,
slots past a sequence's length, tokens before the window's first chunk) holds NaN."""
import numpy as np
import pytest
import torch

import aq_testutil as U
import kv_testutil as K
from paper_2606_12876_gb300.kv import PagedKVCache

pytestmark = pytest.mark.gpu
DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def check(cache, q, seqs=None, layer=0, scale=None, window=0):
    n = q.shape[0]
    idx = None if seqs is None else torch.as_tensor(seqs, dtype=torch.int32, device="cuda")
    lse = torch.full(q.shape[:2], float("nan"), device="cuda")
    out = torch.full(q.shape, float("nan"), dtype=q.dtype, device="cuda")
    got = cache.attend(q, idx, layer=layer, scale=scale, window=window, out=out, lse=lse)
    assert got is out
    cache.check()
    sc = cache.head_dim ** -0.5 if scale is None else scale
    ref, rlse, tol, tol_lse = K.attend_exact(cache, q, range(n) if seqs is None else seqs, layer, sc, window)
    err = (out.double() - ref).abs()
    assert bool((err <= tol).all()), "largest error/bound %.3g" % float((err / tol.clamp(min=1e-300)).max())
    empty = torch.isinf(rlse)
    assert bool((lse[empty] == -np.inf).all())
    assert bool(((lse.double() - rlse).abs()[~empty] <= tol_lse[~empty]).all())
    again = cache.attend(q, idx, layer=layer, scale=scale, window=window)
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))     # bit for bit
    return out


def query(n, heads, dim, dtype, seed=0, gain=2.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 77)
    return (torch.randn(n, heads, dim, device="cuda", generator=g) * gain).to(dtype)


CASES = [  # lengths, q heads, kv heads, head dim, page, type, window
    ([1], 1, 1, 16, 8, "f16", 0),
    ([0], 4, 1, 64, 16, "bf16", 0),
    ([0, 0, 0], 4, 2, 128, 16, "f16", 3),
    ([15, 16, 17, 0, 31, 32, 33, 1], 8, 2, 128, 16, "bf16", 0),
    ([63, 64, 65, 7, 8, 9], 8, 8, 64, 8, "f16", 0),
    ([63, 64, 65, 7, 8, 9], 16, 2, 64, 64, "e4m3", 0),
    ([1000, 3, 257, 0, 129], 32, 8, 128, 32, "bf16", 0),
    ([1000, 3, 257, 0, 129], 32, 8, 128, 32, "e4m3", 0),
    ([700, 5, 0, 300], 8, 2, 256, 16, "bf16", 0),
    ([700, 5, 0, 300], 8, 1, 256, 64, "e4m3", 0),
    ([500, 1, 77], 6, 2, 192, 128, "f16", 0),
    ([500, 1, 77], 6, 2, 80, 8, "e4m3", 0),
    ([130, 2000], 71, 1, 64, 16, "bf16", 0),
    ([130, 2000], 40, 2, 96, 1024, "f16", 0),
    ([130, 900], 17, 1, 48, 32, "e4m3", 0),
    ([1000, 3, 257, 0, 129], 32, 8, 128, 16, "f16", 1),
    ([1000, 3, 257, 0, 129], 32, 8, 128, 8, "bf16", 100),
    ([1000, 3, 257, 0, 129, 96], 32, 8, 64, 8, "e4m3", 33),
    ([5000], 8, 1, 128, 64, "bf16", 0),
    ([5000], 8, 8, 128, 64, "f16", 4097),
    ([70000, 9], 4, 1, 64, 16, "f16", 0),
    ([40000], 16, 2, 128, 32, "e4m3", 0),
    # tiles of 9 to 16 query heads at the largest head dimensions
    ([300, 0, 77, 2000], 32, 2, 256, 32, "bf16", 0),
    ([300, 0, 77, 2000], 24, 2, 208, 16, "e4m3", 50),
    ([300, 1, 77, 9000], 12, 1, 128, 64, "e4m3", 0),
    ([9000], 16, 1, 256, 64, "f16", 0),
    # many short segments per warp, and equal ones of about a warp's share
    ([17] * 300, 8, 4, 64, 16, "bf16", 0),
    ([1000] * 130, 32, 8, 128, 16, "bf16", 0),
    ([1000] * 130, 8, 8, 128, 16, "e4m3", 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s-%dx%dx%d-p%d-%s-w%d" % (("_".join(map(str, c[0][:9])) + "n%d" % len(c[0]),) + c[1:]))
def test_attend(case):
    U.require_gpu()
    lens, qh, kh, hd, page, dt, window = case
    cache = K.filled_cache(PagedKVCache, lens, page, kh, hd, dt, seed=sum(lens) + qh)
    for qd in ([DT[dt]] if dt in DT else [torch.float16, torch.bfloat16]):
        check(cache, query(len(lens), qh, hd, qd), window=window)


def test_many_sequences_cross_the_launch_slices():
    U.require_gpu()
    rng = np.random.Generator(np.random.PCG64(3))
    lens = [int(v) for v in rng.integers(0, 60, 1100)]
    cache = K.filled_cache(PagedKVCache, lens, 16, 2, 64, "bf16", seed=4)
    check(cache, query(1100, 8, 64, torch.bfloat16))
    some = [int(v) for v in rng.integers(0, 1100, 700)]          # repeats included
    check(cache, query(700, 8, 64, torch.bfloat16), seqs=some)


def test_layers_strided_queries_and_scale():
    U.require_gpu()
    lens = [100, 0, 37, 512]
    cache = K.filled_cache(PagedKVCache, lens, 32, 4, 128, "f16", layers=3, seed=5)
    wide = query(4, 8 + 4 + 4, 128, torch.float16)                # one fused q/k/v row
    for layer in range(3):
        check(cache, wide[:, :8], layer=layer, scale=0.2)
    check(cache, wide[:, :8], layer=1, scale=-0.05)
    check(cache, wide[:, :8], layer=1, scale=0.0)


@pytest.mark.parametrize("dt", ["f16", "bf16", "e4m3"])
def test_sharp_softmax(dt):
    """Scores of hundreds: one token's weight is all but one, the maximum moves late."""
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [900, 33, 1], 16, 2, 128, dt, seed=6)
    check(cache, query(3, 8, 128, DT.get(dt, torch.bfloat16), gain=60.0))


def test_e4m3_value_scales_far_apart():
    """Value scales from 2^-60 to 2^60: the weights' range follows p 2^b."""
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [300, 17, 64], 16, 2, 64, "e4m3", seed=7, v_exp=50)
    check(cache, query(3, 8, 64, torch.bfloat16))


def test_e4m3_bf16_queries_beyond_fp16():
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [200, 9], 16, 2, 64, "e4m3", seed=8)
    q = query(2, 4, 64, torch.bfloat16)
    check(cache, (q.float() * 2.0 ** 30).to(torch.bfloat16), scale=2.0 ** -33)
    check(cache, (q.float() * 2.0 ** -40).to(torch.bfloat16), scale=2.0 ** 37)


def test_offsets_past_32_bits():
    """A pool of more than 2^32 bytes and 2^31 elements whose highest pages are the ones in use."""
    U.require_gpu()
    pages = (5 << 30) // (2 * 8 * 64 * 128)                      # 5 GiB of keys
    cache = K.filled_cache(PagedKVCache, [1000, 130], 64, 8, 128, "bf16", seed=9, num_pages=pages)
    assert cache.k.numel() > 1 << 31 and int(cache.tables.max()) == pages - 1
    check(cache, query(2, 16, 128, torch.bfloat16))


@pytest.mark.parametrize("dt,page,window", [("f16", 16, 33), ("bf16", 8, 5), ("e4m3", 32, 70), ("e4m3", 8, 1)])
def test_nan_before_the_window_is_not_seen(dt, page, window):
    """Tokens that the window leaves out hold NaN (8-bit ones with a NaN code and the largest
    scale): also those that share a chunk with tokens that are seen."""
    U.require_gpu()
    lens = [100, 37, 3, 250]
    cache = K.filled_cache(PagedKVCache, lens, page, 2, 64, dt, seed=16)
    for s, n in enumerate(lens):
        for t in range(max(0, n - window)):
            at = int(cache.tables[s, t // page])
            for pool, scales in ((cache.k, cache.k_scales), (cache.v, cache.v_scales)):
                if scales is None:
                    pool[0, at, :, t % page] = float("nan")
                else:
                    pool.view(torch.uint8)[0, at, :, t % page] = 0x7f
                    scales[0, at, :, t % page] = 254
    check(cache, query(4, 8, 64, DT.get(dt, torch.float16)), window=window)


def test_scale_bytes_of_unseen_slots_do_not_matter():
    """The extreme scale bytes in slots past a length, which are fetched four at a time with seen ones."""
    U.require_gpu()
    lens = [5, 33, 62, 1, 127]
    cache = K.filled_cache(PagedKVCache, lens, 16, 2, 64, "e4m3", seed=17)
    q = query(5, 8, 64, torch.bfloat16)
    want = check(cache, q)
    for byte in (0, 1, 127, 254, 255):
        for s, n in enumerate(lens):
            for t in range(n, -(-n // 16) * 16):
                at = int(cache.tables[s, t // 16])
                cache.k_scales[0, at, :, t % 16] = byte
                cache.v_scales[0, at, :, t % 16] = byte
        assert torch.equal(cache.attend(q), want), byte


def test_nan_in_a_cached_value_reaches_its_rows_only():
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [50, 60], 16, 2, 64, "f16", seed=10)
    cache.v[0, int(cache.tables[0, 1]), 1, 3] = float("nan")     # token 19 of sequence 0, head 1
    out = cache.attend(query(2, 4, 64, torch.float16))
    assert bool(torch.isnan(out[0, 2:]).all())
    assert not bool(torch.isnan(out[0, :2]).any()) and not bool(torch.isnan(out[1]).any())


def test_another_stream_and_a_graph():
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [400, 1, 77], 16, 2, 128, "bf16", seed=11)
    q = query(3, 8, 128, torch.bfloat16)
    want = cache.attend(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = cache.attend(q)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graph, static = torch.cuda.CUDAGraph(), torch.empty_like(want)
    with torch.cuda.stream(side):
        cache.attend(q, out=static)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        cache.attend(q, out=static)
    for n in (13, 400, 399):                                     # lengths are read on the device
        cache.lens[0] = n
        static.zero_()
        graph.replay()
        assert torch.equal(static, cache.attend(q))


def test_bad_bookkeeping_is_recorded_not_followed():
    """Indices and lengths outside the cache are kept inside it by the kernel and reported."""
    U.require_gpu()
    from paper_2606_12876_gb300 import AQ_ERR_INVALID_ARG, AQError

    def fails(cache, q, seqs=None):
        out = cache.attend(q, seqs)
        with pytest.raises(AQError) as e:
            cache.check()
        assert e.value.status == AQ_ERR_INVALID_ARG
        cache.check()                                            # cleared
        return out

    q = query(2, 4, 64, torch.float16)
    cache = K.filled_cache(PagedKVCache, [50, 20], 16, 2, 64, "f16", seed=12)
    good = cache.attend(q)
    out = fails(cache, q, torch.tensor([0, 2], dtype=torch.int32, device="cuda"))
    assert torch.equal(out[0], good[0]) and not bool(out[1].any())
    cache.lens[1] = -5
    out = fails(cache, q)
    assert torch.equal(out[0], good[0]) and not bool(out[1].any())
    cache.lens[1] = 20
    cache.tables[1, 1] = 1 << 20                                 # read as zeros
    assert torch.equal(fails(cache, q)[0], good[0])


def test_refusals():
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [50, 20], 16, 2, 64, "f16", seed=13)
    q = query(2, 4, 64, torch.float16)
    bad = [dict(q=q.bfloat16()), dict(q=q[:, :3]), dict(q=q[..., :32]), dict(q=q.transpose(0, 1)),
           dict(q=query(3, 4, 64, torch.float16)), dict(q=q, layer=1), dict(q=q, window=-1),
           dict(q=q, scale=float("nan")), dict(q=q, out=torch.empty(2, 4, 64, device="cuda")),
           dict(q=q, lse=torch.empty(2, 3, device="cuda")), dict(q=q, seqs=torch.zeros(2, device="cuda")),
           dict(q=q, seqs=torch.zeros(3, dtype=torch.int32, device="cuda"))]
    for kw in bad:
        with pytest.raises((TypeError, ValueError, RuntimeError)):
            cache.attend(**kw)
    assert cache.attend(q[:0]).shape == (0, 4, 64)


def test_first_call_inside_a_capture_is_refused():
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [50, 20], 16, 2, 64, "f16", seed=14)
    q = query(2, 4, 64, torch.float16)
    out, graph, x = torch.empty_like(q), torch.cuda.CUDAGraph(), torch.zeros(4, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        x.add_(1)
        with pytest.raises(RuntimeError):
            cache.attend(q, out=out)
    torch.cuda.synchronize()
    cache.attend(q, out=out)
    cache.check()
