"""The paged cache's bookkeeping and writes (aq_kv_init, reserve, fork, free, compact, copy_pages,
write) against a plain model, exactly."""
import numpy as np
import pytest
import torch

import aq_testutil as U
import kv_testutil as K
import paper_2606_12876_gb300 as aq
from paper_2606_12876_gb300.kv import PagedKVCache

pytestmark = pytest.mark.gpu


def ints(v):
    return torch.as_tensor(list(v), dtype=torch.int32, device="cuda")


def raw(t):
    return t.view(torch.uint8 if t.element_size() == 1 else torch.int16)


def scramble(cache, seed=0):
    """Every byte of the pools random (NaN patterns among them): copies are compared bit for bit."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    for t in (cache.k, cache.v, cache.k_scales, cache.v_scales):
        if t is not None:
            t.view(torch.uint8).random_(0, 256, generator=g)


def pools(cache):
    return [raw(t).clone() for t in (cache.k, cache.v, cache.k_scales, cache.v_scales) if t is not None]


def assert_copied(cache, before, copies):
    now = [raw(t) for t in (cache.k, cache.v, cache.k_scales, cache.v_scales) if t is not None]
    for b, t in zip(before, now):
        want = b.clone()
        for a, d in copies:
            want[:, d] = b[:, a]
        assert torch.equal(t, want)


def expect(cache, what):
    status = {"invalid": aq.AQ_ERR_INVALID_ARG, "capacity": aq.AQ_ERR_CAPACITY}
    if what == "ok":
        cache.check()
    else:
        with pytest.raises(aq.AQError) as e:
            cache.check()
        assert e.value.status == status[what]


@pytest.mark.parametrize("dtype,page,heads,dim,layers", [("bf16", 16, 2, 64, 2), ("e4m3", 8, 3, 80, 1),
                                                          ("f16", 64, 1, 16, 3)])
def test_random_traffic_follows_the_model(dtype, page, heads, dim, layers):
    U.require_gpu()
    rng = np.random.Generator(np.random.PCG64(page))
    P, S, W = 90, 24, 11
    cache = PagedKVCache(P, page, heads, dim, S, W, layers=layers, dtype=dtype)
    model = K.Model(P, page, S, W)
    scramble(cache, page)
    seen = set()
    for step in range(150):
        op = rng.choice(["reserve", "reserve", "fork", "free", "compact"])
        before = pools(cache)
        model.copies, what = [], "ok"
        if op == "reserve":
            seqs = [int(s) for s in rng.permutation(S)[: rng.integers(0, 9)]]
            counts = [int(c) for c in rng.integers(0, 3 * page, len(seqs))] if rng.random() < 0.8 else None
            what = model.reserve(seqs, counts)
            cache.reserve(ints(seqs), None if counts is None else ints(counts))
        elif op == "fork":
            empty = [s for s in range(S) if model.lens[s] == 0]
            dst = [int(s) for s in rng.permutation(empty)[: rng.integers(0, 5)]] if empty else []
            if dst and rng.random() < 0.1:
                dst[0] = int(rng.integers(0, S))                 # perhaps not empty
            src = [int(s) for s in rng.integers(0, S, len(dst))]
            what = model.fork(src, dst)
            cache.fork(ints(src), ints(dst))
        elif op == "free":
            seqs = [int(s) for s in rng.integers(0, S, rng.integers(0, 4))]
            model.free(seqs)                                     # repeats are released once
            cache.free(ints(seqs))
        else:
            used = ints([-1])
            U_ = model.compact()
            cache.compact(used)
            assert used.tolist() == [U_]
        seen.add((op, what))
        expect(cache, what)
        model.assert_same(cache)
        assert_copied(cache, before, model.copies)
    assert {("reserve", "ok"), ("reserve", "capacity"), ("fork", "ok"), ("free", "ok"), ("compact", "ok")} <= seen


def test_reserve_refusals_leave_the_cache_as_it_was():
    U.require_gpu()
    cache = PagedKVCache(10, 16, 1, 16, 6, 4)
    model = K.Model(10, 16, 6, 4)
    assert model.reserve([0, 1], [20, 33]) == "ok"
    cache.reserve(ints([0, 1]), ints([20, 33]))
    for seqs, counts, what in [([0, 6], [1, 1], "invalid"), ([-1], [1], "invalid"), ([2, 2], [1, 1], "invalid"),
                               ([2], [-1], "invalid"), ([2], [65], "capacity"), ([1], [32], "capacity"),
                               ([2, 3], [64, 33], "capacity"), ([2], [2147483647], "capacity")]:
        cache.reserve(ints(seqs), ints(counts))
        expect(cache, what)
        model.assert_same(cache)
    for src, dst in [([0], [1]), ([0, 0], [2, 2]), ([9], [2]), ([0], [7]), ([0], [0])]:
        cache.fork(ints(src), ints(dst))
        expect(cache, "invalid")
        model.assert_same(cache)
    cache.free(ints([17]))
    expect(cache, "invalid")
    model.assert_same(cache)
    cache.fork(ints([2]), ints([3]))                             # an empty parent
    expect(cache, "ok")
    model.assert_same(cache)


def test_large_pool_and_long_tables():
    """More pages than one step of the search for free ones, and a table longer than a CTA."""
    U.require_gpu()
    P, page, S, W = 70001, 8, 5, 40000
    cache = PagedKVCache(P, page, 1, 16, S, W)
    model = K.Model(P, page, S, W)

    def both(op, *lists):
        what = getattr(model, op)(*lists)
        getattr(cache, op)(*[ints(v) for v in lists])
        expect(cache, what if op in ("reserve", "fork") else "ok")
        model.assert_same(cache)

    both("reserve", [3, 0], [40000 * 8 - 3, 100000])
    both("reserve", [1], [17 * 8])
    both("free", [3])
    both("fork", [0, 0], [2, 4])
    both("reserve", [2, 4, 1], [7, 8, 9])
    cache.compact()
    model.compact()
    model.assert_same(cache)
    both("reserve", [3], [40000 * 8])
    both("free", [0, 2, 4, 3, 3])
    cache.compact()
    model.compact()
    model.assert_same(cache)


def test_copy_pages():
    U.require_gpu()
    cache = PagedKVCache(40, 32, 3, 96, 2, layers=2, dtype="e4m3")
    scramble(cache, 1)
    before = pools(cache)
    src, dst = [5, 5, 39, 0], [1, 38, 7, 20]
    cache.copy_pages(ints(src), ints(dst))
    expect(cache, "ok")
    assert_copied(cache, before, list(zip(src, dst)))
    before = pools(cache)
    cache.copy_pages(ints([3, 40, 2]), ints([4, 6, -1]))
    expect(cache, "invalid")
    assert_copied(cache, before, [(3, 4)])
    cache.copy_pages(ints([]), ints([]))


def e4m3_exact(x):
    """Codes' values and scale exponents of fp64 rows x: the definition, step by step."""
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -300) / 448)).clamp(-60, 60)
    e = torch.where(amax > 448 * torch.exp2(e), e + 1, e)         # (log2 rounds)
    e = torch.where(amax <= 448 * torch.exp2(e - 1), e - 1, e).clamp(-60, 60)
    z = (x * torch.exp2(-e)).clamp(-448, 448)
    step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(z / step) * step, e[..., 0]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "e4m3"])
@pytest.mark.parametrize("xdt", [torch.float16, torch.bfloat16, torch.float32])
def test_write(dtype, xdt):
    U.require_gpu()
    lens, page, heads, dim = [5, 64, 0, 33, 17], 16, 3, 80
    for stride in (0, 2):                                        # rows alone, rows of a wider matrix
        cache = K.filled_cache(PagedKVCache, lens, page, heads, dim, dtype, layers=2, seed=3)
        scramble(cache, 2)
        seqs, pos = [0, 1, 1, 3, 4, 3], [4, 0, 63, 32, 16, 15]
        g = torch.Generator(device="cuda")
        g.manual_seed(5)
        wide = torch.randn(6, 2 * heads + stride, dim, device="cuda", generator=g) * \
            torch.exp2(torch.randint(-12, 6, (6, 2 * heads + stride, 1), device="cuda", generator=g).float())
        wide[0, 0] = 0
        wide[1, 1, 3:] = 0
        wide[2, 0, 7] = 448 * 2.0 ** 5                            # just fits a scale, and just does not
        wide[2, 1, 7] = 450 * 2.0 ** 5
        wide = wide.to(xdt)
        k, v = wide[:, :heads], wide[:, heads:2 * heads]
        want = pools(cache)
        for which, x in ((0, k), (1, v)):
            for i, (s, p) in enumerate(zip(seqs, pos)):
                at = int(cache.tables[s, p // page])
                if dtype == "e4m3":
                    z, e = e4m3_exact(x[i].double())
                    want[which][1, at, :, p % page] = z.float().to(torch.float8_e4m3fn).view(torch.uint8)
                    want[2 + which][1, at, :, p % page] = (e + 127).to(torch.uint8)
                else:
                    want[which][1, at, :, p % page] = raw(x[i].to(cache.dtype))
        cache.write(k, v, ints(seqs), ints(pos), layer=1)
        expect(cache, "ok")
        for a, b, x in zip(want, pools(cache), "kvab"):
            # (-0 is a code of its own: compare zeros by value)
            same = (a == b) | ((a.int() & 0x7f) + (b.int() & 0x7f) == 0) if dtype == "e4m3" and x in "kv" else a == b
            assert bool(same.all())
        # without positions: each sequence's last token
        cache.write(k[:2], v[:2], ints([4, 0]), layer=0)
        if dtype != "e4m3":
            assert torch.equal(cache.k[0, int(cache.tables[4, 1]), :, 0], k[0].to(cache.dtype))
            assert torch.equal(cache.v[0, int(cache.tables[0, 0]), :, 4], v[1].to(cache.dtype))


def test_write_outside_the_cache_is_skipped():
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [20, 0], 16, 2, 32, "f16", seed=4)
    scramble(cache, 3)
    before = pools(cache)
    x = torch.ones(5, 2, 32, device="cuda", dtype=torch.float16)
    cache.write(x, x, ints([0, 0, 1, 2, -1]), ints([20, -1, 0, 0, 0]))
    expect(cache, "invalid")
    assert_copied(cache, before, [])
    cache.write(x[:0], x[:0], ints([]))
    expect(cache, "ok")


def test_write_special_values_e4m3():
    """Infinities saturate at the largest scale, NaN stays NaN, values past the scales' range
    saturate or vanish."""
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [16], 16, 1, 16, "e4m3", seed=4)
    x = torch.ones(4, 1, 16, device="cuda")
    x[0, 0, 3] = float("inf")
    x[1, 0, 3] = float("nan")
    x[2] = 2.0 ** 100
    x[3] = 2.0 ** -100
    cache.write(x, x, ints([0] * 4), ints([0, 1, 2, 3]))
    got = K.values(cache, "v")[0, int(cache.tables[0, 0]), 0]
    assert float(got[0, 3]) == 448 * 2.0 ** 60 and float(got[0, 0]) == 0
    assert bool(torch.isnan(got[1, 3])) and float(got[1, 0]) == 1
    assert bool((got[2] == 448 * 2.0 ** 60).all()) and not bool(got[3].any())


def test_a_captured_decode_step():
    """reserve, write and attend captured once and replayed: the sequences grow page by page."""
    U.require_gpu()
    page, heads, dim, n = 8, 2, 64, 3
    caches = [PagedKVCache(32, page, heads, dim, n, 10, dtype="bf16") for _ in range(2)]
    seqs = ints(range(n))
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    rows = torch.randn(20, n, 3 * heads, dim, device="cuda", generator=g).bfloat16()
    x = rows[0].clone()

    def step(cache, t):
        cache.reserve(seqs)
        cache.write(t[:, :heads], t[:, heads:2 * heads], seqs)
        return cache.attend(t[:, 2 * heads:])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(caches[1], x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
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


def test_binding_refusals():
    U.require_gpu()
    cache = PagedKVCache(8, 16, 2, 64, 4, dtype="bf16")
    x = torch.zeros(2, 2, 64, device="cuda", dtype=torch.bfloat16)
    s = ints([0, 1])
    for call in [lambda: cache.reserve(s.long()), lambda: cache.reserve(s.cpu()), lambda: cache.reserve(s, ints([1])),
                 lambda: cache.reserve(ints(range(5))), lambda: cache.fork(s, ints([1])), lambda: cache.fork(s, s[::2]),
                 lambda: cache.write(x, x[:, :1], s), lambda: cache.write(x, x.float(), s),
                 lambda: cache.write(x.double(), x.double(), s), lambda: cache.write(x, x, s, layer=1),
                 lambda: cache.write(x, x, s, layer=-1), lambda: cache.write(x.transpose(0, 1), x, s),
                 lambda: cache.compact(ints([1, 2])), lambda: PagedKVCache(8, 24, 2, 64, 4),
                 lambda: PagedKVCache(8, 16, 2, 72, 4), lambda: PagedKVCache(8, 16, 2, 512, 4),
                 lambda: PagedKVCache.from_tensors(cache.k, cache.v[:, ::2], cache.tables, cache.lens, cache.refs)]:
        with pytest.raises((TypeError, ValueError, RuntimeError)):
            call()


def test_lists_of_more_than_a_thousand_sequences():
    """Entries beyond one CTA's threads: reserve and fork of 1500 sequences, and their refusals."""
    U.require_gpu()
    P, page, S, W = 9000, 8, 3200, 6
    cache = PagedKVCache(P, page, 1, 16, S, W, dtype="f16")
    model = K.Model(P, page, S, W)
    scramble(cache, 7)
    rng = np.random.Generator(np.random.PCG64(8))
    some = [int(s) for s in rng.permutation(1600)[:1500]]
    counts = [int(v) for v in rng.integers(0, 30, 1500)]

    def both(op, *lists):
        before = pools(cache)
        model.copies = []
        what = getattr(model, op)(*lists)
        getattr(cache, op)(*[ints(v) for v in lists])
        expect(cache, what if op != "free" else "ok")
        model.assert_same(cache)
        assert_copied(cache, before, model.copies)
        return what

    assert both("reserve", some, counts) == "ok"
    assert both("fork", some, [1600 + i for i in range(1500)]) == "ok"
    assert both("fork", some, [1600 + i for i in range(1500)]) == "invalid"
    assert both("reserve", some[:1499] + some[:1]) == "invalid"
    assert both("reserve", some[:1400], [48] * 1400) == "capacity"
    assert both("reserve", some) in ("ok", "capacity")
    assert both("free", some) is None
    assert both("reserve", list(range(1600, 3100)), [1] * 1500) in ("ok", "capacity")
