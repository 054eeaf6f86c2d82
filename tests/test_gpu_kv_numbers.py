"""The numbers of aq_kv_attend where the weights or the scales are extreme, against fp64 within the
bound that aq.h states: long contexts under one token with most of the weight, scores beyond 2^24,
value and key scales at both ends of their range.

bound() is that statement and nothing else. With E the error of the weights' sum over v, p relative to
their maximum, u = 2^-8 (bf16) or 2^-11 (fp16, E4M3) and b_t the value scales (1 without them):
    E <= u sum_t p_t |v_t| / sum p  +  2^-40 max(p_t b_t) sum_t |v_t| / b_t / sum p     (no second term: bf16)
a score's error d enters out twice (its own weight and the sum), and out is rounded once."""
import pytest
import torch

import aq_testutil as U
import kv_testutil as K
from paper_2606_12876_gb300.kv import PagedKVCache

pytestmark = pytest.mark.gpu
PAGE = 64


def ints(v):
    return torch.as_tensor(v, dtype=torch.int32, device="cuda")


def cache_of(k, v, dtype, k_exp=None, v_exp=None):
    """A cache of one sequence, [kv_heads][tokens][head_dim]; E4M3: k and v are the codes' values,
    k_exp and v_exp ([kv_heads][tokens]) their scales' exponents."""
    heads, n, dim = k.shape
    pages = -(-n // PAGE)
    cache = PagedKVCache(pages, PAGE, heads, dim, 1, dtype=dtype)
    cache.reserve(ints([0]), ints([n]))
    pad = lambda t: torch.nn.functional.pad(t, (0, 0) * (t.dim() - 2) + (0, pages * PAGE - n))

    def put(pool, t):
        pool[0].copy_(pad(t).view(heads, pages, PAGE, *t.shape[2:]).transpose(0, 1))

    put(cache.k, k.to(cache.dtype))
    put(cache.v, v.to(cache.dtype))
    if dtype == "e4m3":
        put(cache.k_scales, (k_exp + 127).to(torch.uint8))
        put(cache.v_scales, (v_exp + 127).to(torch.uint8))
    cache.check()
    return cache


def bound(cache, q, scale):
    """(out, lse, bound on out, bound on lse) of the one sequence, from the cache's contents."""
    n = int(cache.lens[0])
    heads, dim, small = cache.kv_heads, cache.head_dim, cache.k_scales is not None

    def rows(t):
        return t[0, cache.tables[0, : -(-n // PAGE)].long()].transpose(0, 1).reshape(heads, -1, *t.shape[4:])[:, :n]

    k, v = rows(K.values(cache, "k")), rows(K.values(cache, "v"))
    b = torch.exp2(rows(cache.v_scales).double() - 127) if small else torch.ones(heads, n, dtype=torch.float64, device="cuda")
    qd = q[0].double().view(heads, -1, dim)
    s = qd @ k.transpose(1, 2) * scale
    mag = (qd.abs() @ k.abs().transpose(1, 2) * abs(scale)).amax(-1)
    p = torch.softmax(s, -1)
    out, lse = p @ v, torch.logsumexp(s, -1)
    # a score: fp32 products, their sum, the factor to base 2, the difference to the maximum, exp2
    d = (dim + 16) * 2.0 ** -23 * mag + 2.0 ** -19
    A = p @ v.abs()
    E = (2.0 ** -8 if cache.dtype == torch.bfloat16 else 2.0 ** -11) * A
    if cache.dtype != torch.bfloat16:
        E = E + 2.0 ** -40 * (p * b[:, None]).amax(-1)[..., None] * (v.abs() / b[..., None]).sum(1)[:, None]
    e = (E + 2 * d[..., None] * A) * 1.01
    tol = e + K.UNIT[q.dtype] * (out.abs() + e) + K.TINY[q.dtype]
    return out, lse, tol, d + 2.0 ** -21 * lse.abs()


def check(cache, q, scale=1.0):
    lse = torch.empty(q.shape[:2], device="cuda")
    got = cache.attend(q, scale=scale, lse=lse)
    cache.check()
    out, want_lse, tol, tol_lse = bound(cache, q, scale)
    err = (got[0].double().view_as(out) - out).abs()
    assert bool((err <= tol).all()), "largest error/bound %.3g, relative error %.3g" % (
        float((err / tol).max()), float((err / out.abs().clamp(min=1e-300)).max()))
    assert bool(((lse[0].double().view_as(want_lse) - want_lse).abs() <= tol_lse).all())


def first_dim(scores, dim):
    """Keys whose product with a query of (1, 0, ...) is the score."""
    k = torch.zeros(*scores.shape, dim, device="cuda")
    k[..., 0] = scores
    return k


def unit_query(heads, dim, dtype):
    q = torch.zeros(1, heads, dim, device="cuda", dtype=dtype)
    q[..., 0] = 1
    return q


# (1280 heads: a warp has a whole one, so that one maximum holds for all of its tokens)
SIZES = [(2, 300, 64), (2, 131071, 64), (1280, 32760, 16)]


@pytest.mark.parametrize("heads,n,dim", SIZES)
@pytest.mark.parametrize("tail", ["flat", "normal"])
@pytest.mark.parametrize("dtype", ["f16", "bf16", "e4m3"])
def test_a_long_tail_under_one_large_weight(dtype, tail, heads, n, dim):
    """One token with a small value takes most of the weight; every other weight is about 2^-26 of it.
    Together they make up a part of the sum that no output may lose."""
    U.require_gpu()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    s = torch.zeros(heads, n, device="cuda")
    if tail == "normal":
        s.normal_(generator=g)
    s[::2, 7] = s[1::2, n - 9] = 18
    v = torch.randn(heads, n, dim, device="cuda", generator=g).mul_(0.25).add_(1)
    v[::2, 7] = v[1::2, n - 9] = 2.0 ** -7
    zero = torch.zeros(heads, n, device="cuda")
    cache = cache_of(first_dim(s, dim), v, dtype, zero, zero)
    group = 8 if heads == 2 else 1
    for qd in [torch.float16, torch.bfloat16] if dtype == "e4m3" else [cache.dtype]:
        check(cache, unit_query(group * heads, dim, qd))


@pytest.mark.parametrize("heads,n,dim", SIZES)
def test_a_large_value_scale_over_a_long_tail(heads, n, dim):
    """E4M3: the largest weight times scale belongs to a token whose codes are 0; the others' are 2^-26 of it."""
    U.require_gpu()
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    v = torch.randn(heads, n, dim, device="cuda", generator=g).mul_(0.25).add_(1)
    v[:, 3] = 0
    v_exp = torch.zeros(heads, n, device="cuda")
    v_exp[:, 3] = 26
    cache = cache_of(first_dim(torch.zeros(heads, n, device="cuda"), dim), v, "e4m3", v_exp * 0, v_exp)
    check(cache, unit_query(heads, dim, torch.float16))


@pytest.mark.parametrize("n", [40, 5000])
@pytest.mark.parametrize("exp", [1, 5, 20, 37, 60, -37])
def test_scores_whose_sum_with_a_scale_is_rounded(exp, n):
    """E4M3, equal base-2 scores of 2^22 to 2^40 and value scales of 2^exp: the running maximum is taken over
    sums that fp32 rounds. Equal scores have equal weights whatever their size: out is the mean of v, the
    weights' rounding and the sum's (n 2^-23 at worst) aside."""
    U.require_gpu()
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    dim = 64
    v = (1 + 0.25 * torch.randn(1, n, dim, device="cuda", generator=g)).to(torch.float8_e4m3fn).float()
    for top in (2.0 ** 22, 2.0 ** 24, 1.5 * 2.0 ** 24, 2.0 ** 26, 2.0 ** 29, 2.0 ** 40):
        k = first_dim(torch.full((1, n), 1.0, device="cuda"), dim)
        e = torch.full((1, n), float(exp), device="cuda")
        cache = cache_of(k, v, "e4m3", e * 0, e)
        out = cache.attend(unit_query(4, dim, torch.bfloat16), scale=top * 0.6931471805599453)
        want = v[0].double().mean(0) * 2.0 ** exp
        rel = ((out[0].double() - want).abs() / want).max()
        assert float(rel) <= 2.0 ** -8 + 2.0 ** -11 + n * 2.0 ** -23, (top, float(rel))


@pytest.mark.parametrize("kv_heads,n", [(2, 33), (1, 20000), (8, 3000)])
def test_scales_at_both_ends(kv_heads, n):
    """E4M3: key and value scales of exactly 2^-60 and 2^60 side by side, within a warp's piece and in pieces
    that are merged. A key's scale is undone in its code's place in the query, so that the scores stay
    moderate: dimension 0 meets the keys of 2^60, dimension 1 those of 2^-60."""
    U.require_gpu()
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    dim = 64
    pick = torch.rand(kv_heads, n, device="cuda", generator=g) < 0.5
    k = torch.zeros(kv_heads, n, dim, device="cuda")
    code = torch.randint(-8, 9, (kv_heads, n), device="cuda", generator=g).float()
    k[..., 0] = torch.where(pick, code, 0.0)
    k[..., 1] = torch.where(pick, 0.0, code)
    k_exp = torch.where(pick, 60.0, -60.0)
    v = torch.randn(kv_heads, n, dim, device="cuda", generator=g).mul_(100).clamp_(-448, 448)
    for share in (0.5, 1e-3):
        v_exp = torch.where(torch.rand(kv_heads, n, device="cuda", generator=g) < share, 60.0, -60.0)
        v_exp[:, 0], v_exp[:, -1] = -60, 60
        cache = cache_of(k, v, "e4m3", k_exp, v_exp)
        # the small keys' query would need 2^60: the scores of the two kinds are looked at one after the other
        for at, gain in ((0, 2.0 ** -62), (1, 2.0 ** 58)):
            q = torch.zeros(1, 4 * kv_heads, dim, device="cuda", dtype=torch.bfloat16)
            q[..., at] = gain
            check(cache, q)                      # (outputs of up to 2^69: bf16 holds them)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 40 + 1])
def test_windows_longer_than_any_sequence(window):
    U.require_gpu()
    cache = K.filled_cache(PagedKVCache, [100, 7], 16, 2, 64, "bf16", seed=5)
    q = torch.randn(2, 4, 64, device="cuda").bfloat16()
    assert torch.equal(cache.attend(q, window=window), cache.attend(q))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "e4m3"])
@pytest.mark.parametrize("heads,n", [(1, 20000), (8, 700), (8, 40)])
def test_tokens_on_bad_pages_are_zeros(dtype, heads, n):
    """Table entries outside the pool in half of a sequence, all but its end or everywhere: recorded, and the same
    as keys and values of zero, also where a warp's whole piece has no other tokens."""
    U.require_gpu()
    from paper_2606_12876_gb300 import AQ_ERR_INVALID_ARG, AQError
    dim = 64
    cache = K.filled_cache(PagedKVCache, [n], PAGE, heads, dim, dtype, seed=6)
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    q = (torch.randn(1, 4 * heads, dim, device="cuda", generator=g) * 2).to(torch.float16 if dtype == "e4m3" else cache.dtype)
    pages = -(-n // PAGE)
    for bad in {max(pages - 1, 1), -(-pages // 2), pages}:
        zeroed = K.filled_cache(PagedKVCache, [n], PAGE, heads, dim, dtype, seed=6)
        at = zeroed.tables[0, :bad].long()
        for t in (zeroed.k, zeroed.v):
            t.view(torch.uint8)[:, at] = 0
        want, want_lse, tol, tol_lse = K.attend_exact(zeroed, q, [0], 0, dim ** -0.5, 0)
        cache.tables.copy_(zeroed.tables)
        cache.tables[0, :bad] = 1 << 20
        lse = torch.empty(1, 4 * heads, device="cuda")
        out = cache.attend(q, lse=lse)
        with pytest.raises(AQError) as e:
            cache.check()
        assert e.value.status == AQ_ERR_INVALID_ARG
        assert bool(((out.double() - want).abs() <= tol).all()), bad
        assert bool(((lse.double() - want_lse).abs() <= tol_lse).all()), bad
