"""The key-value cache and the RMS norm without a GPU: size queries and the host-side refusals of
the C entry points (fake addresses, never dereferenced)."""
import ctypes

import pytest

import aq_testutil
import paper_2606_12876_gb300 as aq

FAKE = 1 << 20
BIG = 1 << 40
INV, UNS, ALI, WS = aq.AQ_ERR_INVALID_ARG, aq.AQ_ERR_UNSUPPORTED, aq.AQ_ERR_ALIGNMENT, aq.AQ_ERR_WORKSPACE


@pytest.fixture(scope="module", autouse=True)
def built():
    aq_testutil.ensure_built()


def cache(**kw):
    d = dict(layers=2, num_pages=10, page_tokens=16, kv_heads=2, head_dim=64, max_seqs=4, max_pages=5,
             dtype=aq.AQ_BF16, k=FAKE, v=FAKE, k_scales=None, v_scales=None, tables=FAKE, lens=FAKE, refs=FAKE)
    d.update(kw)
    return aq.KVCache(*[d[f] for f, _ in aq.KVCache._fields_])


BAD_CACHES = [(dict(layers=0), INV), (dict(num_pages=0), INV), (dict(kv_heads=0), INV), (dict(max_seqs=0), INV),
              (dict(max_pages=-1), INV), (dict(head_dim=0), INV), (dict(page_tokens=0), INV), (dict(dtype=2), INV),
              (dict(dtype=4), INV), (dict(page_tokens=4), UNS), (dict(page_tokens=24), UNS),
              (dict(page_tokens=2048), UNS), (dict(head_dim=72), UNS), (dict(head_dim=272), UNS),
              (dict(max_pages=1 << 28, page_tokens=16), UNS), (dict(max_pages=(1 << 27) - 1, page_tokens=16), UNS),
              (dict(kv_heads=16385), UNS)]
BAD_BOOKS = [(dict(tables=None), INV), (dict(lens=None), INV), (dict(refs=None), INV), (dict(lens=FAKE + 2), ALI)]
BAD_POOLS = [(dict(k=None), INV), (dict(v=None), INV), (dict(k=FAKE + 8), ALI),
             (dict(dtype=aq.AQ_E4M3), INV), (dict(dtype=aq.AQ_E4M3, k_scales=FAKE, v_scales=FAKE + 8), ALI)]


def calls(c, n=2, lists=FAKE, ws=FAKE, size=BIG):
    L, r = aq.lib(), ctypes.byref(c)
    return {
        "reserve": lambda: L.aq_kv_reserve(r, n, lists, lists, ws, size, None),
        "fork": lambda: L.aq_kv_fork(r, n, lists, lists, ws, size, None),
        "free": lambda: L.aq_kv_free(r, n, lists, ws, size, None),
        "compact": lambda: L.aq_kv_compact(r, None, ws, size, None),
        "copy": lambda: L.aq_kv_copy_pages(r, n, lists, lists, ws, size, None),
        "write": lambda: L.aq_kv_write(r, 0, n, lists, lists, FAKE, FAKE, aq.AQ_BF16, 128, ws, size, None),
        "attend": lambda: L.aq_kv_attend(r, 0, n, lists, FAKE, aq.AQ_BF16, 256, 4, 0.125, 0, FAKE, None, ws, size, None),
    }


@pytest.mark.parametrize("kw,status", BAD_CACHES + BAD_BOOKS)
def test_bad_caches(kw, status):
    for name, call in calls(cache(**kw)).items():
        assert call() == status, name
    assert aq.lib().aq_kv_init(ctypes.byref(cache(**kw)), None) == status
    assert (aq.kv_workspace_bytes(cache(**kw)) == 0) == ((kw, status) in BAD_CACHES)


@pytest.mark.parametrize("kw,status", BAD_POOLS)
def test_bad_pools(kw, status):
    for name, call in calls(cache(**kw)).items():
        if name not in ("reserve", "free"):
            assert call() == status, name


def test_null_cache():
    L = aq.lib()
    assert L.aq_kv_workspace_bytes(None) == 0 and L.aq_kv_attend_workspace_bytes(None, 1, 1) == 0
    assert L.aq_kv_init(None, None) == INV
    assert L.aq_kv_reserve(None, 1, FAKE, FAKE, FAKE, BIG, None) == INV
    assert L.aq_kv_attend(None, 0, 1, FAKE, FAKE, aq.AQ_BF16, 256, 4, 1.0, 0, FAKE, None, FAKE, BIG, None) == INV


def test_lists_and_workspaces():
    c = cache()
    need = aq.kv_workspace_bytes(c)
    assert need > 0
    for name, call in calls(c, n=-1).items():
        if name != "compact":
            assert call() == INV, name
    for name in ("reserve", "fork"):
        assert calls(c, n=5)[name]() == INV                      # more entries than sequences
    for name in ("free", "write", "attend"):
        assert calls(c, n=5, lists=None)[name]() == INV
    for name in ("fork", "copy"):
        assert calls(c, lists=None)[name]() == INV
    for name, call in calls(c, lists=FAKE + 2).items():
        if name != "compact":
            assert call() == ALI, name
    for name, call in calls(c, ws=None).items():
        assert call() == WS, name
    for name, call in calls(c, ws=FAKE + 8).items():
        assert call() == ALI, name
    for name, call in calls(c, size=need - 1).items():
        assert call() == WS, name
    assert calls(c, size=aq.kv_attend_workspace_bytes(c, 2, 4) - 1)["attend"]() == WS
    for name, call in calls(c, n=0).items():
        if name != "compact":
            assert call() == aq.AQ_OK, name                      # nothing to do


def test_attend_arguments():
    L, c = aq.lib(), cache()

    def run(layer=0, q=FAKE, qd=aq.AQ_BF16, stride=256, heads=4, scale=0.1, window=0, out=FAKE, lse=None, cc=c):
        return L.aq_kv_attend(ctypes.byref(cc), layer, 2, FAKE, q, qd, stride, heads, scale, window, out, lse, FAKE,
                              BIG, None)

    for kw, status in [(dict(layer=2), INV), (dict(layer=-1), INV), (dict(heads=0), INV), (dict(heads=3), INV),
                       (dict(qd=aq.AQ_F32), INV), (dict(heads=(1 << 20) + 2, stride=1 << 30), UNS), (dict(qd=aq.AQ_F16), UNS), (dict(stride=248), INV),
                       (dict(stride=260), ALI), (dict(q=None), INV), (dict(out=None), INV), (dict(q=FAKE + 8), ALI),
                       (dict(out=FAKE + 4), ALI), (dict(lse=FAKE + 2), ALI), (dict(window=-1), INV),
                       (dict(scale=float("inf")), INV), (dict(scale=float("nan")), INV)]:
        assert run(**kw) == status, kw


def test_write_arguments():
    L, c = aq.lib(), cache()

    def run(layer=0, k=FAKE, v=FAKE, xd=aq.AQ_F32, stride=128):
        return L.aq_kv_write(ctypes.byref(c), layer, 2, FAKE, FAKE, k, v, xd, stride, FAKE, BIG, None)

    for kw, status in [(dict(layer=2), INV), (dict(layer=-1), INV), (dict(xd=aq.AQ_E4M3), INV), (dict(stride=120), INV),
                       (dict(stride=132), ALI), (dict(k=None), INV), (dict(v=None), INV), (dict(v=FAKE + 8), ALI)]:
        assert run(**kw) == status, kw


def test_rmsnorm_arguments():
    L = aq.lib()

    def run(rows=3, cols=64, x=FAKE, xd=1, xs=64, r=None, ro=None, rd=1, w=FAKE, wd=1, eps=1e-5, y=FAKE, yd=1, s=None,
            b=0):
        return L.aq_rmsnorm(rows, cols, x, xd, xs, r, ro, rd, w, wd, eps, y, yd, s, b, None)

    for kw, status in [(dict(rows=-1), INV), (dict(cols=0), INV), (dict(xd=3), INV), (dict(wd=3), INV), (dict(yd=4), INV),
                       (dict(xs=56), INV), (dict(eps=-1.0), INV), (dict(eps=float("nan")), INV),
                       (dict(r=FAKE, rd=3), INV), (dict(x=None), INV), (dict(w=None), INV), (dict(y=None), INV),
                       (dict(cols=60), UNS), (dict(cols=65544, xs=65544), UNS), (dict(xs=68), ALI),
                       (dict(x=FAKE + 8), ALI), (dict(w=FAKE + 8), ALI), (dict(y=FAKE + 8), ALI), (dict(r=FAKE + 8), ALI),
                       (dict(yd=3, b=32), INV), (dict(yd=3, b=16, s=FAKE), INV), (dict(yd=3, b=32, s=FAKE, cols=40), UNS)]:
        assert run(**kw) == status, kw
    assert run(rows=0, x=None) == aq.AQ_OK


def test_status_text():
    assert aq.status_string(aq.AQ_ERR_CAPACITY) not in ("unknown status", "")
