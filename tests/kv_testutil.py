"""A plain model of the paged key-value cache (Python lists and dictionaries) and attention in
fp64, for the tests of aq_kv_*. Shares no code with the GPU path."""
import numpy as np
import torch

UNIT = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}


class Model:
    """The cache's bookkeeping: what aq.h says each call does."""

    def __init__(self, num_pages, page_tokens, max_seqs, max_pages):
        self.page, self.W = page_tokens, max_pages
        self.refs = [0] * num_pages
        self.lens = [0] * max_seqs
        self.rows = [[] for _ in range(max_seqs)]
        self.copies = []                     # pages copied by the last call, (from, to)

    def _free(self, count):
        got = [p for p, r in enumerate(self.refs) if r == 0][:count]
        return got if len(got) == count else None

    def reserve(self, seqs, counts=None):
        counts = [1] * len(seqs) if counts is None else list(counts)
        if len(set(seqs)) < len(seqs) or any(not 0 <= s < len(self.lens) for s in seqs) or min(counts, default=0) < 0:
            return "invalid"
        if any(-(-(self.lens[s] + c) // self.page) > self.W for s, c in zip(seqs, counts)):
            return "capacity"
        need = [-(-(self.lens[s] + c) // self.page) - len(self.rows[s]) for s, c in zip(seqs, counts)]
        pages = self._free(sum(need))
        if pages is None:
            return "capacity"
        for s, c, k in zip(seqs, counts, need):
            self.rows[s] += pages[:k]
            for p in pages[:k]:
                self.refs[p] = 1
            pages = pages[k:]
            self.lens[s] += c
        return "ok"

    def fork(self, src, dst):
        bad = len(set(dst)) < len(dst) or any(not 0 <= s < len(self.lens) for s in list(src) + list(dst))
        if bad or any(self.lens[d] for d in dst):
            return "invalid"
        part = [self.lens[s] % self.page > 0 for s in src]
        pages = self._free(sum(part))
        if pages is None:
            return "capacity"
        self.copies = []
        before = [(self.lens[s], list(self.rows[s])) for s in src]
        for (n, row), d, x in zip(before, dst, part):
            if x:
                new = pages.pop(0)
                self.copies.append((row[-1], new))
                self.refs[new] = 1
                for p in row[:-1]:
                    self.refs[p] += 1
                row = row[:-1] + [new]
            else:
                for p in row:
                    self.refs[p] += 1
            self.rows[d], self.lens[d] = list(row), n
        return "ok"

    def free(self, seqs):
        for s in seqs:
            for p in self.rows[s]:
                self.refs[p] -= 1
            self.rows[s], self.lens[s] = [], 0

    def compact(self):
        used = [p for p, r in enumerate(self.refs) if r > 0]
        U = len(used)
        holes = [p for p in range(U) if self.refs[p] == 0]
        self.copies = list(zip([p for p in used if p >= U], holes))
        to = dict(self.copies)
        for a, b in self.copies:
            self.refs[b], self.refs[a] = self.refs[a], 0
        self.rows = [[to.get(p, p) for p in r] for r in self.rows]
        return U

    def assert_same(self, cache):
        assert cache.lens.tolist() == self.lens
        assert cache.refs.tolist() == self.refs
        want = [r + [-1] * (self.W - len(r)) for r in self.rows]
        assert cache.tables.tolist() == want


def values(cache, which):
    """The pool's values in fp64 (on the GPU): codes times scales for e4m3."""
    pool, scales = (cache.k, cache.k_scales) if which == "k" else (cache.v, cache.v_scales)
    t = pool.double()
    return t if scales is None else t * torch.exp2(scales.double() - 127)[..., None]


def attend_exact(cache, q, seqs, layer, scale, window):
    """(out, lse, bound on |out - exact|, bound on |lse - exact|) in fp64. The bounds follow from
    the stated arithmetic: fp32 scores (sums of head_dim products), weights rounded to 16 bits
    before the product with V, one rounding of the output."""
    n, qh, hd = q.shape
    kh, page = cache.kv_heads, cache.page_tokens
    group = qh // kh
    small = cache.dtype == torch.float8_e4m3fn
    wt = torch.float16 if small else cache.dtype
    out = torch.zeros(n, qh, hd, dtype=torch.float64, device=q.device)
    lse = torch.full((n, qh), -np.inf, dtype=torch.float64, device=q.device)
    tol, tol_lse = torch.zeros_like(out), torch.zeros_like(lse)
    lens, tables = cache.lens.tolist(), cache.tables.long()
    for i, s in enumerate(seqs):
        L = lens[s]
        lo = max(0, L - window) if window else 0
        if L == 0:
            continue
        at = tables[s, : -(-L // page)]

        def rows(pool, scales):
            t = pool[layer, at].double()
            if scales is not None:
                t = t * torch.exp2(scales[layer, at].double() - 127)[..., None]
            return t.transpose(0, 1).reshape(kh, -1, hd)[:, lo:L]

        k, v = rows(cache.k, cache.k_scales), rows(cache.v, cache.v_scales)
        qi = q[i].double().view(kh, group, hd)
        sc = qi @ k.transpose(1, 2) * scale
        mag = qi.abs() @ k.abs().transpose(1, 2) * abs(scale)
        p = torch.softmax(sc, -1)
        out[i] = (p @ v).reshape(qh, hd)
        lse[i] = torch.logsumexp(sc, -1).reshape(qh)
        # error of a score (also of its base-2 form and the exponential's argument)
        ds = (hd + 16) * 2.0 ** -23 * mag.amax(-1) + 2.0 ** -19
        if small:
            # the query's fp16 form: 2^-25 of 2^15 / (its largest element) at worst
            ds = ds + 2.0 ** -25 * 2 * 2.0 ** -14 * qi.abs().amax(-1) * (k.abs().sum(-1).amax(-1) * abs(scale))[:, None]
        A = p @ v.abs()
        # weights p 2^b / max(p 2^b) in 16 bits: relative UNIT, absolute TINY
        if small:
            b = torch.exp2(cache.v_scales[layer, at].double() - 127).transpose(0, 1).reshape(kh, -1)[:, lo:L]
            top = (p * b[:, None]).amax(-1)
            codes = (v / b[..., None]).abs().sum(1)
            small_err = 2.0 ** -24 * top[..., None] * codes[:, None]
        else:
            small_err = TINY[wt] * 2 * p.amax(-1)[..., None] * v.abs().sum(1)[:, None]
        e = UNIT[wt] * A + small_err + 2 * ds[..., None] * A
        tol[i] = (e + UNIT[q.dtype] * (out[i].view(kh, group, hd).abs() + e) + TINY[q.dtype]).reshape(qh, hd) * 1.01
        tol_lse[i] = (ds + 2.0 ** -21 * lse[i].view(kh, group).abs()).reshape(qh)
    return out, lse, tol, tol_lse


def filled_cache(cls, lens, page, kv_heads, head_dim, dtype, layers=1, seed=0, spare=3, max_pages=None,
                 v_exp=0, junk=float("nan"), num_pages=None):
    """A cache whose sequences have the given lengths, on shuffled pages; everything that no
    sequence has cached (free pages, slots past a length) holds `junk`."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = np.random.Generator(np.random.PCG64(seed))
    need = [-(-n // page) for n in lens]
    total = sum(need) + spare if num_pages is None else num_pages
    W = max(need + [1]) if max_pages is None else max_pages
    c = cls(total, page, kv_heads, head_dim, max_seqs=len(lens), max_pages=W, layers=layers, dtype=dtype)
    order = rng.permutation(total) if num_pages is None else np.arange(total)[::-1]
    tables = np.full((len(lens), W), -1, np.int32)
    refs = np.zeros(total, np.int32)
    seen = np.zeros((total, page), bool)
    at = 0
    for s, (n, k) in enumerate(zip(lens, need)):
        tables[s, :k] = order[at:at + k]
        at += k
        refs[tables[s, :k]] = 1
        for j in range(k):
            seen[tables[s, j], : min(page, n - j * page)] = True
    c.tables.copy_(torch.from_numpy(tables))
    c.refs.copy_(torch.from_numpy(refs))
    c.lens.copy_(torch.as_tensor(lens, dtype=torch.int32))
    used = np.flatnonzero(refs)
    for pool, scales in ((c.k, c.k_scales), (c.v, c.v_scales)):
        for p in used:
            hide = torch.from_numpy(~seen[p]).cuda()[None, None, :, None]
            x = torch.randn(layers, kv_heads, page, head_dim, device="cuda", generator=g)
            pool[:, p] = torch.where(hide, junk, x.clamp(-8, 8) * (40.0 if scales is not None else 1.0)).to(pool.dtype)
        free = np.flatnonzero(refs == 0)
        if num_pages is None and len(free):
            f = torch.from_numpy(free).cuda()
            pool.view(torch.uint8 if scales is not None else torch.int16)[:, f] = 0x7f if scales is not None else 0x7fff
        if scales is not None:
            scales.random_(120, 128, generator=g)
            if v_exp and scales is c.v_scales:
                scales.random_(127 - v_exp, 128 + v_exp, generator=g)
    return c
