"""Cases for the operators around the codebook products in decoding: attention of new tokens over
a paged key-value cache, writing keys and values into it, management of its pages, and the RMS
norm with residual. Each case runs in a plain form (elementary torch operations in fp32) or,
where `own` is true, through this package."""
import math
import random

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
E4M3_MAX = 448.0
SCALE_EXP = 60          # exponents of the power-of-two scales of 8-bit values stay in [-60, 60]


# ------------------------------------------------------------------------------------ the cases

def listed():
    return [
        # One user's chat on the 8B model's head layout, a short context: latency is what counts.
        dict(name="attend-short", kind="attend", n=1, len_min=333, len_max=333, q_heads=32,
             kv_heads=8, head_dim=128, page=16, dtype="bf16", window=0, empty=0),
        # An ordinary serving batch with contexts of all lengths, one slot idle (length zero).
        dict(name="attend-ragged", kind="attend", n=64, len_min=17, len_max=2048, q_heads=32,
             kv_heads=8, head_dim=128, page=64, dtype="bf16", window=0, empty=1),
        # One long document: the split over the length has to fill the GPU.
        dict(name="attend-long", kind="attend", n=1, len_min=131071, len_max=131071, q_heads=32,
             kv_heads=8, head_dim=128, page=64, dtype="f16", window=0, empty=0),
        # The 70B model's head layout over an 8-bit cache, medium contexts.
        dict(name="attend-8bit", kind="attend", n=32, len_min=1000, len_max=16384, q_heads=64,
             kv_heads=8, head_dim=128, page=32, dtype="e4m3", window=0, empty=0),
        # A full server: long contexts in a large batch, the cache's bytes are what counts.
        dict(name="attend-full", kind="attend", n=48, len_min=8192, len_max=32768, q_heads=32,
             kv_heads=8, head_dim=128, page=64, dtype="bf16", window=0, empty=0),
        # The norm in front of a projection for one decoded token of the 8B model.
        dict(name="norm-token", kind="norm", rows=1, cols=4096, x="bf16", res="bf16", y="bf16",
             block=0),
        # The norm in the 70B model's prefill of 4096 tokens.
        dict(name="norm-prefill", kind="norm", rows=4096, cols=8192, x="bf16", res="bf16", y="bf16",
             block=0),
        # Prefill of an odd number of tokens with the 8-bit output in blocks of 32.
        dict(name="norm-8bit", kind="norm", rows=2047, cols=4096, x="bf16", res="f32", y="e4m3",
             block=32),
        # A decode step of 64 sequences: one new key and value per sequence and head.
        dict(name="write-step", kind="write", n=64, new=1, len_min=100, len_max=1000, kv_heads=8,
             head_dim=128, page=64, x="bf16", dtype="bf16"),
        # Prompts of several users written into an 8-bit cache.
        dict(name="write-prompt", kind="write", n=4, new=2047, len_min=2047, len_max=2500,
             kv_heads=8, head_dim=128, page=64, x="bf16", dtype="e4m3"),
        # A beam-search step: the losing beams are dropped, the winners forked, one token each.
        dict(name="pages-beam", kind="fork", parents=8, children=32, len_min=900, len_max=1100,
             layers=4, kv_heads=8, head_dim=128, page=16, dtype="bf16"),
        # A pool after hours of traffic: its pages are moved together so that the tail is free.
        dict(name="pages-compact", kind="compact", n=24, pages=4096, used=2400, moves=1000,
             shared=40, layers=1, kv_heads=8, head_dim=128, page=64, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    v = max(lo, min(hi, v))
    return v + 1 if v == 3 << 10 else v


HEADS = [(32, 8, 128), (64, 8, 128), (16, 16, 64), (12, 1, 128), (20, 4, 80), (40, 2, 96),
         (8, 2, 256), (28, 1, 64)]


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "norm", "norm", "write", "fork", "compact"])
    qh, kh, hd = rng.choice(HEADS)
    if kind == "attend":
        dtype = rng.choice(["f16", "bf16", "bf16", "e4m3"])
        n = _log(rng, 1, 256)
        per_token = kh * hd * 2 * (1 if dtype == "e4m3" else 2)
        # the padded plain form holds n * len_max tokens in fp32; both stay below the largest case
        most = min(131072, int(3.0e9 / (per_token * n)), int(5.0e9 / (4 * kh * hd * n)))
        hi = _log(rng, 1, max(1, most))
        lo = _log(rng, 1, hi)
        return dict(kind=kind, n=n, len_min=min(lo, hi), len_max=hi, q_heads=qh, kv_heads=kh,
                    head_dim=hd, page=rng.choice([16, 32, 64, 128]), dtype=dtype,
                    window=rng.choice([0, 0, 0, _log(rng, 1, hi)]),
                    empty=rng.choice([0, 1]) if n > 1 else 0)
    if kind == "norm":
        cols = 32 * _log(rng, 2, 448)
        cols += 32 if cols == 3 << 10 else 0
        y = rng.choice(["f16", "bf16", "f32", "e4m3"])
        x = rng.choice(["f16", "bf16", "f32"])
        return dict(kind=kind, rows=_log(rng, 1, max(1, 33554432 // cols)), cols=cols, x=x,
                    res=rng.choice(["none", x, "f32"]), y=y,
                    block=rng.choice([0, 32]) if y == "e4m3" else 0)
    if kind == "write":
        n = _log(rng, 1, 64)
        new = rng.choice([1, _log(rng, 1, max(1, 8192 // n))])
        lo = new + _log(rng, 1, 300) - 1
        return dict(kind=kind, n=n, new=new, len_min=lo, len_max=lo + _log(rng, 1, 500),
                    kv_heads=kh, head_dim=hd, page=rng.choice([16, 32, 64, 128]),
                    x=rng.choice(["f16", "bf16", "f32"]), dtype=rng.choice(["f16", "bf16", "e4m3"]))
    if kind == "fork":
        parents = _log(rng, 1, 16)
        lo = _log(rng, 1, 1500)
        return dict(kind=kind, parents=parents, children=parents * rng.randint(1, 8), len_min=lo,
                    len_max=lo + _log(rng, 1, 200), layers=rng.choice([1, 2, 4]), kv_heads=kh,
                    head_dim=hd, page=rng.choice([16, 32, 64]), dtype=rng.choice(["f16", "bf16"]))
    pages = _log(rng, 64, 4000)
    used = max(2, pages * rng.randint(20, 70) // 100)
    page = rng.choice([16, 32, 64])
    return dict(kind=kind, n=rng.randint(1, 32), pages=pages, used=used,
                moves=rng.randint(1, max(1, min(used, pages - used) // 2)), shared=rng.randint(0, used // 4),
                layers=1, kv_heads=min(kh, 8), head_dim=min(hd, 128), page=page,
                dtype=rng.choice(["f16", "bf16"]))


def _lengths(case, n):
    """n lengths spread evenly over the logarithm from len_min to len_max, the first one zero where
    the case has an idle slot; the same for every seed but for their order."""
    lo, hi = case["len_min"], case["len_max"]
    got = [int(round(lo * (hi / lo) ** ((i + 1) / n))) for i in range(n)]
    got = [v + 1 if v == 3 << 10 else v for v in got]
    if case.get("empty"):
        got[0] = 0
    return got


# ---------------------------------------------------------------------------------- the inputs

def _esz(dtype):
    return 1 if dtype == "e4m3" else 4 if dtype == "f32" else 2


def _exponent(amax):
    """The smallest e with amax <= 448 * 2^e, kept in the scales' range."""
    mant, ex = torch.frexp(amax)
    return (ex - 9 + (mant > E4M3_MAX / 512).int()).clamp(-SCALE_EXP, SCALE_EXP)


def _quantise(x):
    """Codes (E4M3) and scale bytes of fp32 x, one power-of-two scale along the last axis."""
    e = _exponent(x.abs().amax(-1))
    codes = torch.ldexp(x, -e[..., None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return codes, (e + 127).to(torch.uint8)


def _scale_values(s, dtype):
    return s.view(torch.float8_e8m0fnu).to(dtype)


def _normal(shape, dtype, g):
    return torch.randn(shape, dtype=dtype, device="cuda", generator=g)


def _pool(case, layers, pages, g):
    """Keys or values of a pool: unit-scale, with some channels a few times larger, as keys have."""
    kh, hd, page = case["kv_heads"], case["head_dim"], case["page"]
    dt = DTYPES.get(case["dtype"], torch.bfloat16)
    t = _normal((layers, pages, kh, page, hd), dt, g)
    t[..., ::17] *= 3
    if case["dtype"] == "e4m3":
        return _quantise(t.float())
    return t, None


def _state(case, g, layers, pages, tables, lens, refs):
    k, ks = _pool(case, layers, pages, g)
    v, vs = _pool(case, layers, pages, g)
    s = dict(case=case, k=k, v=v, ks=ks, vs=vs, tables=tables, lens=lens, refs=refs)
    if own:
        from paper_2606_12876_gb300.kv import PagedKVCache
        s["cache"] = PagedKVCache.from_tensors(k, v, tables, lens, refs, k_scales=ks, v_scales=vs)
    return s


def _tables(rows, width):
    t = torch.full((len(rows), width), -1, dtype=torch.int32)
    for i, r in enumerate(rows):
        t[i, :len(r)] = torch.as_tensor(r, dtype=torch.int32)
    return t.cuda()


def _ints(v):
    return torch.as_tensor(v, dtype=torch.int32).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rng = random.Random(seed)
    kind = case["kind"]
    if kind == "norm":
        rows, cols = case["rows"], case["cols"]
        s = dict(case=case, x=_normal((rows, cols), DTYPES[case["x"]], g),
                 w=(1 + 0.1 * _normal((cols,), torch.float32, g)).to(torch.bfloat16), eps=1e-5)
        s["r"] = None if case["res"] == "none" else _normal((rows, cols), DTYPES[case["res"]], g) * 2
        return s
    page = case["page"]
    if kind in ("attend", "write"):
        lens = _lengths(case, case["n"])
        rng.shuffle(lens)
        need = [-(-v // page) for v in lens]
        pages = sum(need) + sum(need) // 8 + 1
        order = list(range(pages))
        rng.shuffle(order)
        rows, at = [], 0
        for v in need:
            rows.append(order[at:at + v])
            at += v
        refs = torch.zeros(pages, dtype=torch.int32)
        refs[order[:at]] = 1
        s = _state(case, g, 1, pages, _tables(rows, max(need + [1])), _ints(lens), refs.cuda())
        kh, hd = case["kv_heads"], case["head_dim"]
        if kind == "attend":
            dt = torch.bfloat16 if case["dtype"] == "e4m3" else DTYPES[case["dtype"]]
            s["q"] = _normal((case["n"], case["q_heads"], hd), dt, g) * 2
            s["scale"] = hd ** -0.5
        else:
            n, new = case["n"], case["new"]
            s["seqs"] = _ints([i for i in range(n) for _ in range(new)])
            s["pos"] = _ints([lens[i] - new + j for i in range(n) for j in range(new)])
            s["new_k"] = _normal((n * new, kh, hd), DTYPES[case["x"]], g) * 3
            s["new_v"] = _normal((n * new, kh, hd), DTYPES[case["x"]], g)
        return s
    if kind == "fork":
        np_, nc = case["parents"], case["children"]
        lens = _lengths(case, np_)
        rng.shuffle(lens)
        need = [-(-v // page) for v in lens]
        pages = sum(need) + 2 * nc + 8
        order = list(range(pages))
        rng.shuffle(order)
        rows, at = [], 0
        for v in need:
            rows.append(order[at:at + v])
            at += v
        refs = torch.zeros(pages, dtype=torch.int32)
        refs[order[:at]] = 1
        s = _state(case, g, case["layers"], pages, _tables(rows + [[]] * nc, max(need) + 1),
                   _ints(lens + [0] * nc), refs.cuda())
        s["src"] = _ints([rng.randrange(np_) for _ in range(nc)])
        s["dst"] = _ints(range(np_, np_ + nc))
        return s
    # compact: `used` pages, `moves` of them at indices from `used` on; every sequence starts with
    # the `shared` pages of a common prompt
    n, pages, used, moves = case["n"], case["pages"], case["used"], case["moves"]
    inside = rng.sample(range(used), used - moves) + rng.sample(range(used, pages), moves)
    rng.shuffle(inside)
    common, rest = inside[:case["shared"]], inside[case["shared"]:]
    rows = [common + rest[i::n] for i in range(n)]
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[common] = n
    refs[rest] = 1
    s = _state(case, g, case["layers"], pages, _tables(rows, max(len(r) for r in rows)),
               _ints([len(r) * page - (rng.randrange(page) if len(r) > len(common) else 0) for r in rows]),
               refs.cuda())
    s["tables0"], s["refs0"] = s["tables"].clone(), s["refs"].clone()
    return s


# -------------------------------------------------------------------------------- the operators

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        from paper_2606_12876_gb300.norm import rmsnorm, rmsnorm_8bit
        if case["y"] == "e4m3":
            y, sc, h = rmsnorm_8bit(s["x"], s["w"], s["eps"], residual=s["r"], block=case["block"])
            return _values_8bit(y, sc), h
        return rmsnorm(s["x"], s["w"], s["eps"], residual=s["r"], y_dtype=DTYPES[case["y"]])
    cache = s["cache"]
    if kind == "attend":
        return cache.attend(s["q"], scale=s["scale"], window=case["window"])
    if kind == "write":
        cache.write(s["new_k"], s["new_v"], s["seqs"], s["pos"])
        return _pool_values(s)
    if kind == "fork":
        cache.free(s["dst"])
        cache.fork(s["src"], s["dst"])
        cache.reserve(s["dst"])
        return s["tables"], s["lens"], s["refs"], s["k"], s["v"]
    s["tables"].copy_(s["tables0"])
    s["refs"].copy_(s["refs0"])
    cache.compact()
    return s["tables"], s["refs"], s["k"], s["v"]


def _values_8bit(y, sc):
    """The values that E4M3 codes and power-of-two scales stand for: exact in bf16."""
    v = y.to(torch.bfloat16)
    return v.view(*sc.shape, -1).mul_(_scale_values(sc, torch.bfloat16)[..., None]).view(y.shape)


def _pool_values(s):
    if s["ks"] is None:
        return s["k"], s["v"]
    return _values_8bit(s["k"], s["ks"]), _values_8bit(s["v"], s["vs"])


def _run_plain(s):
    return {"norm": _plain_norm, "attend": _plain_attend, "write": _plain_write,
            "fork": _plain_fork, "compact": _plain_compact}[s["case"]["kind"]](s)


def _plain_norm(s):
    case = s["case"]
    h = s["x"].float()
    if s["r"] is not None:
        h = h + s["r"].float()
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + s["eps"]) * s["w"].float()
    kept = None if s["r"] is None else h.to(s["r"].dtype)
    if case["y"] == "e4m3":
        b = y.view(y.shape[0], -1, case["block"] or y.shape[1])
        e = _exponent(b.abs().amax(-1, keepdim=True))
        codes = torch.ldexp(b, -e).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        return torch.ldexp(codes.float(), e).view(y.shape).to(torch.bfloat16), kept
    return y.to(DTYPES[case["y"]]), kept


def _gathered(pool, scales, tables):
    """[n][kv_heads][width * page][head_dim] in fp32: every sequence's pages in order."""
    idx = tables.clamp(min=0).long()
    t = pool[0][idx].float()
    if scales is not None:
        t = t * _scale_values(scales[0][idx], torch.float32)[..., None]
    n, w, kh, page, hd = t.shape
    return t.permute(0, 2, 1, 3, 4).reshape(n, kh, w * page, hd)


def _plain_attend(s):
    case, q = s["case"], s["q"]
    n, qh, hd = q.shape
    k = _gathered(s["k"], s["ks"], s["tables"])
    sc = q.float().view(n, k.shape[1], -1, hd) @ k.transpose(2, 3) * s["scale"]
    pos = torch.arange(k.shape[2], device="cuda", dtype=torch.int32)[None]
    del k
    seen = pos < s["lens"][:, None]
    if case["window"]:
        seen &= pos >= s["lens"][:, None] - case["window"]
    sc.masked_fill_(~seen[:, None, None], -math.inf)
    top = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - torch.where(torch.isinf(top), 0.0, top))
    total = p.sum(-1, keepdim=True)
    o = p @ _gathered(s["v"], s["vs"], s["tables"])
    o = torch.where(total > 0, o / total, 0.0)
    return o.view(n, qh, hd).to(q.dtype)


def _plain_write(s):
    page = s["case"]["page"]
    pos, seqs = s["pos"].long(), s["seqs"].long()
    at, slot = s["tables"][seqs, pos // page].long(), pos % page
    for pool, scales, new in ((s["k"], s["ks"], s["new_k"]), (s["v"], s["vs"], s["new_v"])):
        if scales is None:
            pool[0, at, :, slot] = new.to(pool.dtype)
        else:
            codes, e = _quantise(new.float())
            pool.view(torch.uint8)[0, at, :, slot] = codes.view(torch.uint8)
            scales[0, at, :, slot] = e
    return _pool_values(s)


def _plain_free(s, seqs):
    refs, tables = s["refs"], s["tables"]
    row = tables[seqs]
    refs.index_add_(0, row.clamp(min=0).flatten().long(), -(row >= 0).int().flatten())
    tables[seqs] = -1
    s["lens"][seqs] = 0


def _lowest_free(refs, count):
    """The `count` lowest free pages, in order."""
    return torch.sort((refs > 0).int(), stable=True).indices[:count].int()


def _plain_fork(s):
    refs, tables, lens, page = s["refs"], s["tables"], s["lens"], s["case"]["page"]
    src, dst = s["src"].long(), s["dst"].long()
    _plain_free(s, dst)
    # fork: full pages are shared, a partial last page is copied to a new one
    n = lens[src]
    part = n % page > 0
    last = (n // page).long()
    rank = (torch.cumsum(part.int(), 0) - 1).clamp(min=0)
    row = tables[src]
    old = row.gather(1, last[:, None].clamp(max=row.shape[1] - 1))[:, 0]
    new = torch.where(part, _lowest_free(refs, len(dst))[rank], old)
    row.scatter_(1, last[:, None], new[:, None])
    refs.index_add_(0, row.clamp(min=0).flatten().long(), (row >= 0).int().flatten())
    tables[dst] = row
    lens[dst] = n
    to, frm = torch.where(part, new, row[:, 0]).long(), torch.where(part, old, row[:, 0]).long()
    for pool in (s["k"], s["v"]):
        pool[:, to] = pool[:, frm]
    # reserve: one more token each, a new page where the last one is full
    grow = lens[dst] % page == 0
    rank = (torch.cumsum(grow.int(), 0) - 1).clamp(min=0)
    free = _lowest_free(refs, len(dst))[rank]
    last = (lens[dst] // page).long()
    tables[dst, last] = torch.where(grow, free, tables[dst, last])
    refs.index_add_(0, free.long(), grow.int())
    lens[dst] += 1
    return s["tables"], s["lens"], s["refs"], s["k"], s["v"]


def _plain_compact(s):
    refs, tables = s["refs"], s["tables"]
    tables.copy_(s["tables0"])
    refs.copy_(s["refs0"])
    used = refs > 0
    below = torch.arange(refs.numel(), device="cuda") < used.sum()
    frm = (used & ~below).nonzero()[:, 0]
    to = (~used & below).nonzero()[:, 0]
    for pool in (s["k"], s["v"]):
        pool[:, to] = pool[:, frm]
    moved = torch.arange(refs.numel(), device="cuda", dtype=torch.int32)
    moved[frm] = to.int()
    tables.copy_(torch.where(tables >= 0, moved[tables.clamp(min=0).long()], tables))
    refs[to] = refs[frm]
    refs[frm] = 0
    return s["tables"], s["refs"], s["k"], s["v"]


# --------------------------------------------------------------------------- in 64 bits, and work

def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    kind = case["kind"]
    if kind == "norm":
        h = s["x"].double() if s["r"] is None else s["x"].double() + s["r"].double()
        y = torch.einsum("rc,c->rc", h / (h.square().sum(1, keepdim=True) / h.shape[1] + s["eps"]).sqrt(),
                         s["w"].double())
        if case["y"] == "e4m3":
            y = _exact_8bit(y, case["block"] or y.shape[1])
        return y, None if s["r"] is None else h
    if kind == "attend":
        return _exact_attend(s)
    if kind == "write":
        out = []
        for pool, scales, new in ((s["k"], s["ks"], s["new_k"]), (s["v"], s["vs"], s["new_v"])):
            t = pool.double()
            if scales is not None:
                t = t * torch.exp2(scales.double() - 127)[..., None]
                new = _exact_8bit(new.double(), new.shape[-1])
            where = s["tables"][s["seqs"].long(), torch.div(s["pos"], case["page"], rounding_mode="floor").long()]
            t.transpose(2, 3)[0][where.long(), s["pos"].long() % case["page"]] = new.double()
            out.append(t)
        return tuple(out)
    return None


def _exact_8bit(y, block):
    """64-bit values rounded to E4M3 with a power-of-two scale per block: steps of 2^(e - 3) in the
    binade of 2^e, none finer than 2^-9, at the scale."""
    b = y.reshape(-1, block)
    e = torch.ceil(torch.log2(b.abs().amax(1, keepdim=True).clamp(min=1e-300) / E4M3_MAX)).clamp(-SCALE_EXP, SCALE_EXP)
    z = b * torch.exp2(-e)
    step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(z / step) * step * torch.exp2(e)).reshape(y.shape)


def _exact_attend(s):
    case, q, page = s["case"], s["q"].double(), s["case"]["page"]
    n, qh, hd = q.shape
    kh = case["kv_heads"]
    out = torch.zeros_like(q)
    lens, tables = s["lens"].tolist(), s["tables"].long()
    for i in range(n):
        if not lens[i]:
            continue
        lo = max(0, lens[i] - case["window"]) if case["window"] else 0
        at = tables[i, : -(-lens[i] // page)]
        kv = []
        for pool, scales in ((s["k"], s["ks"]), (s["v"], s["vs"])):
            t = pool[0][at].double()
            if scales is not None:
                t = t * torch.exp2(scales[0][at].double() - 127)[..., None]
            kv.append(t.transpose(0, 1).reshape(kh, -1, hd)[:, lo:lens[i]])
        w = torch.einsum("hgd,htd->hgt", q[i].view(kh, -1, hd), kv[0]) * s["scale"]
        out[i] = torch.einsum("hgt,htd->hgd", torch.softmax(w, -1), kv[1]).reshape(qh, hd)
    return out


def work(case):
    kind = case["kind"]
    if kind == "norm":
        n = case["rows"] * case["cols"]
        per = _esz(case["x"]) + _esz(case["y"])
        per += 0 if case["res"] == "none" else 2 * _esz(case["res"])
        return {"bytes": n * per + 2 * case["cols"], "flops": 6 * n}
    kh, hd, page = case["kv_heads"], case["head_dim"], case["page"]
    esz = _esz(case["dtype"])
    row = hd * esz + (1 if case["dtype"] == "e4m3" else 0)      # one token of one head
    if kind == "attend":
        lens = _lengths(case, case["n"])
        seen = sum(min(v, case["window"]) if case["window"] else v for v in lens)
        return {"bytes": 2 * seen * kh * row + 2 * case["n"] * case["q_heads"] * hd * 2,
                "flops": 4 * seen * case["q_heads"] * hd}
    if kind == "write":
        rows = case["n"] * case["new"] * kh * 2
        return {"bytes": rows * (hd * _esz(case["x"]) + row), "flops": rows * hd}
    one = 2 * case["layers"] * kh * page * row                    # a page's keys and values
    if kind == "fork":
        lens = _lengths(case, case["parents"])
        part = sum(v % page > 0 for v in lens) / len(lens)
        entries = case["children"] * sum(-(-v // page) for v in lens) / len(lens)
        return {"bytes": 2 * one * part * case["children"] + 16 * entries, "flops": 0}
    return {"bytes": 2 * one * case["moves"] + 8 * case["pages"], "flops": 0}
