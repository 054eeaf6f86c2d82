"""AQDecoderBlock over a paged cache against fp64: steps of a few sequences, a fork in between, the
weights those that the oracle reconstructs.

Tolerance: four product roundings (each within the product tolerance of 2e-3 relative Frobenius,
as in the GEMV tests), and about ten roundings to fp16 (2^-11 each) on the way through norm,
rotation, cache, weights of the softmax, gate and residual: 4 * 2e-3 + 10 * 2^-11 = 1.3e-2."""
import numpy as np
import pytest
import torch

import aq_testutil as U
import oracle
import workloads
from paper_2606_12876_gb300.block import AQDecoderBlock, rope_angles
from paper_2606_12876_gb300.kv import PagedKVCache
from paper_2606_12876_gb300.linear import AQLinear

pytestmark = pytest.mark.gpu
HID, QH, KH, HD, FFN, EPS = 256, 4, 2, 64, 512, 1e-5
TOL = 4 * 2e-3 + 10 * 2.0 ** -11


def make(M=3):
    shapes = {"q": (QH * HD, HID), "k": (KH * HD, HID), "v": (KH * HD, HID), "o": (HID, QH * HD),
              "gate": (FFN, HID), "up": (FFN, HID), "down": (HID, FFN)}
    lay = {n: workloads.make_layer(o, i, M=M, book_std=0.03, seed=11 + k) for k, (n, (o, i)) in enumerate(shapes.items())}
    return lay, {n: AQLinear.from_layer(v) for n, v in lay.items()}


def norm64(h, w):
    return h / np.sqrt((h * h).mean(-1, keepdims=True) + EPS) * w


def rotate64(x, pos):
    inv = 500000.0 ** (-np.arange(0, HD, 2) / HD)
    c, s = np.cos(pos * inv), np.sin(pos * inv)
    a, b = x[..., : HD // 2], x[..., HD // 2:]
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def block64(W, x, w1, w2, keys, values):
    """One token of one sequence through the block; keys, values: its lists so far (appended to)."""
    y = norm64(x, w1)
    pos = len(keys)
    q = rotate64((W["q"] @ y).reshape(QH, HD), pos)
    keys.append(rotate64((W["k"] @ y).reshape(KH, HD), pos))
    values.append((W["v"] @ y).reshape(KH, HD))
    K, V = np.stack(keys), np.stack(values)
    a = np.zeros((QH, HD))
    for h in range(QH):
        s = K[:, h // (QH // KH)] @ q[h] / np.sqrt(HD)
        p = np.exp(s - s.max())
        a[h] = p @ V[:, h // (QH // KH)] / p.sum()
    h = x + W["o"] @ a.reshape(-1)
    y = norm64(h, w2)
    g = W["gate"] @ y
    return h + W["down"] @ (g / (1 + np.exp(-g)) * (W["up"] @ y))


@pytest.mark.parametrize("cache_dtype", ["f16", "e4m3"])
def test_block_steps_match_fp64(cache_dtype):
    U.require_gpu()
    lay, lins = make()
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    w1, w2 = ((1 + 0.1 * torch.randn(HID, device="cuda", generator=g)).half() for _ in range(2))
    block = AQDecoderBlock(lins, w1, w2, QH, KH, layer=1, eps=EPS)
    cache = PagedKVCache(40, 8, KH, HD, 6, 8, layers=2, dtype=cache_dtype)
    ints = lambda v: torch.as_tensor(v, dtype=torch.int32, device="cuda")
    # an E4M3 key or value is off by up to 2^-4 of itself, about 2^-5.5 rms: checked by its own bound
    tol = TOL if cache_dtype == "f16" else TOL + 2.0 ** -5
    m = 2
    W = {n: oracle.reconstruct_exact(v, m) for n, v in lay.items()}
    hist = {s: ([], []) for s in range(6)}
    a1, a2 = U.to_f64(w1), U.to_f64(w2)

    def run(seqs):
        x = torch.randn(len(seqs), HID, device="cuda", generator=g).half()
        idx = ints(seqs)
        cache.reserve(idx)
        rope = rope_angles(cache.lens[idx.long()] - 1, HD)
        d, res = block.step(x, None, m, cache, idx, rope)
        got = U.to_f64(d) + U.to_f64(res)
        want = np.stack([block64(W, U.to_f64(x[i]), a1, a2, *hist[s]) for i, s in enumerate(seqs)])
        rel = np.linalg.norm(got - want) / np.linalg.norm(want)
        assert rel <= tol, rel

    for _ in range(11):
        run([0, 3])
    cache.fork(ints([0, 3, 0]), ints([1, 2, 4]))
    for a, b in ((0, 1), (3, 2), (0, 4)):
        hist[b] = (list(hist[a][0]), list(hist[a][1]))
    for _ in range(9):
        run([4, 0, 1, 2, 3])
    cache.free(ints([0, 2]))
    cache.compact()
    for _ in range(3):
        run([1, 4, 3])
    cache.check()


def test_block_takes_more_sequences_than_a_gemv():
    """Twenty sequences: the products go through the GEMM."""
    U.require_gpu()
    lay, lins = make(2)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    w = torch.ones(HID, device="cuda", dtype=torch.float16)
    block = AQDecoderBlock(lins, w, w, QH, KH, eps=EPS)
    cache = PagedKVCache(60, 8, KH, HD, 20, 3, dtype="f16")
    idx = torch.arange(20, dtype=torch.int32, device="cuda")
    W = {n: oracle.reconstruct_exact(v, 2) for n, v in lay.items()}
    hist = [([], []) for _ in range(20)]
    for _ in range(3):
        x = torch.randn(20, HID, device="cuda", generator=g).half()
        cache.reserve(idx)
        d, res = block.step(x, None, 2, cache, idx, rope_angles(cache.lens - 1, HD))
        want = np.stack([block64(W, U.to_f64(x[i]), np.ones(HID), np.ones(HID), *hist[i]) for i in range(20)])
        got = U.to_f64(d) + U.to_f64(res)
        assert np.linalg.norm(got - want) / np.linalg.norm(want) <= TOL
    cache.check()
