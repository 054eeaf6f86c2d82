"""RMS norm with residual (aq_rmsnorm) against fp64. Bounds: the fp32 evaluation of y is within a
few 2^-24 of each factor (the sum of squares adds at most 64 + 10 roundings of positive terms):
2^-17 relative covers it; each output adds one rounding of its type."""
import pytest
import torch

import aq_testutil as U
import kv_testutil as K
from paper_2606_12876_gb300.norm import rmsnorm, rmsnorm_8bit

pytestmark = pytest.mark.gpu
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
REL = 2.0 ** -17


def make(rows, cols, xd, rd, wd, seed=0, gain=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = (torch.randn(rows, cols, device="cuda", generator=g) * gain).to(xd)
    r = None if rd is None else (torch.randn(rows, cols, device="cuda", generator=g) * gain).to(rd)
    w = (1 + 0.2 * torch.randn(cols, device="cuda", generator=g)).to(wd)
    return x, r, w


def exact(x, r, w, eps):
    h = x.double() if r is None else x.double() + r.double()
    return h, h / (h.square().mean(1, keepdim=True) + eps).sqrt() * w.double()


def near(got, ref, dtype, rel=REL):
    bound = ref.abs() * (rel + K.UNIT[dtype] * (1 + rel)) + K.TINY[dtype]
    bad = (got.double() - ref).abs() > bound
    assert not bool(bad.any()), "%d of %d outside" % (int(bad.sum()), bad.numel())


CASES = [  # rows, cols, x, residual, weight, y
    (1, 8, BF16, None, BF16, BF16), (1, 4096, BF16, BF16, BF16, BF16), (3, 264, F16, F16, F32, F16),
    (7, 1000, F32, F32, F32, F32), (1, 65536, BF16, F32, F16, BF16), (5, 32776, F16, None, F16, F32),
    (1000, 128, BF16, BF16, BF16, BF16), (2049, 64, F16, F32, F16, F16), (777, 520, F32, BF16, BF16, F16),
    (600, 4096, BF16, BF16, F32, BF16), (401, 14336, BF16, F32, BF16, BF16), (16, 8192, F16, F16, BF16, F32),
    (333, 2056, BF16, None, BF16, BF16), (310, 65528, BF16, BF16, BF16, BF16),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v).replace("torch.", "") for v in c))
def test_rmsnorm(case):
    U.require_gpu()
    rows, cols, xd, rd, wd, yd = case
    x, r, w = make(rows, cols, xd, rd, wd, seed=rows + cols)
    y, h = rmsnorm(x, w, 1e-5, residual=r, y_dtype=yd)
    rh, ry = exact(x, r, w, 1e-5)
    near(y, ry, yd)
    if r is None:
        assert h is None
    else:
        near(h, rh, rd, 2.0 ** -24)
    again, _ = rmsnorm(x, w, 1e-5, residual=r, y_dtype=yd)
    assert torch.equal(y, again)


def test_in_place_and_strided_rows():
    U.require_gpu()
    x, r, w = make(40, 512, BF16, BF16, BF16, seed=1)
    rh, ry = exact(x, r, w, 1e-6)
    res = r.clone()
    y, h = rmsnorm(x, w, 1e-6, residual=res, residual_out=res)
    assert h is res
    near(res, rh, BF16, 2.0 ** -24)
    near(y, ry, BF16)
    same = x.clone()
    y2, h2 = rmsnorm(same, w, 1e-6, residual=r, y=same)
    assert y2 is same and torch.equal(same, y) and torch.equal(h2, h)
    wide = torch.zeros(40, 1024, dtype=BF16, device="cuda")
    wide[:, 512:] = x
    y3, _ = rmsnorm(wide[:, 512:], w, 1e-6, residual=r)
    assert torch.equal(y3, y)
    _, kept = rmsnorm(x, w, 1e-6, residual_out=torch.empty_like(r))
    assert torch.equal(kept, x)                                  # without a residual: h = x


@pytest.mark.parametrize("gain", [0.0, 1e-18, 1e-3, 3e4, 1e16])
def test_magnitudes(gain):
    """Zero rows, rows whose squares underflow, and large ones."""
    U.require_gpu()
    x, r, w = make(5, 256, F32, F32, F32, seed=2, gain=gain)
    y, _ = rmsnorm(x, w, 1e-5, residual=r)
    _, ry = exact(x, r, w, 1e-5)
    near(y, ry, F32, 2.0 ** -17 if gain >= 1e-3 or gain == 0 else 2.0 ** -16)


def test_nan_and_infinity_stay_in_their_row():
    U.require_gpu()
    x, r, w = make(9, 1024, BF16, BF16, BF16, seed=3)
    want, _ = rmsnorm(x, w, 1e-5, residual=r)
    x[4, 17] = float("nan")
    x[6, 5] = float("inf")
    y, _ = rmsnorm(x, w, 1e-5, residual=r)
    keep = [0, 1, 2, 3, 5, 7, 8]
    assert torch.equal(y[keep], want[keep])
    assert bool(torch.isnan(y[4]).all()) and bool(torch.isnan(y[6, 5]))


@pytest.mark.parametrize("rows,cols,block,xd,rd", [(1, 32, 32, BF16, None), (1, 4096, 32, BF16, BF16),
                                                   (301, 4128, 32, F16, F32), (7, 136, 0, F32, None),
                                                   (900, 128, 0, BF16, BF16), (333, 8192, 0, BF16, F32),
                                                   (2, 65536, 32, BF16, BF16), (2, 65536, 0, BF16, BF16)])
def test_8bit_output(rows, cols, block, xd, rd):
    U.require_gpu()
    x, r, w = make(rows, cols, xd, rd, BF16, seed=rows + cols)
    if rows > 2:
        x[1] = 0
        if r is not None:
            r[1] = 0
    q, s, h = rmsnorm_8bit(x, w, 1e-5, residual=r, block=block)
    rh, ry = exact(x, r, w, 1e-5)
    nb = block or cols
    assert q.dtype == torch.float8_e4m3fn and s.shape == (rows, cols // nb) and s.dtype == torch.uint8
    if r is not None:
        near(h, rh, rd, 2.0 ** -24)
    b = ry.view(rows, -1, nb)
    amax = b.abs().amax(-1)
    scale = torch.exp2(s.double() - 127)
    low = s == 127 - 60
    # the smallest exponent that holds the block, up to the fp32 error of its maximum
    assert bool((amax * (1 - REL) <= 448 * scale).all())
    assert bool((amax * (1 + REL) > 224 * scale)[~low].all())
    z = q.double().view(rows, -1, nb) * scale[..., None]
    bound = b.abs() * (2.0 ** -4 + 2 * REL) + 2.0 ** -10 * scale[..., None]
    assert bool(((z - b).abs() <= bound).all())
    half = torch.equal(s.view(torch.float8_e8m0fnu).float().double(), scale)
    assert half


def test_refusals():
    U.require_gpu()
    x, r, w = make(4, 64, BF16, BF16, BF16)
    bad = [lambda: rmsnorm(x[:, :60], w[:60]), lambda: rmsnorm(x, w[:32]), lambda: rmsnorm(x.double(), w),
           lambda: rmsnorm(x, w, residual=r[:3]), lambda: rmsnorm(x, w, residual=r, residual_out=r.float()),
           lambda: rmsnorm(x, w, -1.0), lambda: rmsnorm(x, w, float("nan")), lambda: rmsnorm(x.t(), w[:4]),
           lambda: rmsnorm(x, w, y_dtype=torch.float64), lambda: rmsnorm(x.cpu(), w.cpu()),
           lambda: rmsnorm_8bit(x[:, :40].contiguous(), w[:40]), lambda: rmsnorm_8bit(x, w, block=16),
           lambda: rmsnorm(x[:, 4:60], w[4:60].contiguous()),
           lambda: rmsnorm(torch.zeros(1, 65544, device="cuda"), torch.ones(65544, device="cuda"))]
    for f in bad:
        with pytest.raises((TypeError, ValueError, RuntimeError)):
            f()
    y, h = rmsnorm(x[:0], w, residual=r[:0])
    assert y.shape == (0, 64) and h.shape == (0, 64)
