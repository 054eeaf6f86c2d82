"""RMS norm with the residual's addition (aq_rmsnorm of libaq), 16/32-bit or 8-bit output."""
import torch

from . import AQ_BF16, AQ_E4M3, AQ_F16, AQ_F32, aq_rmsnorm

_CODES = {torch.float16: AQ_F16, torch.bfloat16: AQ_BF16, torch.float32: AQ_F32}


def _args(x, weight, residual, residual_out):
    if x.dim() != 2 or (x.stride(1) != 1 and x.shape[1] > 1):
        raise ValueError("x must be [rows][cols] with contiguous rows")
    rows, cols = x.shape
    if weight.shape != (cols,) or not weight.is_contiguous() or weight.device != x.device:
        raise ValueError("weight must be a contiguous [%d] tensor on x's device" % cols)
    for t in (residual, residual_out):
        if t is not None and (t.shape != x.shape or not t.is_contiguous() or t.device != x.device):
            raise ValueError("the residual must be contiguous, of x's shape and on its device")
    if not x.is_cuda:
        raise ValueError("x must be a CUDA tensor")
    if residual is not None:
        if residual_out is None:
            residual_out = torch.empty_like(residual)
        elif residual_out.dtype != residual.dtype:
            raise ValueError("residual_out must have the residual's dtype")
    for t in (x, weight, residual if residual is not None else residual_out):
        if t is not None and t.dtype not in _CODES:
            raise TypeError("unsupported dtype %s" % t.dtype)
    r = residual_out
    return (rows, cols, x, _CODES[x.dtype], x.stride(0) if rows > 1 else cols, residual, r,
            AQ_F32 if r is None else _CODES[r.dtype], weight, _CODES[weight.dtype])


def rmsnorm(x, weight, eps=1e-5, residual=None, residual_out=None, y_dtype=None, y=None):
    """h = x + residual and y = weight * h / sqrt(mean(h^2) + eps) for each row of x ([rows][cols],
    rows may be strided). Returns (y, h): y of y_dtype (x's by default), h of the residual's dtype
    (into residual_out where given, which may be the residual itself), or None without one."""
    a = _args(x, weight, residual, residual_out)
    if y is None:
        y = torch.empty(x.shape, dtype=x.dtype if y_dtype is None else y_dtype, device=x.device)
    elif y.shape != x.shape or not y.is_contiguous() or y.device != x.device:
        raise ValueError("y must be contiguous, of x's shape and on its device")
    if y.dtype not in _CODES:
        raise TypeError("unsupported output dtype %s" % y.dtype)
    aq_rmsnorm(*a, eps, y, _CODES[y.dtype], None, 0)
    return y, a[6]


def rmsnorm_8bit(x, weight, eps=1e-5, residual=None, residual_out=None, block=32):
    """As rmsnorm with y in 8 bits: returns (codes, scales, h), codes float8_e4m3fn [rows][cols],
    scales uint8 [rows][cols / block] (value = code * 2^(scale - 127), exact in bf16; a uint8
    scale viewed as float8_e8m0fnu is its power of two). block: 32 columns, or 0 for one scale
    per row."""
    a = _args(x, weight, residual, residual_out)
    rows, cols = x.shape
    block = block or cols
    if cols % block:
        raise ValueError("cols must be a multiple of the block")
    codes = torch.empty((rows, cols), dtype=torch.float8_e4m3fn, device=x.device)
    scales = torch.empty((rows, cols // block), dtype=torch.uint8, device=x.device)
    aq_rmsnorm(*a, eps, codes, AQ_E4M3, scales, block)
    return codes, scales, a[6]
