"""RMS norm with the residual's addition (aq_rmsnorm of libaq), 16/32-bit or 8-bit output."""
import torch

from . import AQ_BF16, AQ_E4M3, AQ_F16, AQ_F32, AQError, aq_rmsnorm, _stream_of

_CODES = {torch.float16: AQ_F16, torch.bfloat16: AQ_BF16, torch.float32: AQ_F32}


def _norm(x, weight, eps, residual, residual_out, y, y_code, scales, block):
    # The checks and the call; returns the tensor that received h, or None.
    shape = x.shape
    rows, cols = shape
    x_stride, one = x.stride()
    index = x.get_device()
    if (one != 1 and cols > 1) or index < 0:
        raise ValueError("x must be a CUDA tensor [rows][cols] with contiguous rows")
    if weight.shape != (cols,) or not weight.is_contiguous() or weight.get_device() != index:
        raise ValueError("weight must be a contiguous [%d] tensor on x's device" % cols)
    r, r_out, r_code = None, None, AQ_F32
    try:
        x_code, w_code = _CODES[x.dtype], _CODES[weight.dtype]
        if residual is not None:
            if residual.shape != shape or not residual.is_contiguous() or residual.get_device() != index:
                raise ValueError("the residual must be contiguous, of x's shape and on its device")
            r, r_code = residual.data_ptr(), _CODES[residual.dtype]
            if residual_out is None:
                residual_out = torch.empty_like(residual)
                r_out = residual_out.data_ptr()
        if residual_out is not None and r_out is None:
            if residual_out.shape != shape or not residual_out.is_contiguous() or \
                    residual_out.get_device() != index:
                raise ValueError("residual_out must be contiguous, of x's shape and on its device")
            r_out = residual_out.data_ptr()
            if residual is None:
                r_code = _CODES[residual_out.dtype]
            elif residual_out.dtype != residual.dtype:
                raise ValueError("residual_out must have the residual's dtype")
    except KeyError as e:
        raise TypeError("unsupported dtype %s" % e.args[0]) from None
    status = aq_rmsnorm(rows, cols, x.data_ptr(), x_code, x_stride if rows > 1 else cols, r, r_out, r_code,
                        weight.data_ptr(), w_code, eps, y.data_ptr(), y_code, scales, block, _stream_of(index))
    if status:
        raise AQError(status, "aq_rmsnorm")
    return residual_out


def rmsnorm(x, weight, eps=1e-5, residual=None, residual_out=None, y_dtype=None, y=None):
    """h = x + residual and y = weight * h / sqrt(mean(h^2) + eps) for each row of x ([rows][cols],
    rows may be strided). Returns (y, h): y of y_dtype (x's by default), h of the residual's dtype
    (into residual_out where given, which may be the residual itself), or None without one."""
    if y is None:
        if x.is_contiguous():
            y = torch.empty_like(x, dtype=y_dtype)
        else:
            y = torch.empty(x.shape, dtype=x.dtype if y_dtype is None else y_dtype, device=x.device)
    elif y.shape != x.shape or not y.is_contiguous() or y.get_device() != x.get_device():
        raise ValueError("y must be contiguous, of x's shape and on its device")
    code = _CODES.get(y.dtype)
    if code is None:
        raise TypeError("unsupported output dtype %s" % y.dtype)
    return y, _norm(x, weight, eps, residual, residual_out, y, code, None, 0)


def rmsnorm_8bit(x, weight, eps=1e-5, residual=None, residual_out=None, block=32):
    """As rmsnorm with y in 8 bits: returns (codes, scales, h), codes float8_e4m3fn [rows][cols],
    scales uint8 [rows][cols / block] (value = code * 2^(scale - 127), exact in bf16; a uint8
    scale viewed as float8_e8m0fnu is its power of two). block: 32 columns, or 0 for one scale
    per row."""
    rows, cols = x.shape
    block = block or cols
    if cols % block:
        raise ValueError("cols must be a multiple of the block")
    codes = torch.empty((rows, cols), dtype=torch.float8_e4m3fn, device=x.device)
    scales = torch.empty((rows, cols // block), dtype=torch.uint8, device=x.device)
    h = _norm(x, weight, eps, residual, residual_out, codes, AQ_E4M3, scales.data_ptr(), block)
    return codes, scales, h
