"""PagedKVCache: the key-value cache of a model's layers on the GPU, in pages (aq_kv_* of libaq).

Lists of sequences, counts, positions and pages are int32 tensors on the cache's device. Nothing
synchronises: conditions found on the device (no free page, a bad index) are recorded and raised
by check(). Work is enqueued on the current stream; calls that change the cache must not overlap
other calls on it.
"""
import torch

from . import (AQ_BF16, AQ_E4M3, AQ_F16, AQ_F32, AQ_OK, AQError, KVCache, aq_kv_attend,
               aq_kv_compact, aq_kv_copy_pages, aq_kv_fork, aq_kv_free, aq_kv_init, aq_kv_reserve,
               aq_kv_write, aq_workspace_status, kv_attend_workspace_bytes, kv_workspace_bytes,
               workspace, _stream)

_CODES = {torch.float16: AQ_F16, torch.bfloat16: AQ_BF16, torch.float32: AQ_F32,
          torch.float8_e4m3fn: AQ_E4M3}
_NAMES = {"f16": torch.float16, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}


class PagedKVCache:
    """Keys and values of `layers` layers: num_pages pages of page_tokens tokens, kv_heads heads
    of head_dim; max_seqs sequence slots of up to max_pages pages each (default: the whole pool).
    dtype: "f16", "bf16", or "e4m3" (8-bit values with a power-of-two scale per token and head).

    k, v: [layers][num_pages][kv_heads][page_tokens][head_dim]; k_scales, v_scales (e4m3): uint8,
    the scale's exponent + 127; tables [max_seqs][max_pages], lens [max_seqs], refs [num_pages].
    """

    def __init__(self, num_pages, page_tokens, kv_heads, head_dim, max_seqs, max_pages=None,
                 layers=1, dtype="bf16", device="cuda"):
        dt = _NAMES[dtype]
        shape = (layers, num_pages, kv_heads, page_tokens, head_dim)
        new = lambda s, d: torch.empty(s, dtype=d, device=device)
        scales = [new(shape[:-1], torch.uint8) for _ in range(2)] if dtype == "e4m3" else [None] * 2
        if max_pages is None:
            max_pages = num_pages
        self._adopt(new(shape, dt), new(shape, dt), new((max_seqs, max_pages), torch.int32),
                    new((max_seqs,), torch.int32), new((num_pages,), torch.int32), *scales)
        with torch.cuda.device(self.device):
            aq_kv_init(self._c)

    @classmethod
    def from_tensors(cls, k, v, tables, lens, refs, k_scales=None, v_scales=None):
        """A cache over existing tensors (contiguous, shaped as the attributes above), as they
        stand: the bookkeeping must be consistent."""
        self = cls.__new__(cls)
        self._adopt(k, v, tables, lens, refs, k_scales, v_scales)
        return self

    def _adopt(self, k, v, tables, lens, refs, k_scales, v_scales):
        if k.dtype not in _NAMES.values():
            raise TypeError("unsupported cache dtype %s" % k.dtype)
        if k.dim() != 5:
            raise ValueError("k must be [layers][num_pages][kv_heads][page_tokens][head_dim]")
        layers, pages, heads, page, dim = k.shape
        small = k.dtype == torch.float8_e4m3fn
        if small != (k_scales is not None) or small != (v_scales is not None):
            raise ValueError("scales belong to an e4m3 cache, and only there")
        want = [("v", v, k.shape, k.dtype), ("tables", tables, (lens.numel(), tables.shape[-1]), torch.int32),
                ("lens", lens, (lens.numel(),), torch.int32), ("refs", refs, (pages,), torch.int32)]
        if small:
            want += [("k_scales", k_scales, k.shape[:-1], torch.uint8),
                     ("v_scales", v_scales, k.shape[:-1], torch.uint8)]
        for name, t, shape, dt in [("k", k, k.shape, k.dtype)] + want:
            if tuple(t.shape) != tuple(shape) or t.dtype != dt:
                raise ValueError("%s must be %s of shape %s" % (name, dt, tuple(shape)))
            if not t.is_cuda or t.device != k.device or not t.is_contiguous():
                raise ValueError("%s must be contiguous and on the cache's CUDA device" % name)
        self.k, self.v, self.k_scales, self.v_scales = k, v, k_scales, v_scales
        self.tables, self.lens, self.refs = tables, lens, refs
        self.device, self.dtype = k.device, k.dtype
        self.kv_heads, self.head_dim, self.page_tokens, self.layers = heads, dim, page, layers
        self._ptr = lambda t: None if t is None else t.data_ptr()
        self._c = KVCache(layers, pages, page, heads, dim, lens.numel(), tables.shape[1],
                          _CODES[k.dtype], *[self._ptr(t) for t in (k, v, k_scales, v_scales, tables,
                                                                    lens, refs)])
        self._ws = {}
        if not kv_workspace_bytes(self._c):
            raise ValueError("unsupported cache: page_tokens must be a power of two in 8..1024 and "
                             "head_dim a multiple of 16 up to 256")

    def _scratch(self, kind, q_heads=None):
        # One workspace per (kind, stream), as calls on different streams may overlap.
        key = (kind, _stream(None))
        ws = self._ws.get(key)
        if ws is None:
            n = kv_workspace_bytes(self._c) if kind == "pages" else \
                kv_attend_workspace_bytes(self._c, 1, q_heads)
            ws = self._ws[key] = workspace(n, self.device)
        return ws, ws.numel()

    def _list(self, t, what, n=None):
        if t.dtype != torch.int32 or t.device != self.device or t.dim() != 1 or not t.is_contiguous():
            raise ValueError("%s must be a contiguous int32 list on the cache's device" % what)
        if n is not None and t.numel() != n:
            raise ValueError("%s must have %d entries" % (what, n))
        return t.numel()

    def reserve(self, seqs, counts=None):
        """Lengthen the listed sequences by counts tokens (default one each), taking the lowest
        free pages in the order of the list; all or nothing (see check)."""
        n = self._list(seqs, "seqs")
        if counts is not None:
            self._list(counts, "counts", n)
        aq_kv_reserve(self._c, n, seqs, counts, *self._scratch("pages"))

    def fork(self, src, dst):
        """Make the empty sequences dst copies of src: full pages are shared, a partial last page
        is copied; all or nothing (see check)."""
        n = self._list(src, "src")
        self._list(dst, "dst", n)
        aq_kv_fork(self._c, n, src, dst, *self._scratch("pages"))

    def free(self, seqs):
        """Release the listed sequences and the pages that no other sequence holds."""
        aq_kv_free(self._c, self._list(seqs, "seqs"), seqs, *self._scratch("pages"))

    def compact(self, used=None):
        """Move the pages in use to the lowest indices; used: an int32 tensor of one element that
        receives their number, or None."""
        if used is not None:
            self._list(used, "used", 1)
        aq_kv_compact(self._c, used, *self._scratch("pages"))

    def copy_pages(self, src, dst):
        """Copy pages src to pages dst in all layers (dst distinct, none of them in src)."""
        n = self._list(src, "src")
        self._list(dst, "dst", n)
        aq_kv_copy_pages(self._c, n, src, dst, *self._scratch("pages"))

    def write(self, k, v, seqs, positions=None, layer=0):
        """Store row i of k and v ([n][kv_heads][head_dim], fp16, bf16 or fp32; rows may be
        strided) as token positions[i] of sequence seqs[i] (default: its last token)."""
        n = self._list(seqs, "seqs")
        if positions is not None:
            self._list(positions, "positions", n)
        stride = self._rows(k, "k", n, self.kv_heads)
        if self._rows(v, "v", n, self.kv_heads) != stride or v.dtype != k.dtype:
            raise ValueError("k and v must have the same dtype and row stride")
        if k.dtype not in _CODES or k.dtype == torch.float8_e4m3fn:
            raise TypeError("unsupported dtype %s" % k.dtype)
        aq_kv_write(self._c, layer, n, seqs, positions, k, v, _CODES[k.dtype], stride,
                    *self._scratch("pages"))

    def attend(self, q, seqs=None, layer=0, scale=None, window=0, out=None, lse=None):
        """Attention of q ([n][q_heads][head_dim], the cache's dtype, or fp16/bf16 for an e4m3
        cache; rows may be strided) over the cached tokens of the listed sequences (default
        0..n-1): [n][q_heads][head_dim] of q's dtype. scale: head_dim**-0.5 by default; window:
        tokens seen from the end (0: all); lse: an fp32 [n][q_heads] tensor that receives the
        log of each row's sum of exponentials, or None."""
        n, q_heads = q.shape[0], q.shape[1]
        if seqs is not None:
            self._list(seqs, "seqs", n)
        stride = self._rows(q, "q", n, q_heads)
        if q_heads == 0 or q_heads % self.kv_heads:
            raise ValueError("q_heads must be a positive multiple of %d" % self.kv_heads)
        if q.dtype != self.dtype and not (self.dtype == torch.float8_e4m3fn and
                                          q.dtype in (torch.float16, torch.bfloat16)):
            raise TypeError("q is %s, the cache %s" % (q.dtype, self.dtype))
        if out is None:
            out = torch.empty((n, q_heads, self.head_dim), dtype=q.dtype, device=self.device)
        elif out.shape != q.shape or out.dtype != q.dtype or out.device != self.device or \
                not out.is_contiguous():
            raise ValueError("out must be contiguous, of q's shape and dtype")
        if lse is not None and (lse.shape != q.shape[:2] or lse.dtype != torch.float32 or
                                lse.device != self.device or not lse.is_contiguous()):
            raise ValueError("lse must be a contiguous fp32 [n][q_heads] tensor")
        aq_kv_attend(self._c, layer, n, seqs, q, _CODES[q.dtype], stride, q_heads,
                     self.head_dim ** -0.5 if scale is None else scale, window, out, lse,
                     *self._scratch("attend", q_heads))
        return out

    def _rows(self, t, what, n, heads):
        # The row stride of a [n][heads][head_dim] tensor whose rows are contiguous.
        if t.dim() != 3 or t.shape[0] != n or t.shape[1] != heads or t.shape[2] != self.head_dim or \
                t.device != self.device:
            raise ValueError("%s must be [%d][%d][%d] on the cache's device" % (what, n, heads, self.head_dim))
        s = t.stride()
        if s[2] != 1 or (heads > 1 and s[1] != self.head_dim):
            raise ValueError("the rows of %s must be contiguous" % what)
        return s[0] if n > 1 else heads * self.head_dim

    def check(self):
        """Synchronise the streams that used the cache and raise AQError if a call recorded a
        condition (AQ_ERR_CAPACITY: no free page or a full table; AQ_ERR_INVALID_ARG)."""
        bad = AQ_OK
        for (_, stream), ws in self._ws.items():
            bad = aq_workspace_status(ws, stream) or bad
        if bad != AQ_OK:
            raise AQError(bad, "PagedKVCache")
