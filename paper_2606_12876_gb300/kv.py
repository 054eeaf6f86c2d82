"""PagedKVCache: the key-value cache of a model's layers on the GPU, in pages (aq_kv_* of libaq).

Lists of sequences, counts, positions and pages are int32 tensors on the cache's device. Nothing
synchronises: conditions found on the device (no free page, a bad index) are recorded and raised
by check(). Work is enqueued on the current stream; calls that change the cache must not overlap
other calls on it. Calls may be captured in CUDA graphs, on any stream, once the cache has been
called outside a capture; a graph may be replayed on any stream, and graphs that only attend beside
each other and beside eager calls. Every capture has workspaces of its own, a few MB that the cache
keeps (so it has to outlive its graphs).
"""
import ctypes

import torch

from . import (AQ_BF16, AQ_E4M3, AQ_F16, AQ_F32, AQ_OK, AQError, KVCache, aq_kv_attend,
               aq_kv_compact, aq_kv_copy_pages, aq_kv_fork, aq_kv_free, aq_kv_init, aq_kv_reserve,
               aq_kv_write, aq_workspace_status, kv_attend_workspace_bytes, kv_workspace_bytes,
               workspace, CaptureWorkspace, capture_id, _capturing, _stream_of)

_FLOATS = {torch.float16: AQ_F16, torch.bfloat16: AQ_BF16, torch.float32: AQ_F32}
_CODES = dict(_FLOATS)
_CODES[torch.float8_e4m3fn] = AQ_E4M3
_INT32 = torch.int32
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
            aq_kv_init(self._c, _stream_of(self._index))

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
        self.device, self.dtype, self._index = k.device, k.dtype, k.get_device()
        self.kv_heads, self.head_dim, self.page_tokens, self.layers = heads, dim, page, layers
        self._c = KVCache(layers, pages, page, heads, dim, lens.numel(), tables.shape[1], _CODES[k.dtype],
                          *[None if t is None else t.data_ptr()
                            for t in (k, v, k_scales, v_scales, tables, lens, refs)])
        self._ref = ctypes.byref(self._c)
        # the query's dtype codes that attend takes
        self._q_codes = {torch.float16: AQ_F16, torch.bfloat16: AQ_BF16} if small else {k.dtype: _CODES[k.dtype]}
        self._ws = {}
        if not kv_workspace_bytes(self._c):
            raise ValueError("unsupported cache: page_tokens must be a power of two in 8..1024, "
                             "head_dim a multiple of 16 up to 256, and no size may be 0")

    def _scratch(self, q_heads=0):
        # (stream, workspace address, bytes, its owner). One workspace per stream for eager calls, as
        # calls on different streams may overlap, and one per stream of a capture, as its graph may be
        # replayed on any stream; attention has its own (by query heads), page operations share one.
        stream = _stream_of(self._index)
        capturing = stream != 0 and _capturing()
        key = (stream, q_heads, capture_id(stream)) if capturing else (stream, q_heads)
        got = self._ws.get(key)
        if got is None:
            if capturing and not self._ws:
                raise RuntimeError("the cache's first call is inside a capture: make one outside before, on any stream")
            n = kv_attend_workspace_bytes(self._c, 1, q_heads) if q_heads else kv_workspace_bytes(self._c)
            ws = CaptureWorkspace(n) if capturing else workspace(n, self.device)
            got = self._ws[key] = (stream, ws.data_ptr(), ws.numel(), ws)
        return got

    def _pages(self, call, *args):
        stream, ws, size, _ = self._scratch()
        status = call(self._ref, *args, ws, size, stream)
        if status:
            raise AQError(status, call.__name__)

    def _list(self, t, what, n=None):
        if t.dtype != _INT32 or t.get_device() != self._index or t.dim() != 1 or not t.is_contiguous():
            raise ValueError("%s must be a contiguous int32 list on the cache's device" % what)
        if n is not None and t.shape[0] != n:
            raise ValueError("%s must have %d entries" % (what, n))
        return t.shape[0]

    def reserve(self, seqs, counts=None):
        """Lengthen the listed sequences by counts tokens (default one each), taking the lowest
        free pages in the order of the list; all or nothing (see check)."""
        n = self._list(seqs, "seqs")
        if counts is not None:
            self._list(counts, "counts", n)
        self._pages(aq_kv_reserve, n, seqs.data_ptr(), None if counts is None else counts.data_ptr())

    def fork(self, src, dst):
        """Make the empty sequences dst copies of src: full pages are shared, a partial last page
        is copied; all or nothing (see check)."""
        n = self._list(src, "src")
        self._list(dst, "dst", n)
        self._pages(aq_kv_fork, n, src.data_ptr(), dst.data_ptr())

    def free(self, seqs):
        """Release the listed sequences and the pages that no other sequence holds."""
        self._pages(aq_kv_free, self._list(seqs, "seqs"), seqs.data_ptr())

    def compact(self, used=None):
        """Move the pages in use to the lowest indices; used: an int32 tensor of one element that
        receives their number, or None."""
        if used is not None:
            self._list(used, "used", 1)
        self._pages(aq_kv_compact, None if used is None else used.data_ptr())

    def copy_pages(self, src, dst):
        """Copy pages src to pages dst in all layers (dst distinct, none of them in src)."""
        n = self._list(src, "src")
        self._list(dst, "dst", n)
        self._pages(aq_kv_copy_pages, n, src.data_ptr(), dst.data_ptr())

    def write(self, k, v, seqs, positions=None, layer=0):
        """Store row i of k and v ([n][kv_heads][head_dim], fp16, bf16 or fp32; rows may be
        strided, with the same stride in both) as token positions[i] of sequence seqs[i] (default: its last token)."""
        n = self._list(seqs, "seqs")
        at = None
        if positions is not None:
            self._list(positions, "positions", n)
            at = positions.data_ptr()
        stride = self._rows(k, "k", n, self.kv_heads)
        code = _FLOATS.get(k.dtype)
        if code is None:
            raise TypeError("unsupported dtype %s" % k.dtype)
        if self._rows(v, "v", n, self.kv_heads) != stride or v.dtype != k.dtype:
            raise ValueError("k and v must have the same dtype and row stride")
        stream, ws, size, _ = self._scratch()
        status = aq_kv_write(self._ref, layer, n, seqs.data_ptr(), at, k.data_ptr(), v.data_ptr(),
                             code, stride, ws, size, stream)
        if status:
            raise AQError(status, "aq_kv_write")

    def attend(self, q, seqs=None, layer=0, scale=None, window=0, out=None, lse=None):
        """Attention of q ([n][q_heads][head_dim], the cache's dtype, or fp16/bf16 for an e4m3
        cache; rows may be strided) over the cached tokens of the listed sequences (default
        0..n-1): [n][q_heads][head_dim] of q's dtype. scale: head_dim**-0.5 by default; window:
        tokens seen from the end (0: all); lse: an fp32 [n][q_heads] tensor that receives the
        log of each row's sum of exponentials, or None."""
        code = self._q_codes.get(q.dtype)
        if code is None:
            raise TypeError("q is %s, the cache %s" % (q.dtype, self.dtype))
        shape = q.shape
        if len(shape) != 3 or shape[1] == 0 or shape[1] % self.kv_heads:
            raise ValueError("q must be [n][q_heads][head_dim], q_heads a positive multiple of %d" % self.kv_heads)
        n, q_heads = shape[0], shape[1]
        stride = self._rows(q, "q", n, q_heads)
        # (Arguments keep their names until after the launch: one that only the caller's expression
        # held would be freed, and its memory given to `out`.)
        seqs_at = lse_at = None
        if seqs is not None:
            self._list(seqs, "seqs", n)
            seqs_at = seqs.data_ptr()
        if out is None:
            out = torch.empty_like(q) if q.is_contiguous() else torch.empty(shape, dtype=q.dtype, device=self.device)
        elif out.shape != shape or out.dtype != q.dtype or out.get_device() != self._index or \
                not out.is_contiguous():
            raise ValueError("out must be contiguous, of q's shape and dtype")
        if lse is not None:
            if lse.shape != shape[:2] or lse.dtype != torch.float32 or \
                    lse.get_device() != self._index or not lse.is_contiguous():
                raise ValueError("lse must be a contiguous fp32 [n][q_heads] tensor")
            lse_at = lse.data_ptr()
        if window > 0x7fffffff:                     # (longer than any sequence; the C call takes an int)
            window = 0
        stream, ws, size, _ = self._scratch(q_heads)
        status = aq_kv_attend(self._ref, layer, n, seqs_at, q.data_ptr(), code, stride, q_heads,
                              self.head_dim ** -0.5 if scale is None else scale, window,
                              out.data_ptr(), lse_at, ws, size, stream)
        if status:
            raise AQError(status, "aq_kv_attend")
        return out

    def _rows(self, t, what, n, heads):
        # The row stride of a [n][heads][head_dim] tensor whose rows are contiguous.
        dim = self.head_dim
        if t.shape != (n, heads, dim) or t.get_device() != self._index:
            raise ValueError("%s must be [%d][%d][%d] on the cache's device" % (what, n, heads, dim))
        s = t.stride()
        if s[2] != 1 or (heads > 1 and s[1] != dim):
            raise ValueError("the rows of %s must be contiguous" % what)
        return s[0] if n > 1 else heads * dim

    def check(self):
        """Synchronise the device (a captured call may have been replayed on any stream) and raise
        AQError if a call recorded a condition (AQ_ERR_CAPACITY: no free page or a full table;
        AQ_ERR_INVALID_ARG)."""
        bad = AQ_OK
        with torch.cuda.device(self.device):
            torch.cuda.synchronize()
            for _, _, _, ws in self._ws.values():
                bad = aq_workspace_status(ws) or bad
        if bad != AQ_OK:
            raise AQError(bad, "PagedKVCache")
