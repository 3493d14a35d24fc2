"""The paged cache of keys and values that scores a member, and the attention
over it: the binding of es_kv_* in include/esopt.h, which defines every result.

    cache = KVCache.allocate(pages, kv_heads, head_dim, format="e4m3", page=64)
    q = cache.append(k, v, slots, q=q, q_gain=gq, k_gain=gk, rope=table, positions=pos)
    out = cache.attend(q, tables, lengths, starts)
    k, v = cache.read(slots)

Argument marshalling only: the work runs in the library's HIP kernels.  Calls
are stream-ordered, allocate nothing but the outputs that the caller does not
give, and can be captured in a graph.
"""

import ctypes

import torch

from .esopt import (EsKvAppend, EsKvAttend, EsKvDesc, _check, _stream, _u32_arg, load)

ES_KV_INT8 = 0
ES_KV_E4M3 = 1
ES_KV_BF16 = 2
ES_KV_ADJACENT = 1
ES_KV_BAD_SLOT = 1
ES_KV_BAD_POSITION = 2
ES_KV_BAD_PAGE = 4
ES_KV_BAD_LENGTH = 8

_FORMATS = {torch.int8: ES_KV_INT8, torch.float8_e4m3fn: ES_KV_E4M3, torch.bfloat16: ES_KV_BF16}
_DTYPES = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn, "bf16": torch.bfloat16}


def _rows(t, shape, what):
    """Pointer and token stride of [tokens, heads, dim] bf16 rows whose heads
    are adjacent (a slice of a packed projection qualifies)."""
    if t.dtype != torch.bfloat16 or not t.is_cuda or t.dim() != 3:
        raise ValueError(f"{what} must be a bf16 CUDA tensor [tokens, heads, head_dim]")
    if tuple(t.shape) != shape:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {shape}")
    s = t.stride()
    if t.numel() and ((shape[2] > 1 and s[2] != 1) or (shape[1] > 1 and s[1] != shape[2])):
        raise ValueError(f"{what}: a token's heads must be adjacent")
    if s[0] < 0:
        raise ValueError(f"{what}: negative stride")
    return t.data_ptr(), s[0]


def _array(t, dtype, n, what):
    if t is None:
        return None
    if t.dtype != dtype or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} CUDA tensor")
    if t.numel() != n:
        raise ValueError(f"{what} has {t.numel()} elements, expected {n}")
    return t.data_ptr()


class KVCache:
    """A cache over the caller's pages: k_pages [pages, heads, page, dim],
    v_pages [pages, heads, dim, page] (torch.bfloat16, torch.int8 or
    torch.float8_e4m3fn, which sets the format) and, for the 8-bit formats,
    k_scales and v_scales [pages, heads, page] in float32.  The object keeps
    references to them.  `allocate` makes them."""

    def __init__(self, k_pages, v_pages, k_scales=None, v_scales=None):
        self._h = None
        if k_pages.dtype not in _FORMATS or v_pages.dtype != k_pages.dtype:
            raise ValueError("pages must both be bfloat16, int8 or float8_e4m3fn")
        if k_pages.dim() != 4:
            raise ValueError("k_pages must have the shape [pages, heads, page, dim]")
        pages, heads, page, dim = k_pages.shape
        if tuple(v_pages.shape) != (pages, heads, dim, page):
            raise ValueError(f"v_pages has shape {tuple(v_pages.shape)}, expected "
                             f"{(pages, heads, dim, page)}")
        scaled = k_pages.dtype != torch.bfloat16
        for t, what in ((k_pages, "k_pages"), (v_pages, "v_pages")):
            if not t.is_cuda or not t.is_contiguous():
                raise ValueError(f"{what} must be a contiguous CUDA tensor")
        for t, what in ((k_scales, "k_scales"), (v_scales, "v_scales")):
            if scaled != (t is not None):
                raise ValueError(f"{what}: 8-bit pages have scales, bf16 pages have none")
            if scaled and (t.dtype != torch.float32 or not t.is_cuda or not t.is_contiguous()
                           or tuple(t.shape) != (pages, heads, page)):
                raise ValueError(f"{what} must be a contiguous float32 CUDA tensor of shape "
                                 f"{(pages, heads, page)}")
        self.k_pages, self.v_pages, self.k_scales, self.v_scales = (k_pages, v_pages, k_scales,
                                                                    v_scales)
        self.pages, self.kv_heads, self.page, self.head_dim = pages, heads, page, dim
        self.device = k_pages.device
        d = EsKvDesc(k_pages.data_ptr(), v_pages.data_ptr(),
                     k_scales.data_ptr() if scaled else None,
                     v_scales.data_ptr() if scaled else None, pages, page, heads, dim,
                     _FORMATS[k_pages.dtype], 0)
        handle = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check(load().es_kv_create(ctypes.byref(d), ctypes.byref(handle)), "es_kv_create")
        self._h = handle

    @classmethod
    def allocate(cls, pages, kv_heads, head_dim, format="bf16", page=64, device="cuda"):
        """A cache over pages of its own (zeroed)."""
        if format not in _DTYPES:
            raise ValueError(f"format must be one of {sorted(_DTYPES)}")
        size = 2 if format == "bf16" else 1

        def room(*shape):
            n = size
            for x in shape:
                n *= x
            return torch.zeros(n, dtype=torch.uint8, device=device).view(
                _DTYPES[format]).view(*shape)
        scales = [None if format == "bf16" else
                  torch.zeros(pages, kv_heads, page, dtype=torch.float32, device=device)
                  for _ in range(2)]
        return cls(room(pages, kv_heads, page, head_dim), room(pages, kv_heads, head_dim, page),
                   *scales)

    @property
    def device_bytes(self):
        return int(load().es_kv_device_bytes(self._h))

    def close(self):
        if self._h is not None:
            h, self._h = self._h, None
            _check(load().es_kv_destroy(h), "es_kv_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def append(self, k, v, slots, q=None, q_out=None, q_gain=None, k_gain=None, eps=1e-6,
               rope=None, positions=None, adjacent=False, status=None, stream=None):
        """Store tokens' keys (normalised and rotated) and values, and return
        their queries, normalised and rotated (None without q).

        k, v [tokens, kv_heads, dim] and q [tokens, q_heads, dim] are bf16,
        any token stride; slots [tokens] int64 (negative: not stored); gains
        [dim] bf16 or None (no norm); rope [positions, rot] float32, cosines
        then sines, with positions [tokens] int32, or None (no rotation);
        adjacent pairs dimensions 2 i and 2 i + 1 instead of i and
        i + rot / 2.  q_out may be q.  status: uint32-sized CUDA tensor
        (int32) that collects the ES_KV_BAD_* bits."""
        tokens = int(k.shape[0])
        shape = (tokens, self.kv_heads, self.head_dim)
        a = EsKvAppend()
        a.k, a.k_stride = _rows(k, shape, "k")
        a.v, a.v_stride = _rows(v, shape, "v")
        if q is not None:
            heads = int(q.shape[1]) if q.dim() == 3 else 0
            q_shape = (tokens, heads, self.head_dim)
            a.q, a.q_stride = _rows(q, q_shape, "q")
            if q_out is None:
                q_out = torch.empty(q_shape, dtype=torch.bfloat16, device=q.device)
            a.q_out, a.q_out_stride = _rows(q_out, q_shape, "q_out")
            a.q_heads = heads
        elif q_out is not None:
            raise ValueError("q_out without q")
        a.q_gain = _array(q_gain, torch.bfloat16, self.head_dim, "q_gain")
        a.k_gain = _array(k_gain, torch.bfloat16, self.head_dim, "k_gain")
        a.eps = float(eps)
        if rope is not None:
            if rope.dim() != 2 or positions is None:
                raise ValueError("rope must be [positions, rot], with positions")
            a.rope = _array(rope, torch.float32, rope.numel(), "rope")
            a.rope_rows, a.rot = rope.shape
            a.positions = _array(positions, torch.int32, tokens, "positions")
        elif positions is not None:
            raise ValueError("positions without rope")
        a.slots = _array(slots, torch.int64, tokens, "slots")
        a.status = _array(status, torch.int32, 1, "status")
        a.tokens = _u32_arg(tokens, "tokens")
        a.flags = ES_KV_ADJACENT if adjacent else 0
        _check(load().es_kv_append(self._h, ctypes.byref(a), _stream(stream)), "es_kv_append")
        return q_out

    def read(self, slots, k_out=None, v_out=None, status=None, stream=None):
        """The keys and values that slots [tokens] int64 hold, as bf16
        [tokens, kv_heads, dim] (a negative slot: zeros)."""
        tokens = int(slots.numel())
        shape = (tokens, self.kv_heads, self.head_dim)
        outs = []
        for t, what in ((k_out, "k_out"), (v_out, "v_out")):
            if t is None:
                t = torch.empty(shape, dtype=torch.bfloat16, device=self.device)
            outs.append((t, *_rows(t, shape, what)))
        _check(load().es_kv_read(self._h, _array(slots, torch.int64, tokens, "slots"),
                                 _u32_arg(tokens, "tokens"), outs[0][1], outs[0][2], outs[1][1],
                                 outs[1][2], _array(status, torch.int32, 1, "status"),
                                 _stream(stream)), "es_kv_read")
        return outs[0][0], outs[1][0]

    def attend(self, q, tables, lengths, starts, max_rows=None, max_length=None, out=None,
               first=None, limit=None, scale=None, cap=0.0, slopes=None, status=None,
               stream=None):
        """Attention of q [rows, q_heads, dim] (bf16) over the cache.

        tables [seqs, pages] int32, lengths [seqs] int32 (the rows' own tokens
        among them) and starts [seqs + 1] int32 (rows of each sequence) lie on
        the GPU.  first and limit [rows] int32 set the keys that a row sees
        (default: up to its own position); scale defaults to dim^-1/2; cap > 0
        caps scores by a tanh; slopes [q_heads] float32 weigh a bias by
        distance.  max_rows and max_length, the caller's bounds of rows and
        length of a sequence, choose how the work is cut."""
        rows, heads = int(q.shape[0]), int(q.shape[1]) if q.dim() == 3 else 0
        shape = (rows, heads, self.head_dim)
        a = EsKvAttend()
        a.q, a.q_stride = _rows(q, shape, "q")
        if out is None:
            out = torch.empty(shape, dtype=torch.bfloat16, device=q.device)
        a.out, a.out_stride = _rows(out, shape, "out")
        if tables.dim() != 2:
            raise ValueError("tables must be [seqs, pages]")
        seqs, a.table_stride = tables.shape
        a.tables = _array(tables, torch.int32, tables.numel(), "tables")
        a.lengths = _array(lengths, torch.int32, seqs, "lengths")
        a.starts = _array(starts, torch.int32, seqs + 1, "starts")
        a.first = _array(first, torch.int32, rows, "first")
        a.limit = _array(limit, torch.int32, rows, "limit")
        a.slopes = _array(slopes, torch.float32, heads, "slopes")
        a.status = _array(status, torch.int32, 1, "status")
        a.rows, a.n_seqs, a.q_heads = _u32_arg(rows, "rows"), _u32_arg(seqs, "seqs"), heads
        a.max_rows = _u32_arg(rows if max_rows is None else max_rows, "max_rows")
        a.max_length = _u32_arg(tables.shape[1] * self.page if max_length is None else max_length,
                                "max_length")
        a.scale = float(self.head_dim ** -0.5 if scale is None else scale)
        a.cap = float(cap)
        _check(load().es_kv_attend(self._h, ctypes.byref(a), _stream(stream)), "es_kv_attend")
        return out
