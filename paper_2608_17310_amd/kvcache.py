"""The paged cache of keys and values that scores a member, and the attention
over it: the binding of es_kv_* in include/esopt.h, which defines every result.

    cache = KVCache.allocate(pages, kv_heads, head_dim, format="e4m3", page=64)
    q = cache.append(k, v, slots, q=q, q_gain=gq, k_gain=gk, rope=table, positions=pos)
    out = cache.attend(q, tables, lengths, starts)
    k, v = cache.read(slots)

Argument marshalling only: the work runs in the library's HIP kernels.  Calls
are stream-ordered, allocate nothing but the outputs that the caller does not
give, and can be captured in a graph.  `stream` (a torch.cuda.Stream or a raw
handle; default: the current one) is where a call runs and where its outputs'
memory belongs: as under torch.cuda.stream, other streams wait for it before
they use them.
"""

import ctypes
import struct

import torch

from .esopt import EsKvDesc, ES_OK, _check, _stream, load

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


# The argument structs of include/esopt.h, packed in one step: at single tokens
# the calls are bound by the host, and setting twenty ctypes fields one by one
# takes 3 us of them.
_APPEND = struct.Struct("=3Q Q 4Q 6Q 4I f I")
_ATTEND = struct.Struct("=2Q 2Q 7Q 6I 2f")


def _current_stream(stream):
    """The raw handle of `stream`, or of PyTorch's current one."""
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return _stream(stream)


def _output(shape, device, stream):
    """A bf16 output for a call on `stream`, in that stream's memory: a block of
    the current stream's may still be in use by work queued there, and would be
    handed out again while the call's stream uses it."""
    if stream is None:
        return torch.empty(shape, dtype=torch.bfloat16, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=torch.bfloat16, device=device)


def _rows(t, shape, what):
    """Pointer and token stride of [tokens, heads, dim] bf16 rows whose heads
    are adjacent (a slice of a packed projection qualifies)."""
    if t.dtype != torch.bfloat16 or not t.is_cuda or t.shape != shape:
        raise ValueError(f"{what} must be a bf16 CUDA tensor of shape {tuple(shape)}, not "
                         f"{tuple(t.shape)} {t.dtype}")
    s = t.stride()
    if (s[2] != 1 or s[1] != shape[2]) and t.numel() and (s[2] != 1 or shape[1] > 1):
        raise ValueError(f"{what}: a token's heads must be adjacent")
    if s[0] < 0:
        raise ValueError(f"{what}: negative stride")
    return t.data_ptr(), s[0]


def _array(t, dtype, n, what):
    """Address of a contiguous tensor of n elements; 0 for None."""
    if t is None:
        return 0
    if t.dtype != dtype or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous {dtype} CUDA tensor")
    if t.numel() != n:
        raise ValueError(f"{what} has {t.numel()} elements, expected {n}")
    return t.data_ptr()


def _heads(t, what):
    if t.dim() != 3:
        raise ValueError(f"{what} must be [tokens, heads, head_dim]")
    return t.shape[1]


def _count(x, what):
    if not 0 <= x < (1 << 32):
        raise ValueError(f"{what} must be in [0, 2^32), got {x}")
    return x


class KVCache:
    """A cache over the caller's pages: k_pages [pages, heads, page, dim],
    v_pages [pages, heads, dim, page] (torch.bfloat16, torch.int8 or
    torch.float8_e4m3fn, which sets the format) and, for the 8-bit formats,
    k_scales and v_scales [pages, heads, page] in float32.  The object keeps
    references to them.  `allocate` makes them.

    The parts of a long history are joined in scratch that belongs to the
    object: calls of `attend` on one cache, from any streams or threads, must be
    ordered one after another (two caches over the same pages have a scratch
    each)."""

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
        self._lib = load()

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
        tokens = k.shape[0] if k.dim() == 3 else -1
        dim = self.head_dim
        shape = (tokens, self.kv_heads, dim)
        k_at, k_stride = _rows(k, shape, "k")
        v_at, v_stride = _rows(v, shape, "v")
        q_at = q_stride = out_at = out_stride = q_heads = 0
        if q is not None:
            q_heads = _heads(q, "q")
            shape = (tokens, q_heads, dim)
            q_at, q_stride = _rows(q, shape, "q")
            if q_out is None:
                q_out = _output(shape, q.device, stream)
            out_at, out_stride = _rows(q_out, shape, "q_out")
        elif q_out is not None:
            raise ValueError("q_out without q")
        rope_at = pos_at = rope_rows = rot = 0
        if rope is not None:
            if rope.dim() != 2 or positions is None:
                raise ValueError("rope must be [positions, rot], with positions")
            rope_rows, rot = rope.shape
            rope_at = _array(rope, torch.float32, rope_rows * rot, "rope")
            pos_at = _array(positions, torch.int32, tokens, "positions")
        elif positions is not None:
            raise ValueError("positions without rope")
        args = _APPEND.pack(
            q_at, k_at, v_at, out_at, q_stride, k_stride, v_stride, out_stride,
            _array(q_gain, torch.bfloat16, dim, "q_gain"),
            _array(k_gain, torch.bfloat16, dim, "k_gain"), rope_at, pos_at,
            _array(slots, torch.int64, tokens, "slots"), _array(status, torch.int32, 1, "status"),
            _count(tokens, "tokens"), q_heads, rot, _count(rope_rows, "rope rows"), eps,
            ES_KV_ADJACENT if adjacent else 0)
        rc = self._lib.es_kv_append(self._h, args, _current_stream(stream))
        if rc != ES_OK:
            _check(rc, "es_kv_append")
        return q_out

    def read(self, slots, k_out=None, v_out=None, status=None, stream=None):
        """The keys and values that slots [tokens] int64 hold, as bf16
        [tokens, kv_heads, dim] (a negative slot: zeros)."""
        tokens = slots.numel()
        shape = (tokens, self.kv_heads, self.head_dim)
        if k_out is None and v_out is None:
            k_out, v_out = _output((2,) + shape, self.device, stream).unbind(0)
        elif k_out is None or v_out is None:
            raise ValueError("give both outputs or none")
        k_at, k_stride = _rows(k_out, shape, "k_out")
        v_at, v_stride = _rows(v_out, shape, "v_out")
        rc = self._lib.es_kv_read(self._h, _array(slots, torch.int64, tokens, "slots"),
                                  _count(tokens, "tokens"), k_at, k_stride, v_at, v_stride,
                                  _array(status, torch.int32, 1, "status"),
                                  _current_stream(stream))
        if rc != ES_OK:
            _check(rc, "es_kv_read")
        return k_out, v_out

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
        heads = _heads(q, "q")
        rows = q.shape[0]
        shape = (rows, heads, self.head_dim)
        q_at, q_stride = _rows(q, shape, "q")
        if out is None:
            out = _output(shape, q.device, stream)
        out_at, out_stride = _rows(out, shape, "out")
        if tables.dim() != 2:
            raise ValueError("tables must be [seqs, pages]")
        seqs, width = tables.shape
        args = _ATTEND.pack(
            q_at, out_at, q_stride, out_stride,
            _array(tables, torch.int32, seqs * width, "tables"),
            _array(lengths, torch.int32, seqs, "lengths"),
            _array(starts, torch.int32, seqs + 1, "starts"),
            _array(first, torch.int32, rows, "first"), _array(limit, torch.int32, rows, "limit"),
            _array(slopes, torch.float32, heads, "slopes"),
            _array(status, torch.int32, 1, "status"), _count(rows, "rows"),
            _count(seqs, "seqs"), _count(width, "table width"), heads,
            _count(rows if max_rows is None else max_rows, "max_rows"),
            _count(width * self.page if max_length is None else max_length, "max_length"),
            self.head_dim ** -0.5 if scale is None else scale, cap)
        rc = self._lib.es_kv_attend(self._h, args, _current_stream(stream))
        if rc != ES_OK:
            _check(rc, "es_kv_attend")
        return out
