"""Low-rank adapters of many members beside a shared projection: the binding of
es_adapt_* in include/esopt.h, which defines the result.

    adapters = Adapters(a, b, scales)        # [members, rank, inner], [members, outer, rank]
    y = adapters.project(x, weight, index)   # row r under the adapter of member index[r]

A population of low-rank members is scored side by side in one batch instead of
one after another.  The adapters of a member are two bf16 tensors like any
others: esopt.Plan([a[i], b[i]]) perturbs, restores and updates them in place, with
the same noise for the same seed whichever member's they are.

Argument marshalling only: the work runs in the library's HIP kernels.  Calls
are stream-ordered and can be captured in a graph; each takes a workspace of its
own from PyTorch's allocator, so calls may overlap.  `stream` is as in kvcache.
"""

import struct

import torch

from .esopt import ES_OK, _check, load
from .head import _empty, _matrix
from .kvcache import _array, _count, _current_stream

ES_ADAPT_BAD_INDEX = 1

_ADAPT = struct.Struct("=3Q 3Q 2Q 3Q Q Q 6I")


class Adapters:
    """The adapters a [members, rank, inner] and b [members, outer, rank] (bf16,
    contiguous; rank a multiple of 8 up to 128, inner one of 8) with scales
    [members] (float32; None: ones).  The object keeps references to them and
    reads them anew in every call."""

    def __init__(self, a, b, scales=None):
        for t, what in ((a, "a"), (b, "b")):
            if t.dtype != torch.bfloat16 or not t.is_cuda or not t.is_contiguous() or t.dim() != 3:
                raise ValueError(f"{what} must be a contiguous bf16 CUDA tensor of three dimensions")
        self.members, self.rank, self.inner = a.shape
        self.outer = b.shape[1]
        if b.shape[0] != self.members or b.shape[2] != self.rank:
            raise ValueError(f"b has shape {tuple(b.shape)}, expected "
                             f"{(self.members, 'outer', self.rank)}")
        if not 1 <= self.members <= 65536:
            raise ValueError(f"{self.members} members, must be in 1 .. 65536")
        if self.rank % 8 or not 8 <= self.rank <= 128:
            raise ValueError(f"rank must be a multiple of 8 up to 128, got {self.rank}")
        _array(scales, torch.float32, self.members, "scales")
        self.a, self.b, self.scales = a, b, scales

    def project(self, x, weight, index, out=None, status=None, stream=None):
        """W x + s_i B_i (A_i x) for rows x [rows, inner] (bf16, any row stride), weight
        [outer, inner] and i = index [rows] (int32; negative: no adapter), as bf16
        [rows, outer].  status: a CUDA tensor of one int32 that collects
        ES_ADAPT_BAD_INDEX."""
        x_at, x_stride = _matrix(x, (None, self.inner), "x")
        w_at, w_stride = _matrix(weight, (self.outer, self.inner), "weight")
        rows = x.shape[0]
        if out is None:
            out = _empty((rows, self.outer), torch.bfloat16, x.device, stream)
        out_at, out_stride = _matrix(out, (rows, self.outer), "out")
        head = (x_at, w_at, out_at, x_stride, w_stride, out_stride, self.a.data_ptr(),
                self.b.data_ptr(), 0 if self.scales is None else self.scales.data_ptr(),
                _array(index, torch.int32, rows, "index"),
                _array(status, torch.int32, 1, "status"))
        sizes = (_count(rows, "rows"), self.inner, self.outer, self.members, self.rank, 0)
        lib = load()
        size = lib.es_adapt_bytes(_ADAPT.pack(*head, 0, 0, *sizes))
        room = _empty(size, torch.uint8, x.device, stream)
        rc = lib.es_adapt_project(_ADAPT.pack(*head, room.data_ptr(), size, *sizes),
                                  _current_stream(stream))
        if rc != ES_OK:
            _check(rc, "es_adapt_project")
        return out
