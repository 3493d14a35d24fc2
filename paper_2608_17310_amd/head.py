"""A decoder's head without its logits: log-probabilities of given tokens, the
divergence from a teacher that is known by its top logits, and the gradients of
both: the binding of es_head_* in include/esopt.h, which defines every result.

    head = Head(weight)                                   # [vocab, hidden]
    logp, lse = head.score(hidden, targets)
    dx, dw = head.score_gradient(hidden, targets, logp, lse, grad)
    loss, logp, lse = head.distill(hidden, ids, logits)
    dx, dw = head.distill_gradient(hidden, ids, logits, logp, lse, grad)

Argument marshalling only: the work runs in the library's HIP kernels.  Calls
are stream-ordered and can be captured in a graph; each takes a workspace of its
own from PyTorch's allocator, so calls on one head may overlap.  `stream` is as in
kvcache.
"""

import struct

import torch

from .esopt import ES_OK, _check, load
from .kvcache import _array, _count, _current_stream

ES_HEAD_BAD_ID = 1

_SCORE = struct.Struct("=2Q 2Q 7Q Q 4I f I")
_GRADIENT = struct.Struct("=2Q 2Q 7Q 2Q 2Q Q 4I f I")


def _empty(shape, dtype, device, stream):
    """An output or workspace of a call on `stream`, in that stream's memory."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _matrix(t, shape, what):
    """Address and row stride of a bf16 matrix whose rows are contiguous."""
    if t.dtype != torch.bfloat16 or not t.is_cuda or t.dim() != 2:
        raise ValueError(f"{what} must be a bf16 CUDA matrix, not {tuple(t.shape)} {t.dtype}")
    for have, want in zip(t.shape, shape):
        if want is not None and have != want:
            raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {shape}")
    s = t.stride()
    if (s[1] != 1 and t.shape[1] > 1) or s[0] < 0:
        raise ValueError(f"{what}: rows must be contiguous")
    if t.shape[0] > 1 and s[0] == 0:
        raise ValueError(f"{what}: an expanded matrix has no rows of its own")
    return t.data_ptr(), s[0]


class Head:
    """The head `weight` [vocab, hidden] (bf16, contiguous rows); the object keeps
    a reference to it and reads it anew in every call."""

    def __init__(self, weight):
        _matrix(weight, (None, None), "weight")
        if not weight.shape[0] or not weight.shape[1]:
            raise ValueError("weight is empty")
        self.weight = weight
        self.vocab, self.hidden = weight.shape

    def score(self, hidden, targets, scale=1.0, status=None, stream=None):
        """Log-probabilities [rows] of targets [rows] (int64; negative: none) after
        hidden [rows, hidden] (bf16), and the logarithms [rows] of the normalisers,
        float32, with logits scale hidden weight^T.  status: a CUDA tensor of one
        int32 that collects ES_HEAD_BAD_ID."""
        _matrix(hidden, (None, self.hidden), "hidden")
        rows = hidden.shape[0]
        if targets.dim() != 1:
            raise ValueError("targets must be [rows]")
        out = _empty((2, rows), torch.float32, hidden.device, stream)
        self._score(hidden, targets, None, None, out[0], out[1], 1, scale, status, stream)
        return out[0], out[1]

    def distill(self, hidden, ids, logits, scale=1.0, status=None, stream=None):
        """Divergences [rows] from a teacher whose logits [rows, entries] (float32)
        stand at ids [rows, entries] (int64; negative: none), the student's
        log-probabilities [rows, entries] there and the logarithms [rows] of its
        normalisers.  scale, the inverse temperature, applies to both sides."""
        if ids.dim() != 2 or logits.shape != ids.shape:
            raise ValueError("ids and logits must be [rows, entries]")
        _matrix(hidden, (ids.shape[0], self.hidden), "hidden")
        rows, entries = ids.shape
        out = _empty((2, rows), torch.float32, hidden.device, stream)
        logp = _empty((rows, entries), torch.float32, hidden.device, stream)
        self._score(hidden, ids, logits, out[0], logp, out[1], entries, scale, status, stream)
        return out[0], logp, out[1]

    def score_gradient(self, hidden, targets, logp, lse, grad, scale=1.0, hidden_grad=True,
                       weight_grad=True, status=None, stream=None):
        """Gradients of sum(grad logp), grad [rows] float32, for hidden and for the
        weight, bf16 (None where not wanted), from what `score` returned."""
        if targets.dim() != 1:
            raise ValueError("targets must be [rows]")
        return self._gradient(hidden, targets, None, logp, lse, grad, 1, scale, hidden_grad,
                              weight_grad, status, stream)

    def distill_gradient(self, hidden, ids, logits, logp, lse, grad, scale=1.0, hidden_grad=True,
                         weight_grad=True, status=None, stream=None):
        """Gradients of sum(grad loss) for hidden and for the weight, bf16, from what
        `distill` returned."""
        if ids.dim() != 2 or logits.shape != ids.shape:
            raise ValueError("ids and logits must be [rows, entries]")
        return self._gradient(hidden, ids, logits, logp, lse, grad, ids.shape[1], scale,
                              hidden_grad, weight_grad, status, stream)

    def _sizes(self, rows, entries, scale):
        return (_count(rows, "rows"), _count(self.vocab, "vocab"), _count(self.hidden, "hidden"),
                _count(entries, "entries"), scale, 0)

    def _score(self, hidden, ids, logits, loss, logp, lse, entries, scale, status, stream):
        x, x_stride = _matrix(hidden, (None, self.hidden), "hidden")
        w, w_stride = _matrix(self.weight, (None, None), "weight")
        rows = hidden.shape[0]
        head = (x, w, x_stride, w_stride, _array(ids, torch.int64, rows * entries, "ids"),
                _array(logits, torch.float32, rows * entries, "logits"),
                0 if loss is None else loss.data_ptr(), logp.data_ptr(), lse.data_ptr(),
                _array(status, torch.int32, 1, "status"))
        sizes = self._sizes(rows, entries, scale)
        lib = load()
        size = lib.es_head_score_bytes(_SCORE.pack(*head, 0, 0, *sizes))
        room = _empty(size, torch.uint8, hidden.device, stream)
        rc = lib.es_head_score(_SCORE.pack(*head, room.data_ptr(), size, *sizes),
                               _current_stream(stream))
        if rc != ES_OK:
            _check(rc, "es_head_score")

    def _gradient(self, hidden, ids, logits, logp, lse, grad, entries, scale, hidden_grad,
                  weight_grad, status, stream):
        x, x_stride = _matrix(hidden, (None, self.hidden), "hidden")
        w, w_stride = _matrix(self.weight, (None, None), "weight")
        rows = hidden.shape[0]
        dev = hidden.device
        dx = _empty((rows, self.hidden), torch.bfloat16, dev, stream) if hidden_grad else None
        dw = None
        if weight_grad:
            dw = _empty((self.vocab, self.hidden), torch.bfloat16, dev, stream)
            if not rows:
                return dx, dw.zero_() if stream is None else _zeroed(dw, stream)
        head = (x, w, x_stride, w_stride, _array(ids, torch.int64, rows * entries, "ids"),
                _array(logits, torch.float32, rows * entries, "logits"),
                _array(logp, torch.float32, rows * entries, "logp"),
                _array(lse, torch.float32, rows, "lse"), _array(grad, torch.float32, rows, "grad"),
                0 if dx is None else dx.data_ptr(), 0 if dw is None else dw.data_ptr(),
                self.hidden, self.hidden, _array(status, torch.int32, 1, "status"))
        sizes = self._sizes(rows, entries, scale)
        lib = load()
        size = lib.es_head_gradient_bytes(_GRADIENT.pack(*head, 0, 0, *sizes))
        room = _empty(size, torch.uint8, dev, stream)
        rc = lib.es_head_gradient(_GRADIENT.pack(*head, room.data_ptr(), size, *sizes),
                                  _current_stream(stream))
        if rc != ES_OK:
            _check(rc, "es_head_gradient")
        return dx, dw


def _zeroed(t, stream):
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream), device=t.device)
    with torch.cuda.stream(stream):
        return t.zero_()
