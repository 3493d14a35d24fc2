"""Scoring a member: rows for the paged cache and attention over it (oracle;
test-only), in fp64 from the definitions in the library's header.

A member is evaluated between two moves of the parameters (Section 3: apply,
evaluate, revert); the paper does not describe its models' attention, so the
definitions are the library's: queries and keys normalised for each head,
rotated by position, keys and values stored as bf16, int8 or E4M3 with one
binary32 scale per token and head, softmax attention with capped scores, a
bias by distance and an interval of visible keys for each row.

Pins (tests/test_oracle_attention.py): element-by-element renderings with the
math module, closed forms (equal scores average the values, one visible key
returns its value, rotation by 90 degrees), and PyTorch's conversion for E4M3.
"""

import numpy as np

from .fp8 import e4m3_decode, e4m3_encode, GRID

CODE_MAX = {"int8": 127.0, "e4m3": 448.0}
TINY_ROW = 2.0 ** -100


def norm_rotate(x, gain=None, eps=1e-6, turn=None, adjacent=False):
    """Rows x [tokens, heads, dim] normalised (with a gain) and rotated by
    turn [tokens, rot] (cosines, then sines)."""
    x = np.array(x, dtype=np.float64)
    if gain is not None:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps) * np.asarray(gain, np.float64)
    if turn is None:
        return x
    turn = np.asarray(turn, np.float64)[:, None, :]
    half = turn.shape[-1] // 2
    i = np.arange(half)
    a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
    c, s = turn[..., :half], turn[..., half:]
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def quantise_f32(x, form):
    """Codes and scales of binary32 rows x, in the cache's own arithmetic
    (binary32 scale, reciprocal and products; one rounding to nearest even)."""
    x = np.asarray(x, np.float32)
    top = np.max(np.abs(x), axis=-1, keepdims=True)
    live = top >= np.float32(TINY_ROW)
    big = np.float32(CODE_MAX[form])
    safe = np.where(live, top, np.float32(1.0))
    y = np.where(live, x * (big * (np.float32(1.0) / safe)), np.float32(0.0)).astype(np.float32)
    scale = np.where(live, safe / big, np.float32(0.0)).astype(np.float32)
    if form == "int8":
        return np.rint(y).astype(np.int8), scale[..., 0]
    return e4m3_encode(nearest_e4m3(y.astype(np.float64))), scale[..., 0]


def nearest_e4m3(y):
    """The nearest E4M3 value (ties to the even code), |y| <= 448 (1 + 2^-20)."""
    y = np.clip(np.asarray(y, np.float64), -448.0, 448.0)
    hi = np.clip(np.searchsorted(GRID, y, side="left"), 1, GRID.size - 1)
    lo, up = GRID[hi - 1], GRID[hi]
    down, above = y - lo, up - y
    tie_up = (e4m3_encode(up) & 1) == 0
    return np.where((above < down) | ((above == down) & tie_up), up, lo)


def code_values(codes, scales, form):
    """Values of codes [..., dim] with scales [...]."""
    v = (np.asarray(codes).view(np.int8).astype(np.float64) if form == "int8"
         else e4m3_decode(codes))
    return v * np.asarray(scales, np.float64)[..., None]


def visible(length, n, first=None, limit=None):
    """[n, length] truth values: the keys that the last n rows of a sequence see."""
    pos = np.arange(length - n, length)
    lo = np.zeros(n, np.int64) if first is None else np.maximum(np.asarray(first, np.int64), 0)
    hi = pos + 1 if limit is None else np.asarray(limit, np.int64)
    key = np.arange(length)
    return (key >= lo[:, None]) & (key < np.minimum(hi, length)[:, None])


def attend(q, k, v, scale, cap=0.0, slopes=None, first=None, limit=None):
    """(out, spread): attention of q [n, q_heads, dim] over k, v [length,
    kv_heads, dim], and sum_j p_j |v_j|, which bounds the effect of relative
    errors of the weights.  Rows stand at length - n + i; a row that sees
    nothing gives zeros."""
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    n, hq, d = q.shape
    length, h = k.shape[:2]
    see = visible(length, n, first, limit)
    pos = np.arange(length - n, length)
    out = np.zeros((n, hq, d))
    spread = np.zeros((n, hq, d))
    rows = see.any(axis=1)
    if not rows.any():
        return out, spread
    away = np.abs(pos[:, None] - np.arange(length))
    for i in range(hq):
        j = i // (hq // h)
        with np.errstate(invalid="ignore", over="ignore"):
            t = q[:, i] @ k[:, j].T * scale
            if cap > 0:
                t = cap * np.tanh(t / cap)
            if slopes is not None:
                t = t - float(slopes[i]) * away
            t = np.where(see, t, -np.inf)[rows]
            p = np.exp(t - np.max(t, axis=1, keepdims=True))
            p /= p.sum(axis=1, keepdims=True)
            out[rows, i] = p @ v[:, j]
            spread[rows, i] = p @ np.abs(v[:, j])
    return out, spread
