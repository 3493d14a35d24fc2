"""Scores at a head, divergence from a teacher's top logits, their gradients, and
projections under low-rank adapters, in fp64 NumPy (include/esopt.h, es_head_* and
es_adapt_*).  Inputs are arrays of the stored values; nothing is rounded."""
import numpy as np


def kinds(ids, vocab):
    """live [rows] (some id, none past the vocabulary) and void [rows] (some past it)."""
    void = (ids >= vocab).any(1)
    return (ids >= 0).any(1) & ~void, void


def weighty(ids, teacher, scale):
    """The entries that have a weight: -infinity leaves none at any scale, infinity none at one below 0."""
    return (ids >= 0) & ~np.isneginf(teacher) & ~((scale < 0) & np.isposinf(teacher))


def weights(ids, teacher, scale):
    """The wanted weights q [rows, entries] and their logarithms (0 where q is 0)."""
    here = ids >= 0
    if teacher is None:
        return here.astype(np.float64), np.zeros(ids.shape)
    here = weighty(ids, teacher, scale)
    t = np.where(here, np.where(here, teacher, 0.0) * scale, -np.inf)
    top = t.max(1, keepdims=True)
    e = np.exp(t - np.where(np.isneginf(top), 0.0, top))
    total = e.sum(1, keepdims=True)
    q = np.divide(e, total, out=np.zeros_like(e), where=total != 0)      # (NaN stays NaN)
    log_q = np.log(q, out=np.zeros_like(q), where=q != 0)
    return q, log_q


def logits(x, w, scale):
    return x @ w.T * scale


def score(x, w, ids, scale=1.0, teacher=None):
    """(loss [rows], logp [rows, entries], lse [rows]); without a teacher loss is zeros."""
    live, void = kinds(ids, len(w))
    n, k = ids.shape
    loss, logp, lse = np.zeros(n), np.zeros((n, k)), np.zeros(n)
    q, log_q = weights(ids, teacher, scale)
    for r in np.flatnonzero(live):
        z = x[r] @ w.T * scale
        lse[r] = z.max() + np.log(np.exp(z - z.max()).sum())
        here = ids[r] >= 0
        logp[r, here] = z[ids[r, here]] - lse[r]
        if teacher is not None:
            some = q[r] != 0
            loss[r] = (q[r, some] * (log_q[r, some] - logp[r, some])).sum()
    for out in (loss, logp, lse):
        out[void] = np.nan
    return loss, logp, lse


def logit_gradients(x, w, ids, grad, scale=1.0, teacher=None):
    """d [rows, vocab]: of sum grad logp, or with a teacher sum grad loss."""
    live, _ = kinds(ids, len(w))
    q, _ = weights(ids, teacher, scale)
    d = np.zeros((len(x), len(w)))
    for r in np.flatnonzero(live):
        z = x[r] @ w.T * scale
        p = np.exp(z - z.max())
        d[r] = q[r].sum() * p / p.sum()
        for e in np.flatnonzero(ids[r] >= 0):
            d[r, ids[r, e]] -= q[r, e]
        d[r] *= grad[r] * (-scale if teacher is None else scale)
    return d


def gradients(x, w, ids, grad, scale=1.0, teacher=None):
    """(d_x, d_w); rows that are void have NaN and add nothing."""
    live, void = kinds(ids, len(w))
    if teacher is not None:
        live &= weighty(ids, teacher, scale).any(1)
    x = np.where(live[:, None], x, 0.0)
    d = logit_gradients(x, w, ids, grad, scale, teacher)
    dx = d @ w
    dx[void] = np.nan
    return dx, d.T @ x


def project(x, w, a, b, index, scales=None):
    """[rows, outer]; an index past the members gives NaN."""
    y = x @ w.T
    for r, i in enumerate(index):
        if i >= len(a):
            y[r] = np.nan
        elif i >= 0:
            y[r] += b[i] @ (a[i] @ x[r]) * (1.0 if scales is None else scales[i])
    return y
