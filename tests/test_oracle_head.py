"""The fp64 definitions of scores, divergences, their gradients and projections
under adapters, against closed forms, differences and PyTorch's in 64 bits."""
import math

import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import head as oh


def make(seed, rows=6, vocab=11, hidden=5, entries=1):
    rng = np.random.default_rng(seed)
    x, w = rng.standard_normal((rows, hidden)), rng.standard_normal((vocab, hidden))
    ids = rng.integers(0, vocab, (rows, entries))
    return x, w, ids, rng.standard_normal((rows, entries)), rng.standard_normal(rows)


def test_equal_logits_have_equal_probabilities():
    x, w, ids, _, _ = make(0)
    loss, logp, lse = oh.score(np.zeros_like(x), w, ids)
    assert np.allclose(logp, -math.log(11)) and np.allclose(lse, math.log(11)) and not loss.any()
    # a teacher with two equal entries, against 11 equal ones: log(11 / 2)
    loss, _, _ = oh.score(np.zeros_like(x), w, np.tile([[3, 5]], (6, 1)), teacher=np.ones((6, 2)))
    assert np.allclose(loss, math.log(11 / 2))


def test_one_entry_is_a_target():
    x, w, ids, t, grad = make(1)
    loss, logp, _ = oh.score(x, w, ids, 0.7, t)
    assert np.allclose(loss, -logp[:, 0])
    for a, b in zip(oh.gradients(x, w, ids, grad, 0.7, t), oh.gradients(x, w, ids, grad, 0.7)):
        assert np.allclose(a, -b)


@pytest.mark.parametrize("scale", [1.0, 0.5])
def test_scores_and_gradients_against_torch(scale):
    x, w, ids, _, grad = make(2)
    ids[4] = -100
    tx, tw = (torch.tensor(a, requires_grad=True) for a in (x, w))
    nll = F.cross_entropy(tx @ tw.t() * scale, torch.tensor(ids[:, 0]), ignore_index=-100, reduction="none")
    (-nll * torch.tensor(grad)).sum().backward()
    _, logp, _ = oh.score(x, w, ids, scale)
    dx, dw = oh.gradients(x, w, ids, grad, scale)
    assert np.allclose(logp[:, 0], -nll.detach().numpy())
    assert np.allclose(dx, tx.grad.numpy()) and np.allclose(dw, tw.grad.numpy())


@pytest.mark.parametrize("scale", [1.0, 0.5])
def test_divergences_and_gradients_against_torch(scale):
    """Every id given: the divergence of whole distributions."""
    x, w, _, _, grad = make(3)
    ids = np.stack([np.random.default_rng(i).permutation(11) for i in range(6)])
    t = np.random.default_rng(4).standard_normal((6, 11))
    tx, tw = (torch.tensor(a, requires_grad=True) for a in (x, w))
    q = torch.zeros(6, 11, dtype=torch.float64).scatter(1, torch.tensor(ids), torch.tensor(t * scale))
    kl = F.kl_div((tx @ tw.t() * scale).log_softmax(-1), q.log_softmax(-1), reduction="none",
                  log_target=True).sum(-1)
    (kl * torch.tensor(grad)).sum().backward()
    loss, _, _ = oh.score(x, w, ids, scale, t)
    dx, dw = oh.gradients(x, w, ids, grad, scale, t)
    assert np.allclose(loss, kl.detach().numpy())
    assert np.allclose(dx, tx.grad.numpy()) and np.allclose(dw, tw.grad.numpy())


def test_gradients_against_differences():
    x, w, ids, t, grad = make(5, entries=4)
    ids[1, 2:], ids[2] = -1, ids[2, 0]
    t[3, 1] = -np.inf

    def value(x, w):
        return (oh.score(x, w, ids, 0.8, t)[0] * grad).sum()
    dx, dw = oh.gradients(x, w, ids, grad, 0.8, t)
    for at, g in ((0, dx), (1, dw)):
        v = np.random.default_rng(6).standard_normal(g.shape)
        h = 1e-6
        args = [[x, w], [x, w]]
        args[0][at], args[1][at] = args[0][at] + h * v, args[1][at] - h * v
        assert abs((value(*args[0]) - value(*args[1])) / (2 * h) - (g * v).sum()) <= 1e-6 * np.abs(g * v).sum()


def test_rows_without_a_result():
    x, w, ids, t, grad = make(7, entries=3)
    ids[0], ids[1, 1], t[2] = -1, 11, -np.inf
    x[0], t[0], grad[0] = np.nan, np.nan, np.nan
    loss, logp, lse = oh.score(x, w, ids, 1.0, t)
    assert loss[0] == lse[0] == 0 and not logp[0].any()
    assert np.isnan(loss[1]) and np.isnan(lse[1]) and np.isnan(logp[1]).all()
    assert loss[2] == 0 and lse[2] != 0 and logp[2].all()
    dx, dw = oh.gradients(x, w, ids, grad, 1.0, t)
    assert not dx[0].any() and np.isnan(dx[1]).all() and not dx[2].any() and np.isfinite(dw).all()


def test_projections_are_those_of_merged_weights():
    rng = np.random.default_rng(8)
    x, w = rng.standard_normal((7, 5)), rng.standard_normal((4, 5))
    a, b, s = rng.standard_normal((3, 2, 5)), rng.standard_normal((3, 4, 2)), rng.standard_normal(3)
    index = np.array([0, -1, 2, 1, 1, -7, 3])
    got = oh.project(x, w, a, b, index, s)
    for r, i in enumerate(index):
        if i < 3:
            merged = w if i < 0 else w + s[i] * b[i] @ a[i]
            assert np.allclose(got[r], merged @ x[r])
    assert np.isnan(got[6]).all()


@pytest.mark.parametrize("scale", [1.0, 0.0, -0.5])
def test_a_teacher_that_leaves_nothing(scale):
    x, w, ids, t, grad = make(9, entries=3)
    t[2] = -np.inf
    t[3, 1] = -np.inf
    loss, _, _ = oh.score(x, w, ids, scale, t)
    gone = np.where(np.isneginf(t), -1, ids)
    assert np.isfinite(loss).all() and loss[2] == 0
    assert loss[3] == oh.score(x, w, gone, scale, t)[0][3]
    x[2] = np.nan
    dx, dw = oh.gradients(x, w, ids, grad, scale, t)
    wx, ww = oh.gradients(x, w, gone, grad, scale, t)
    assert np.array_equal(dx, wx) and np.array_equal(dw, ww) and not dx[2].any()


def test_a_teacher_that_is_no_number():
    x, w, ids, t, grad = make(10, entries=3)
    t[1, 2], t[4, 0] = np.nan, np.inf
    ids[5, 1], t[5, 1] = -1, np.nan                        # absent: not looked at
    with np.errstate(invalid="ignore"):
        for scale, lost in ((0.7, [1, 4]), (-0.7, [1])):
            loss, logp, lse = oh.score(x, w, ids, scale, t)
            assert np.flatnonzero(np.isnan(loss)).tolist() == lost and np.isfinite(logp).all()
            dx, dw = oh.gradients(x, w, ids, grad, scale, t)
            assert np.flatnonzero(np.isnan(dx).any(1)).tolist() == lost
            assert np.isnan(dx[lost]).all() and np.isnan(dw).all()
