"""Pins of oracle/attention.py: element-by-element renderings with the math
module, closed forms, and PyTorch's own rounding to E4M3."""
import math

import numpy as np
import pytest
import torch

from oracle import attention as oa


def test_norm_and_rotation_against_scalar_code():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 2, 8))
    gain = rng.standard_normal(8)
    angle = rng.uniform(-9, 9, (3, 2))
    turn = np.concatenate([np.cos(angle), np.sin(angle)], axis=1)       # rot = 4
    for adjacent in (False, True):
        y = oa.norm_rotate(x, gain, 1e-3, turn, adjacent)
        for t in range(3):
            for h in range(2):
                r = math.sqrt(sum(a * a for a in x[t, h]) / 8 + 1e-3)
                z = [a / r * g for a, g in zip(x[t, h], gain)]
                w = list(z)
                for i in range(2):
                    a, b = (2 * i, 2 * i + 1) if adjacent else (i, i + 2)
                    c, s = math.cos(angle[t, i]), math.sin(angle[t, i])
                    w[a], w[b] = z[a] * c - z[b] * s, z[b] * c + z[a] * s
                np.testing.assert_allclose(y[t, h], w, rtol=1e-13, atol=1e-15)
    # a quarter turn takes (1, 0) to (0, 1)
    e = np.zeros((1, 1, 4))
    e[0, 0, 0] = 1
    out = oa.norm_rotate(e, turn=np.array([[0.0, 1.0, 1.0, 0.0]]))
    np.testing.assert_array_equal(out[0, 0], [0, 0, 1, 0])


def test_e4m3_rounding_is_pytorchs():
    rng = np.random.default_rng(2)
    grid = oa.GRID
    mid = (grid[:-1] + grid[1:]) / 2                       # every tie
    y = np.concatenate([grid, mid, rng.uniform(-448, 448, 4000), rng.normal(0, 0.01, 4000)])
    y = y.astype(np.float32)
    want = torch.from_numpy(y).to(torch.float8_e4m3fn).float().numpy()
    np.testing.assert_array_equal(oa.nearest_e4m3(y), want)


@pytest.mark.parametrize("form", ["int8", "e4m3"])
def test_quantised_rows_are_within_half_a_step(form):
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((5, 3, 64)) * np.exp(rng.uniform(-20, 20, (5, 3, 1)))).astype(np.float32)
    x[0, 0] = 0
    x[1, 1] = 1e-38
    codes, scale = oa.quantise_f32(x, form)
    assert scale[0, 0] == 0 and scale[1, 1] == 0
    v = oa.code_values(codes, scale, form)
    top = np.max(np.abs(x), axis=-1, keepdims=True).astype(np.float64)
    step = top / 127 if form == "int8" else np.maximum(np.abs(x) / 8, top / 448 * 2.0 ** -9)
    big = top >= 2.0 ** -100
    assert np.all(np.abs(v - x)[np.broadcast_to(big, x.shape)]
                  <= (0.5 * step * (1 + 1e-5) + 1e-6 * np.abs(x))[np.broadcast_to(big, x.shape)])
    assert np.all(v[~np.broadcast_to(big, x.shape)] == 0)


def test_attention_against_scalar_code_and_closed_forms():
    rng = np.random.default_rng(4)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((7, 2, 8)), rng.standard_normal((7, 2, 8))
    first, limit, slopes, cap = [0, 2, 6], [5, 9, 6], [0.1, 0.2, 0.3, 0.4], 1.5
    out, spread = oa.attend(q, k, v, 0.4, cap, slopes, first, limit)
    for i in range(3):
        for h in range(4):
            keys = [j for j in range(7) if first[i] <= j < min(limit[i], 7)]
            w = []
            for j in keys:
                t = cap * math.tanh(0.4 * sum(a * b for a, b in zip(q[i, h], k[j, h // 2])) / cap)
                w.append(math.exp(t - slopes[h] * abs(7 - 3 + i - j)))
            if not keys:
                assert np.all(out[i, h] == 0)
                continue
            want = [sum(a * v[j, h // 2, d] for a, j in zip(w, keys)) / sum(w) for d in range(8)]
            np.testing.assert_allclose(out[i, h], want, rtol=1e-12, atol=1e-14)
    # one visible key gives its value; equal scores average; causal by default
    one, _ = oa.attend(q, k, v, 0.4, first=[3, 3, 3], limit=[4, 4, 4])
    np.testing.assert_allclose(one[:, 0], np.broadcast_to(v[3, 0], (3, 8)), rtol=1e-14)
    flat, _ = oa.attend(np.zeros_like(q), k, v, 0.4)
    for i in range(3):
        np.testing.assert_allclose(flat[i, 3], v[:5 + i, 1].mean(axis=0), rtol=1e-12)
