"""Pins of the MX oracle: closed forms, invariants and differences."""

import numpy as np
import pytest

from oracle import mx_oracle as mx


def test_grids():
    assert mx.grid(mx.MXFP4).tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    g = mx.grid(mx.MXFP8)
    assert g.size == 127 and g[-1] == 448 and g[1] == 2.0 ** -9 and g[8] == 2.0 ** -6 and (np.diff(g) > 0).all()


def test_closed_forms():
    row = np.zeros((1, 33))
    row[0, :14] = [7.9, 5.0, 3.5, 2.5, 1.75, 1.25, 0.75, 0.25, 0.26, -0.75, -6.0, 4.0, -0.0, 0.5]
    row[0, 32] = 3e-39                                                   # a block of its own: below 2^-126, E = -127
    codes, scales = mx.quantize(row, mx.MXFP4)
    assert scales.tolist() == [[127, 0]]
    got = mx.values(codes, scales, 33, mx.MXFP4)[0]
    # ties go to the even code: 5 -> 4, 3.5 -> 4, 2.5 -> 2, 1.75 -> 2, 1.25 -> 1, 0.75 -> 1, 0.25 -> 0
    assert got[:14].tolist() == [6, 4, 4, 2, 2, 1, 1, 0, 0.5, -1, -6, 4, 0, 0.5]
    assert got[32] == 0.5 * 2.0 ** -127                                  # 3e-39 = 0.51 2^-127
    codes, scales = mx.quantize(np.array([[500.0, 464.0, 448.0, 432.0, 1.0, 2.0 ** -10, 2.0 ** -10 * 1.01]]), mx.MXFP8)
    assert scales.tolist() == [[127]]
    assert mx.values(codes, scales, 7, mx.MXFP8)[0].tolist() == [448, 448, 448, 448, 1, 0, 2.0 ** -9]
    assert (mx.unpack(mx.pack(np.arange(32, dtype=np.uint8)[None] % 16, mx.MXFP4), mx.MXFP4) == np.arange(32) % 16).all()


@pytest.mark.parametrize("fmt", [mx.MXFP4, mx.MXFP8])
def test_invariants(fmt):
    g = np.random.Generator(np.random.Philox(3))
    X = g.standard_t(3, size=(50, 100)) * np.exp(3 * g.standard_normal((50, 1)))
    once = mx.through(X, fmt)
    assert np.array_equal(mx.through(once, fmt), once)                    # representable values stay
    assert np.array_equal(mx.through(X * 2.0 ** 9, fmt), once * 2.0 ** 9)
    assert np.array_equal(mx.through(-X, fmt), -once)
    err = np.abs(X - once)
    top = np.pad(np.abs(X), ((0, 0), (0, 28))).reshape(50, 4, 32).max(-1).repeat(32, 1)[:, :100]
    # e2m1: half a step of 2 in the top binade, or the cut from below 8 to 6: a quarter of the block's largest; e4m3: 2^-4 of the
    # value, the cut from 512 to 448, or half the smallest step, 2^-10 2^-8 of the largest
    assert (err <= (0.25 * top if fmt == mx.MXFP4 else np.maximum(np.abs(X) / 8, top * 2.0 ** -18))).all()
    bad = X.copy()
    bad[3, 40] = np.nan
    bad[4, 2] = -np.inf
    codes, scales = mx.quantize(bad, fmt)
    assert scales[3, 1] == 255 and scales[4, 0] == 255 and (scales == 255).sum() == 2
    v = mx.values(codes, scales, 100, fmt)
    assert np.isnan(v[3, 32:64]).all() and np.isnan(v[4, :32]).all() and np.isnan(v).sum() == 64


@pytest.mark.parametrize("fmt", [mx.MXFP4, mx.MXFP8])
def test_objective_gradient_is_the_difference_quotient(fmt):
    g = np.random.Generator(np.random.Philox(4))
    Y = g.standard_normal((3, 70))
    loss, dY = mx.objective(Y, fmt, "mean")
    assert mx.objective(Y, fmt, "sum")[0] == pytest.approx(3 * loss)
    h = 1e-9
    for t, i in ((0, 0), (1, 33), (2, 69), (0, 31), (1, 5)):
        up, down = Y.copy(), Y.copy()
        up[t, i] += h
        down[t, i] -= h
        fd = (mx.objective(up, fmt)[0] - mx.objective(down, fmt)[0]) / (2 * h)
        assert fd == pytest.approx(dY[t, i], abs=1e-6)
    assert mx.objective(mx.through(Y, fmt), fmt)[0] == 0.0


def test_rms_norm():
    assert np.allclose(mx.rms_norm(np.array([[3.0, 4.0]]), None, 0.0), np.array([[3.0, 4.0]]) / np.sqrt(12.5))
    assert (mx.rms_norm(np.zeros((2, 5)), None, 0.0) == 0).all()
    assert np.allclose(mx.rms_norm(np.ones((1, 4)), [1, 2, 3, 4], 3.0), [[0.5, 1, 1.5, 2]])
