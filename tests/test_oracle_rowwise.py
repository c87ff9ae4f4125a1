"""Pins of oracle/rowwise.py: hand-worked codes, bounds that the definition
implies, closed forms of the norm, and its gradient by differences."""
import numpy as np
import pytest

from oracle import rowwise as R


def test_codes_by_hand():
    # a = 127: factor 1, scale 1; ties to even
    q, s = R.codes(np.float32([[127.0, -127.0, 0.5, 1.5, 2.5, -0.5, -1.5, 63.49]]))
    assert q.tolist() == [[127, -127, 0, 2, 2, 0, -2, 63]]
    assert s.tolist() == [1.0]
    # a = 1: 0.25 * 127 = 31.75
    q, s = R.codes(np.float32([[1.0, 0.25, -0.25]]))
    assert q.tolist() == [[127, 32, -32]] and s[0] == np.float32(1.0) / np.float32(127)


def test_codes_of_rows_without_a_magnitude():
    q, s = R.codes(np.float32([[0, 0], [np.nan, 1], [1, -np.inf], [2.0 ** -101, 0]]))
    assert q.tolist() == [[0, 0], [0, 0], [0, 0], [64, 0]]  # 2^-101 is half of 2^-100: 63.5, the even neighbour
    assert s[0] == np.float32(2.0 ** -100) / np.float32(127) and s[3] == s[0]
    assert np.isnan(s[1]) and np.isnan(s[2])


@pytest.mark.parametrize("seed", range(4))
def test_codes_are_within_half_a_step(seed):
    g = np.random.default_rng(seed)
    t = (g.standard_normal((64, 333)) * np.exp(5 * g.standard_normal((64, 1)))).astype(np.float32)
    q, s = R.codes(t)
    # half a step, and the roundings of 127 / a, the product and the scale: at most 3 * 2^-24 of 127 steps
    assert np.all(np.abs(q * s[:, None].astype(np.float64) - t) <= s[:, None] * (0.5 + 127 * 4 * 2.0 ** -24))
    assert np.abs(q).max(axis=1).tolist() == [127] * 64


def test_codes_of_extreme_maxima_stay_in_range():
    top = np.float32([2.0 ** -100, 2.0 ** -126, 3.4e38, 1e-45, 1.17e-38, 65504.0, np.nextafter(np.float32(1), 2)])
    q, s = R.codes(np.stack([top, -top, top / 2], axis=1))
    assert np.abs(q.astype(int)).max() <= 127 and np.isfinite(s).all() and (s > 0).all()


def test_gemm_i8_by_hand():
    d = R.gemm_i8([[1, -2], [3, 4]], [0.5, 2.0], [[10, 20], [-1, 1]], [1.0, 0.25], bias=[1.0, -1.0], relu=True)
    # sums: [[-30, -3], [110, 1]]
    assert d.tolist() == [[0.0, 0.0], [221.0, 0.0]]
    d = R.gemm_i8([[1, -2], [3, 4]], [0.5, 2.0], [[10, 20], [-1, 1]], [1.0, 0.25])
    assert d.tolist() == [[-15.0, -0.375], [220.0, 0.5]]


def test_rmsnorm_closed_forms():
    y = R.rmsnorm([[3.0, 4.0]], [1.0, 2.0], 0.0)
    r = np.sqrt(12.5)
    assert np.allclose(y, [[3 / r, 8 / r]], rtol=1e-15)
    assert R.rmsnorm([[0.0, 0.0]], [1.0, 1.0], 1e-6).tolist() == [[0.0, 0.0]]
    h = np.random.default_rng(1).standard_normal((5, 17))
    assert np.allclose(np.mean(R.rmsnorm(h, np.ones(17), 0.0) ** 2, axis=1), 1.0, rtol=1e-14)


def test_rmsnorm_codes_stand_for_the_norm():
    g = np.random.default_rng(2)
    x, res = g.standard_normal((9, 201)).astype(np.float32), g.standard_normal((9, 201)).astype(np.float32)
    gamma = (1 + 0.1 * g.standard_normal(201)).astype(np.float32)
    q, s = R.rmsnorm_codes(x, res, gamma, 1e-6)
    y = R.rmsnorm(x.astype(np.float64) + res, gamma, 1e-6)
    assert np.all(np.abs(q * s[:, None] - y) <= s[:, None] * 0.5001)


@pytest.mark.parametrize("with_res", [False, True])
def test_rmsnorm_gradient_by_differences(with_res):
    g = np.random.default_rng(3)
    h, dy, gamma = g.standard_normal((3, 7)), g.standard_normal((3, 7)), 1 + 0.3 * g.standard_normal(7)
    dres = g.standard_normal((3, 7)) if with_res else None
    dx, dg = R.rmsnorm_bwd(dy, h, gamma, 1e-3, dres)
    loss = lambda hh, gg: np.sum(dy * R.rmsnorm(hh, gg, 1e-3)) + (np.sum(dres * hh) if with_res else 0.0)
    e = 1e-6
    for i in np.ndindex(*h.shape):
        d = np.zeros_like(h)
        d[i] = e
        assert abs((loss(h + d, gamma) - loss(h - d, gamma)) / (2 * e) - dx[i]) <= 1e-8
    for j in range(7):
        d = np.zeros(7)
        d[j] = e
        assert abs((loss(h, gamma + d) - loss(h, gamma - d)) / (2 * e) - dg[j]) <= 1e-8
