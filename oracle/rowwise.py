"""8-bit codes and the root-mean-square norm, restated in numpy.

The codes are defined down to their rounding, so they are computed here in
fp32 steps by numpy's correctly rounded operations; everything else is fp64 on
exact input values.
"""
from __future__ import annotations

import numpy as np

A_MIN = np.float32(2.0 ** -100)


def codes(t):
    """(codes, scales) of the rows of an fp32 matrix t: with a = max(max|t|, 2^-100),
    rint(fl(t * fl(127 / a))) and fl(a / 127).  A row with Inf or NaN: 0 and NaN."""
    t = np.asarray(t, np.float32)
    rows, cols = t.shape
    fine = np.isfinite(t).all(axis=1)
    safe = np.where(fine[:, None], t, np.float32(0))
    a = np.maximum(np.abs(safe).max(axis=1) if cols else np.zeros(rows, np.float32), A_MIN).astype(np.float32)
    inv = (np.float32(127) / a).astype(np.float32)
    q = np.rint((safe * inv[:, None]).astype(np.float32)).astype(np.int8)
    scale = (a / np.float32(127)).astype(np.float32)
    return q, np.where(fine, scale, np.float32(np.nan)).astype(np.float32)


def gemm_i8(a, a_scale, b, b_scale, bias=None, relu=False):
    """act((a b^T) * a_scale * b_scale + bias), sums exact."""
    acc = np.asarray(a, np.int64) @ np.asarray(b, np.int64).T
    v = acc.astype(np.float64) * np.asarray(a_scale, np.float64)[:, None] * np.asarray(b_scale, np.float64)
    if bias is not None:
        v = v + np.asarray(bias, np.float64)
    return np.where(v < 0, 0.0, v) if relu else v


def rmsnorm(h, gamma, eps):
    """y of the rows of h."""
    h = np.asarray(h, np.float64)
    return h / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps) * np.asarray(gamma, np.float64)


def rmsnorm_codes(x, res, gamma, eps):
    """(codes, scales) of rmsnorm's rows from fp32 x (+ res): codes of fl(fl(x + res) * gamma), scales
    fl(a / 127) / rms."""
    h = np.asarray(x, np.float32)
    if res is not None:
        h = (h + np.asarray(res, np.float32)).astype(np.float32)
    t = h if gamma is None else (h * np.asarray(gamma, np.float32)).astype(np.float32)
    q, s = codes(t)
    h = h.astype(np.float64)
    return q, s.astype(np.float64) / np.sqrt(np.mean(h * h, axis=1) + eps)


def rmsnorm_bwd(dy, h, gamma, eps, dres=None):
    """(dx, dgamma): y_c = gamma_c h_c / r, r = sqrt(mean h^2 + eps), so
    dL/dh_j = gamma_j dy_j / r - h_j sum_c(gamma_c dy_c h_c) / (n r^3)."""
    dy, h, gamma = (np.asarray(v, np.float64) for v in (dy, h, gamma))
    n = h.shape[1]
    r = np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    dx = gamma * dy / r - h * np.sum(gamma * dy * h, axis=1, keepdims=True) / (n * r ** 3)
    if dres is not None:
        dx = dx + np.asarray(dres, np.float64)
    return dx, np.sum(dy * h / r, axis=0)
