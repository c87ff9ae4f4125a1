"""Dropout from a counter-based generator, layer norm with its gradients, and a
last layer with its softmax cross entropy, restated in numpy.

The generator is Philox 4x32 with ten rounds (Salmon, Moraes, Dror and Shaw,
2011), in Python's whole numbers; everything else is fp64 on exact input values.
"""
from __future__ import annotations

import numpy as np


def philox(ctr, key):
    """Four 32-bit words from four words of counter and two of key."""
    c, k = [np.asarray(v, np.uint64) for v in ctr], [int(v) for v in key]
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), p1 & low,
             (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def kept(rows, cols, p, seed, step, site, row0=0):
    """The factor of each element: 0 where it is dropped, 2^16 / (2^16 - t) elsewhere, t = floor(p 2^16 + 1/2)."""
    t = int(np.floor(float(np.float32(p)) * 65536 + 0.5))
    if t == 0:
        return np.ones((rows, cols))
    if t == 65536:
        return np.zeros((rows, cols))
    blocks = -(-cols // 8)
    r, b = np.meshgrid(np.arange(row0, row0 + rows), np.arange(blocks), indexing="ij")
    words = philox([b, r, np.full_like(b, step % 2 ** 32), np.full_like(b, site)],
                   [seed % 2 ** 32, seed // 2 ** 32 % 2 ** 32])
    bits = np.empty((rows, blocks, 8), np.int64)
    for j in range(8):
        bits[:, :, j] = (words[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF)
    return np.where(bits.reshape(rows, -1)[:, :cols] >= t, 65536.0 / (65536 - t), 0.0)


def layernorm(h, gamma, beta, eps):
    """y of the rows of h."""
    h = np.asarray(h, np.float64)
    d = h - h.mean(axis=1, keepdims=True)
    return d / np.sqrt(np.mean(d * d, axis=1, keepdims=True) + eps) * np.asarray(gamma, np.float64) + np.asarray(beta, np.float64)


def layernorm_bwd(dy, h, gamma, eps, dres=None):
    """(dh, dgamma, dbeta): with u = h - mean(h) and r = sqrt(mean u^2 + eps), y_c = gamma_c u_c / r + beta_c, so
    dy_c / dh_j = gamma_c (([c = j] - 1 / n) / r - u_c u_j / (n r^3))."""
    dy, h, gamma = (np.asarray(v, np.float64) for v in (dy, h, gamma))
    n = h.shape[1]
    u = h - h.mean(axis=1, keepdims=True)
    r = np.sqrt(np.mean(u * u, axis=1, keepdims=True) + eps)
    g = dy * gamma
    dh = (g - g.sum(axis=1, keepdims=True) / n) / r - u * np.sum(g * u, axis=1, keepdims=True) / (n * r ** 3)
    if dres is not None:
        dh = dh + np.asarray(dres, np.float64)
    return dh, np.sum(dy * u / r, axis=0), np.sum(dy, axis=0)


def linear_xent(x, w, bias, labels, ignored):
    """(loss, row_loss, lse, z) for w [in, classes]."""
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64)
    if bias is not None:
        z = z + np.asarray(bias, np.float64)
    top = z.max(axis=1)
    with np.errstate(invalid="ignore", divide="ignore"):
        lse = top + np.log(np.sum(np.exp(z - np.where(np.isinf(top), 0.0, top)[:, None]), axis=1))
        labels = np.asarray(labels)
        counted = labels != ignored
        inside = (labels >= 0) & (labels < z.shape[1])
        at = z[np.arange(len(labels)), np.where(inside, labels, 0)]
        row = np.where(counted, np.where(inside, lse - at, np.nan), 0.0)
    return row.sum() / max(1, counted.sum()), row, lse, z


def linear_xent_grad(z, lse, labels, ignored):
    """G_ij = exp(z_ij - lse_i) - [j = label_i], 0 in ignored rows, NaN in rows of labels that are no class."""
    labels = np.asarray(labels)
    inside = (labels >= 0) & (labels < z.shape[1])
    g = np.exp(z - np.asarray(lse, np.float64)[:, None])
    g[np.arange(len(labels)), np.where(inside, labels, 0)] -= 1.0
    g[~inside] = np.nan
    g[labels == ignored] = 0.0
    return g


def linear_xent_bwd(x, w, g, labels, ignored, loss_scale=1.0):
    """(dx, dw, db) for w [in, classes]."""
    a = loss_scale / max(1, int(np.sum(np.asarray(labels) != ignored)))
    x = np.where((np.asarray(labels) == ignored)[:, None], 0.0, np.asarray(x, np.float64))
    return a * (g @ np.asarray(w, np.float64).T), a * (x.T @ g), a * g.sum(axis=0)
