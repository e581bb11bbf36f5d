"""fp64 reference of the decode linear layers, y = x . w^T (the projections whose flops the paper's
T_compute^d counts as BS * (8 h1^2 + 4 h1 h2) per layer, Section IV-C).

TEST INFRASTRUCTURE ONLY.  The definition written out: every output is the plain dot product of a
token row with a weight row, accumulated in fp64 over inputs widened exactly from their 16-bit
values.  ``numpy.matmul`` serves as the contraction step.
"""
from __future__ import annotations

import numpy as np

from .attn import to_f64


def linear(x, w) -> np.ndarray:
    """x [M, K], w [N, K] (fp16 numpy, bf16 torch or float arrays) -> y [M, N] float64."""
    x64 = to_f64(x)
    w64 = to_f64(w)
    assert x64.ndim == 2 and w64.ndim == 2 and x64.shape[1] == w64.shape[1]
    return np.matmul(x64, w64.T)


def linear_flops_per_layer(BS: int, h1: int, h2: int) -> float:
    """Flops of one layer's decode projections: QKV (3 h1^2), output (h1^2) and the two MLP
    matrices (2 h1 h2), two flops per multiply-add: BS * (8 h1^2 + 4 h1 h2)."""
    return 2.0 * BS * (3 * h1 * h1 + h1 * h1 + 2 * h1 * h2)


def linear4(x, w4: np.ndarray, scales, group: int) -> np.ndarray:
    """x [M, K], w4 uint8 [N, K / 2] (even k in the low four bits), scales [N, K / group] -> y [M, N] float64 with
    w[n][k] = (u[n][k] - 8) * scale[n][k / group]."""
    u = np.empty((w4.shape[0], 2 * w4.shape[1]), np.float64)
    u[:, 0::2] = w4 & 15
    u[:, 1::2] = w4 >> 4
    w = (u - 8.0) * np.repeat(to_f64(scales), group, axis=1)
    return np.matmul(to_f64(x), w.T)


def linear4_error(x, w4: np.ndarray, scales, group: int) -> np.ndarray:
    """How far fp32 sums may be from :func:`linear4`: K exact products are summed with at most 2^-23 of the running
    magnitude lost per addition (2^-24 by rounding, twice that where a sum truncates), and each of the K / group
    scalings rounds once: (K + K / group + 64) * 2^-23 of the sum of the magnitudes."""
    u = np.empty((w4.shape[0], 2 * w4.shape[1]), np.float64)
    u[:, 0::2] = w4 & 15
    u[:, 1::2] = w4 >> 4
    K = u.shape[1]
    w = np.abs(u - 8.0) * np.repeat(np.abs(to_f64(scales)), group, axis=1)
    return (K + K // group + 64) * 2.0 ** -23 * np.matmul(np.abs(to_f64(x)), w.T)


def linear4_typical(x, w4: np.ndarray, scales, group: int) -> np.ndarray:
    """How far sums in fp32 may be from :func:`linear4`, output by output, when their roundings are independent (what
    :func:`linear4_error` bounds is the worst case).  A running sum stays near r = root of the sum of the squared terms, or near the
    largest partial sum where that is more; each of the K / 16 steps rounds by at most 2^-23 of it, and independent
    roundings add like the root of their number: 4 * sqrt(K / 16) * 2^-23 of it, and 8 more for the last sums."""
    u = np.empty((w4.shape[0], 2 * w4.shape[1]), np.float64)
    u[:, 0::2] = w4 & 15
    u[:, 1::2] = w4 >> 4
    K = u.shape[1]
    w = (u - 8.0) * np.repeat(to_f64(scales), group, axis=1)
    x = to_f64(x)
    size = np.sqrt(np.matmul(np.square(x), np.square(w).T))
    part = np.zeros_like(size)
    for k in range(0, K, group):
        part += np.matmul(x[:, k:k + group], w[:, k:k + group].T)
        size = np.maximum(size, np.abs(part))
    return (8 + 4 * np.sqrt(K / 16)) * 2.0 ** -23 * size
