"""TEST INFRASTRUCTURE -- plain CPU statement of the layer norm with modulation (or a weight) and of its gradients, in FP64 on the
values of BF16 inputs; shares nothing with the CUDA path.

    xhat = (x - mean) / sqrt(var + eps);   y = xhat gain + shift,   gain [rows, K] the row's scale plus the offset

The gradients are the chain rule through mean and variance, written with the norm's Jacobian applied row by row (a projection onto what
is orthogonal to 1 and to xhat).  Each function also returns the magnitudes that an FP32 evaluation's roundings are relative to.
"""
from __future__ import annotations

import numpy as np


def rows_of(per_sample, rows: int, rows_per_sample: int):
    """[samples, K] -> [rows, K]: what each row uses."""
    return per_sample[np.arange(rows) // rows_per_sample]


def statistics(x, eps: float):
    mean = x.mean(axis=1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(axis=1, keepdims=True) + eps)
    return mean, rstd


def forward(x, gain, shift, eps: float):
    """-> (y, bound, mean, rstd); bound: sum of the magnitudes an output is made of, the mean's own among them."""
    mean, rstd = statistics(x, eps)
    xhat = (x - mean) * rstd
    spread = np.abs(xhat) + rstd * (np.abs(x) + np.abs(x).mean(axis=1, keepdims=True))
    return xhat * gain + shift, spread * np.abs(gain) + np.abs(shift), mean, rstd


def backward(dy, x, gain, eps: float, rows_per_sample: int):
    """-> (dx, dscale, dshift, bound of each)."""
    rows, K = x.shape
    mean, rstd = statistics(x, eps)
    xhat = (x - mean) * rstd
    off = rstd * (np.abs(x) + np.abs(mean))             # what a rounding of x rstd or of mean rstd is relative to
    w = dy * gain
    dx = np.empty_like(x)
    for m in range(rows):
        u = np.stack((np.ones(K), xhat[m])) / np.sqrt(K)
        dx[m] = rstd[m] * (w[m] - u.T @ (u @ w[m]))
    aw = np.abs(w)
    bound = rstd * (aw + aw.mean(axis=1, keepdims=True) + (np.abs(xhat) + off) * (aw * (np.abs(xhat) + off)).mean(axis=1, keepdims=True))
    starts = np.arange(0, rows, rows_per_sample)
    total = lambda v: np.add.reduceat(v, starts, axis=0)  # noqa: E731
    return dx, total(dy * xhat), total(dy), bound, total(np.abs(dy) * (np.abs(xhat) + off)), total(np.abs(dy))
