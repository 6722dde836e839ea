"""TEST INFRASTRUCTURE -- plain CPU statement of the weight-only 4-bit linear; shares nothing with the CUDA path.

    y[m, n] = sum_k act(x[m, k]) w[n, k] + bias[n],   act = identity or x / (1 + exp(-x)),

w the dequantized weight (oracle.dequantize / oracle.mxfp4_dequantize), everything in FP64, and the bound that a
kernel which multiplies FP16 operands with FP32 sums keeps.
"""
from __future__ import annotations

import numpy as np


def silu(x):
    x = np.asarray(x, np.float64)
    with np.errstate(over="ignore"):
        return x / (1.0 + np.exp(-x))


def linear(x, w, bias=None, act: bool = False):
    h = silu(x) if act else np.asarray(x, np.float64)
    y = h @ np.asarray(w, np.float64).T
    return y if bias is None else y + np.asarray(bias, np.float64)


def tolerance(x, w, y, act: bool = False, mx: bool = False):
    """|error| bound per output.

    Output rounding to BF16: 2^-8 |y| (half a step).  FP32 sums: the tensor core adds 16 products to a sum at a time; a sum
    that truncates instead of rounding is off by at most 2^-22 of the magnitudes at each of K / 16 additions, and the
    slices, the bias and the scale add a few more.  An activation's result rounded to FP16: 2^-11 / 2 of each term, and
    2^-19 for the fast exponential and quotient.  Operands scaled into FP16: elements far below the largest of their
    slice are off by 2^-25 2^-14 of it (subnormal steps of 2^-24, values up to 2^15 scaled); doubled for a maximum
    just above a power of two.  MXFP4: blocks whose scale is far below the row's largest, 2^-25 / 2^13 of that scale.
    """
    h = np.abs(silu(x) if act else np.asarray(x, np.float64))
    aw = np.abs(np.asarray(w, np.float64))
    S = h @ aw.T
    K = aw.shape[1]
    tol = 2.0 ** -8 * np.abs(y) + S * (K / 16 + 64) * 2.0 ** -22
    if act:
        tol = tol + S * (2.0 ** -12 + 2.0 ** -19)
    tol = tol + 2.0 ** -38 * h.max(axis=1, keepdims=True) * aw.sum(axis=1)[None, :]
    if mx:
        tol = tol + 2.0 ** -38 * h.sum(axis=1, keepdims=True) * aw.max(axis=1)[None, :]
    return tol + 1e-37
