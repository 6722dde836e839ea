"""TEST INFRASTRUCTURE -- plain CPU statement of the per-head RMS norm and the rotary positions that precede
attention in a DiT block, and of their gradients; shares nothing with the CUDA path.

Everything in FP64 on the values of BF16 inputs:

    n = w * x / sqrt(mean(x^2) + eps)                      (w is None: n = x)
    pair (a, b) -> s (a cos t - b sin t), s (b cos t + a sin t),   t = position[axis of the pair] * freq[pair]

The turn is written as one matrix product per token (a rotation matrix built pair by pair), the gradients as
its transpose and the quotient rule -- the textbook forms, so that they share no arithmetic with the kernel.
"""
from __future__ import annotations

import numpy as np


def pair_columns(rot: int, half: bool):
    """Column indices (first, second) of the rot / 2 pairs."""
    i = np.arange(rot // 2)
    return (i, i + rot // 2) if half else (2 * i, 2 * i + 1)


def angles(positions, freqs, axis_dims):
    """[R, axes] integer positions, [rot / 2] radians per position -> [R, rot / 2] angles."""
    axis = np.repeat(np.arange(len(axis_dims)), np.asarray(axis_dims) // 2)
    return np.asarray(positions, np.float64)[:, axis] * np.asarray(freqs, np.float64)


def rotation(theta, D: int, half: bool, scale: float):
    """[R, rot / 2] angles -> [R, D, D] matrices that map a head's columns."""
    R, pairs = theta.shape
    a, b = pair_columns(2 * pairs, half)
    M = np.tile(np.eye(D), (R, 1, 1))
    c, s = scale * np.cos(theta), scale * np.sin(theta)
    M[:, a, a], M[:, b, b] = c, c
    M[:, a, b], M[:, b, a] = -s, s
    return M


def norm(x, w, eps: float):
    if w is None:
        return x, None, None
    r = 1.0 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    return x * r * w, x * r, r


def forward(x, w, M, eps: float):
    """x [rows, H, D]; M [R, D, D] (row m uses M[m % R]) or None -> (y, bound): y the exact values, bound the sum of
    the magnitudes that each output is made of."""
    n, _, _ = norm(x, w, eps)
    if M is None:
        return n, np.abs(n)
    M = M[np.arange(x.shape[0]) % M.shape[0]]
    return np.einsum("mij,mhj->mhi", M, n), np.einsum("mij,mhj->mhi", np.abs(M), np.abs(n))


def backward(dy, x, w, M, eps: float):
    """-> (dx, dw, bound of dx, bound of dw); dw is None without a weight."""
    if M is None:
        dn, mag = dy, np.abs(dy)
    else:
        M = M[np.arange(dy.shape[0]) % M.shape[0]]
        dn, mag = np.einsum("mji,mhj->mhi", M, dy), np.einsum("mji,mhj->mhi", np.abs(M), np.abs(dy))
    if w is None:
        return dn, None, mag, None
    _, xhat, r = norm(x, w, eps)
    dh = dn * w
    dx = r * (dh - xhat * (dh * xhat).mean(axis=-1, keepdims=True))
    mdh = mag * np.abs(w)
    bound = r * (mdh + np.abs(xhat) * (mdh * np.abs(xhat)).mean(axis=-1, keepdims=True))
    return dx, (dn * xhat).sum(axis=(0, 1)), bound, (mag * np.abs(xhat)).sum(axis=(0, 1))
