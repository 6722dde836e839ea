"""TEST INFRASTRUCTURE -- plain CPU statement of low-rank adapters of many requests and of their gradients, in FP64 on the values of
BF16 inputs; shares nothing with the CUDA path.  Request by request, with the adapter's full update matrix s B A where the result allows it.

Each result comes with the magnitude that FP32 roundings are relative to: the same sums over absolute values.
"""
from __future__ import annotations

import numpy as np


def requests(offsets, ids, rows: int, adapters: int):
    """(slice of rows, adapter) of every request that has both."""
    for i, a in enumerate(ids):
        begin = min(max(int(offsets[i]), 0), rows)
        end = min(max(int(offsets[i + 1]), begin), rows)
        if 0 <= a < adapters and end > begin:
            yield slice(begin, end), int(a)


def apply(x, A, B, scaling, offsets, ids, y):
    """-> (new y, magnitude of the update, t, magnitude of t)."""
    out, size = y.copy(), np.zeros_like(y)
    t, t_size = (np.zeros((x.shape[0], A.shape[1])) for _ in range(2))
    for rows, a in requests(offsets, ids, x.shape[0], A.shape[0]):
        out[rows] += x[rows] @ (scaling[a] * (B[a] @ A[a])).T
        t[rows], t_size[rows] = x[rows] @ A[a].T, np.abs(x[rows]) @ np.abs(A[a]).T
        size[rows] = abs(scaling[a]) * t_size[rows] @ np.abs(B[a]).T
    return out, size, t, t_size


def backward(dy, x, t, A, B, scaling, offsets, ids, dx):
    """-> (dA, dB, new dx) and the magnitudes of their sums; t as the forward call gave it."""
    da, db = np.zeros(A.shape), np.zeros(B.shape)
    da_size, db_size = np.zeros(A.shape), np.zeros(B.shape)
    out, size = dx.copy(), np.zeros_like(dx)
    for rows, a in requests(offsets, ids, x.shape[0], A.shape[0]):
        s = scaling[a]
        da[a] += s * B[a].T @ (dy[rows].T @ x[rows])
        db[a] += s * dy[rows].T @ t[rows]
        out[rows] += dy[rows] @ (s * (B[a] @ A[a]))
        dt_size = abs(s) * np.abs(dy[rows]) @ np.abs(B[a])
        da_size[a] += dt_size.T @ np.abs(x[rows])
        db_size[a] += abs(s) * np.abs(dy[rows]).T @ np.abs(t[rows])
        size[rows] = dt_size @ np.abs(A[a])
    return da, db, out, da_size, db_size, size
