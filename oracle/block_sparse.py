"""TEST INFRASTRUCTURE -- plain CPU statement of block selection and block-sparse attention; shares nothing with the
CUDA path.

Query blocks of 256 tokens, key blocks of 128; per batch element and head the score of a pair of blocks is the dot product
of the mean query row and the mean key row; a query block keeps the `count` highest-scored key blocks (the first
`keep_first` always; among equal scores the lower index) and attends to their keys alone.  FP64 throughout.
"""
from __future__ import annotations

import numpy as np

from . import attention as dense

QUERY_BLOCK, KEY_BLOCK = 256, 128


def means(x, size):
    """[S, d] -> [ceil(S / size), d] means of the rows that exist."""
    return np.stack([x[i:i + size].sum(axis=0) / len(x[i:i + size]) for i in range(0, len(x), size)]) if len(x) else np.zeros((0, x.shape[1]))


def scores(q, k):
    """q [Sq, d], k [Skv, d] of one head -> [query blocks, key blocks].  Every pair is summed the same way (a library
    matrix product may round equal columns differently by their place): equal blocks have equal scores."""
    a, b = means(np.asarray(q, np.float64), QUERY_BLOCK), means(np.asarray(k, np.float64), KEY_BLOCK)
    return np.stack([(row * b).sum(axis=1) for row in a])


def choose(row, count, keep_first):
    """Scores of one query block -> the chosen key blocks, ascending."""
    forced = list(range(min(keep_first, len(row), count)))
    rest = sorted((j for j in range(len(forced), len(row))), key=lambda j: (-row[j], j))
    return sorted(forced + rest[:max(0, min(count, len(row)) - len(forced))])


def select(q, k, count, keep_first=0, lens=None):
    """q [B, Sq, H, d], k [B, Skv, Hk, d] -> (lists with -1 behind the last, counts, scores with -inf behind the last)."""
    B, Sq, H, _ = q.shape
    Skv, Hk = k.shape[1], k.shape[2]
    nq = -(-Sq // QUERY_BLOCK)
    lists = np.full((B, H, nq, count), -1, np.int32)
    counts = np.zeros((B, H, nq), np.int32)
    values = np.full((B, H, nq, count), -np.inf)
    for b in range(B):
        n = Skv if lens is None else min(max(int(lens[b]), 0), Skv)
        for h in range(H):
            s = scores(q[b, :, h], k[b, :n, h * Hk // H])
            for i in range(nq):
                got = choose(s[i] if n else [], count, keep_first)
                lists[b, h, i, :len(got)], counts[b, h, i], values[b, h, i, :len(got)] = got, len(got), s[i, got] if n else []
    return lists, counts, values


def attend(q, k, v, lists, counts, lens=None):
    """Attention over the listed blocks (a block listed twice counts twice); zeros where no key is listed."""
    B, Sq, H, d = q.shape
    Skv, Hk = k.shape[1], k.shape[2]
    out = np.zeros((B, Sq, H, d))
    for b in range(B):
        n = Skv if lens is None else min(max(int(lens[b]), 0), Skv)
        for h in range(H):
            hk = h * Hk // H
            for i in range(lists.shape[2]):
                c = min(max(int(counts[b, h, i]), 0), lists.shape[3])
                keys = [t for e in lists[b, h, i, :c] if 0 <= e for t in range(e * KEY_BLOCK, min((e + 1) * KEY_BLOCK, n))]
                if keys:
                    rows = slice(i * QUERY_BLOCK, min(Sq, (i + 1) * QUERY_BLOCK))
                    out[b, rows, h] = dense.attention_head(q[b, rows, h], k[b, keys, hk], v[b, keys, hk])
    return out
