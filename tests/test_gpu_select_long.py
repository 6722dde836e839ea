"""GPU parity: block selection over more than 1 024 key blocks, where a CTA takes one query block instead of four, up to the
8 192 that are allowed (beyond some 6 000 the scores need more than 48 KB of shared memory).  Lists are compared for equality
with the FP64 oracle; several query blocks with a ragged end, shared key heads, lengths, ties on both sides of the cut.
"""
import numpy as np
import pytest
import torch

from oracle import block_sparse as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def check(B, q, k, cases, lens=None):
    qn, kn = f64(q), f64(k)
    for count, first in cases:
        blocks, counts, scores = B.sol_select_blocks(q, k, count, first, lens, with_scores=True)
        want, wcounts, wscores = S.select(qn, kn, count, first, None if lens is None else lens.tolist())
        assert np.array_equal(counts.cpu().numpy(), wcounts) and np.array_equal(blocks.cpu().numpy(), want)
        live = want >= 0
        assert np.all(np.abs(f64(scores)[live] - wscores[live]) <= 2.0 ** -23 * np.abs(wscores[live]) + 1e-13)
        assert torch.all(scores[blocks < 0] == -np.inf)


def randn(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16)


@pytest.mark.parametrize("blocks,tail", [(1024, 128), (1025, 1), (1100, 77)])
def test_both_sides_of_the_last_shared_size(B, blocks, tail):
    skv = 128 * (blocks - 1) + tail
    q, k = randn(blocks, 2, 530, 2, 64), randn(tail, 2, skv, 1, 64)
    check(B, q, k, [(1, 0), (40, 3), (blocks - 1, 0), (blocks + 5, 7)])
    check(B, q, k, [(40, 3)], torch.tensor([skv - 128, 131], dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("blocks,D", [(6000, 64), (6200, 128), (8192, 64), (8192, 128)])
def test_the_longest_contexts(B, blocks, D):
    q, k = randn(blocks, 1, 513, 1, D), randn(D, 1, 128 * blocks, 1, D)
    check(B, q, k, [(64, 2), (8192, 0)])
    check(B, q, k[:, :-127], [(300, 0)])


def test_ties_over_many_blocks(B):
    q, k = torch.zeros((1, 300, 1, 64), device="cuda", dtype=torch.bfloat16), torch.zeros((1, 128 * 1500, 1, 64), device="cuda", dtype=torch.bfloat16)
    q[..., 0] = 1.0
    k[0, ::128, 0, 0] = 1.0                                          # one row of a block decides its mean: all equal
    check(B, q, k, [(1, 0), (700, 3), (1500, 0)])
    k[0, 1::128, 0, 0] = (torch.arange(1500, device="cuda") % 100).to(torch.bfloat16) * 2.0 ** -40      # fifteen of each
    check(B, q, k, [(7, 0), (15, 0), (16, 0), (100, 2), (1499, 0)])
    k = -k
    check(B, q, k, [(7, 0), (100, 2)])
