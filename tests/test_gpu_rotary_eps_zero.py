"""GPU parity: the head norm and its gradients with eps = 0, where lanes without a head must still add nothing.

Were such lanes to hold zeros, the reciprocal root of their mean square would be infinite and zero times it not a number:
head counts on both sides of a step (eight heads for 128 and 64 columns, four for 256, eight for 32) and q and k with different ones.
Tolerances: those of the rotary parity tests -- BF16's half step, 2^-19 (forward) and 2^-18 (gradients) of the magnitudes
for FP32 roundings; a weight gradient 2^-24 for each of (64 + 16) roundings, its chain here being at most eight terms.
"""
import numpy as np
import pytest
import torch

from oracle import rotary as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def close(got, ref, bound, slack):
    tol = 2.0 ** -8 * np.abs(ref) + slack * bound + 1e-38
    err = np.abs(f64(got).reshape(ref.shape) - ref)
    assert np.all(err <= tol), f"err/tol {np.nanmax(err / tol):.3f}, finite: {np.isfinite(err).all()}"


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("H,Hk,D", [(12, 5, 128), (1, 1, 128), (8, 16, 128), (38, 19, 64), (9, 8, 64), (3, 1, 256), (4, 6, 256), (7, 33, 32)])
@pytest.mark.parametrize("rows", [1, 45])
def test_norm_without_epsilon(B, rows, H, Hk, D, half):
    g = torch.Generator(device="cuda").manual_seed(rows + H + Hk + D)
    mk = lambda h: torch.randn((1, rows, h, D), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    q, k, dq, dk = mk(H), mk(Hk), mk(H), mk(Hk)
    qw, kw = (torch.randn(D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    freqs, _ = B.rotary_frequencies([D // 2])
    pos = torch.arange(rows, device="cuda")[:, None]
    args = dict(layout=B.ROTARY_HALF if half else B.ROTARY_INTERLEAVED, q_weight=qw, k_weight=kw, eps=0.0)
    out = B.sol_qk_rotary(q, k, pos, freqs, **args)
    got = B.sol_qk_rotary_backward(dq, dk, q, k, pos, freqs, **args)
    M = R.rotation(R.angles(f64(pos), f64(freqs), [D // 2]), D, half, 1.0)
    for i, (x, dy, w) in enumerate(((q, dq, qw), (k, dk, kw))):
        y, bound = R.forward(f64(x)[0], f64(w), M, 0.0)
        close(out[i], y, bound, 2.0 ** -19)
        dx, dw, bound, wbound = R.backward(f64(dy)[0], f64(x)[0], f64(w), M, 0.0)
        close(got[i], dx, bound, 2.0 ** -18)
        assert torch.isfinite(got[2 + i]).all()
        assert np.all(np.abs(f64(got[2 + i]) - dw) <= (64 + 16) * 2.0 ** -24 * wbound + 1e-38)
