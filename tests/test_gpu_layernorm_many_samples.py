"""GPU parity: gradients of the norm where samples outnumber the SMs, so that a block takes several, one after the other: their sums share
its registers, its shared memory and its two buffers.  Tolerances as in the norm's other tests."""
import numpy as np
import pytest
import torch

from oracle import layernorm as N

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


@pytest.mark.parametrize("M,K,rows", [(900, 96, 3), (901, 256, 3), (1000, 1032, 4), (1499, 2432, 10), (600, 4000, 2), (455, 6144, 3), (301, 8192, 2),
                                      (460, 12288, 3), (310, 16384, 2), (149, 520, 1), (2000, 264, 1), (7777, 768, 51)])
@pytest.mark.parametrize("with_scale", [True, False])
def test_more_samples_than_sms(B, M, K, rows, with_scale):
    samples = -(-M // rows)
    assert samples > 148
    g = torch.Generator(device="cuda").manual_seed(M + K)
    x, dy = ((torch.randn((M, K), generator=g, device="cuda") + 0.2).to(torch.bfloat16) for _ in range(2))
    scale = (0.3 * torch.randn((samples, K), generator=g, device="cuda")).to(torch.bfloat16) if with_scale else None
    stats = B.sol_layernorm(x, scale, None, rows, with_stats=True)[1]
    dx, dscale, dshift = B.sol_layernorm_backward(dy, x, stats, scale, rows)
    gain = N.rows_of(np.ones((samples, K)) if scale is None else f64(scale) + 1.0, M, rows)
    ref = N.backward(f64(dy), f64(x), gain, 1e-6, rows)
    chain = K / 64 + 26
    tol = 2.0 ** -8 * np.abs(ref[0]) + (4 * chain + 32) * U * ref[3] + 1e-38
    assert np.all(np.abs(f64(dx) - ref[0]) <= tol)
    for got, want, bound in ((dscale, ref[1], ref[4]), (dshift, ref[2], ref[5])):
        assert np.all(np.abs(f64(got) - want) <= (rows + 2 * chain + 24) * U * bound + 1e-38)
    again = B.sol_layernorm_backward(dy, x, stats, scale, rows)
    assert all(torch.equal(a, b) for a, b in zip((dx, dscale, dshift), again))
