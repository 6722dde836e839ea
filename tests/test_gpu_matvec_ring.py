"""GPU parity: weight-only 4-bit linears whose ring of stages goes round several times, at every number of x rows.

A stage is 256 columns of K.  Sixteen to 48 rows of x leave room for four stages in flight, 64 rows for three: a CTA needs more
than six of its own before a stage's place and parity come round twice.  136 columns leave the SMs to clusters of eight (60 stages of
K, eight or fewer a CTA), 9 600 columns are 75 groups of 128, more than half the SMs: no cluster, sixteen stages in one CTA.
The tolerance is oracle.matvec.tolerance.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import matvec as OM
from paper_2604_06916_b200 import workloads

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


@pytest.mark.parametrize("fmt", ["nv", "mx"])
@pytest.mark.parametrize("M,N,K", [(16, 136, 15360), (33, 136, 15360), (49, 136, 15360), (64, 136, 15360), (70, 136, 15392), (200, 40, 13824),
                                   (64, 9600, 4096), (20, 9600, 4128)])
def test_many_stages_of_a_cta(B, fmt, M, N, K):
    rng = np.random.default_rng(M + N + K)
    q = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
    g = torch.Generator(device="cuda").manual_seed(M + K)
    x = workloads.make_activation("outlier", M, K, g, "cuda")
    if fmt == "nv":
        sf, T = rng.integers(0, 127, (N, K // 16), dtype=np.uint8), np.float32(2.0 ** -9 * 0.7)
        w = oracle.dequantize(q, sf, T)
        run = lambda: B.nvfp4_matvec(x, dq, dsf, torch.tensor([T], device="cuda"), activation=B.ACT_SILU)  # noqa: E731
        dsf = dev(oracle.sf_swizzle(sf, K))
    else:
        sf = rng.integers(115, 128, (N, K // 32), dtype=np.uint8)
        w = oracle.mxfp4_dequantize(q, sf)
        run = lambda: B.mxfp4_matvec(x, dq, dsf, activation=B.ACT_SILU)  # noqa: E731
        dsf = dev(oracle.mx_sf_swizzle(sf, K))
    dq = dev(q)
    y = run()
    ref = OM.linear(f64(x), w, None, True)
    err, tol = np.abs(f64(y) - ref), OM.tolerance(f64(x), w, ref, True, fmt == "mx")
    assert np.all(err <= tol), f"err/tol {np.max(err / tol):.3f} at {np.unravel_index((err / tol).argmax(), err.shape)}"
    for _ in range(3):
        assert torch.equal(run(), y)
    assert B.sol_last_device_status() == 0
