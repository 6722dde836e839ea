"""GPU parity: weight-only 4-bit linears whose operands' scales lie far apart while the result is an ordinary FP32 number.

x, the block scales and the tensor scale are each taken out as powers of two, and undoing one after another may leave FP32's
range on the way to a finite result: huge MXFP4 scales against tiny x and the other way round, x near 2^120 against a
small tensor scale.  Both forms (x prepared by the products' blocks; x prepared in a launch of its own), with K shared by
a cluster and not.  The tolerance is oracle.matvec.tolerance; results stay below 2^127.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import matvec as OM

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


def check(got, x, w, mx, bias=None, act=False):
    ref = OM.linear(f64(x), w, None if bias is None else f64(bias), act)
    assert np.abs(ref).max() < 2.0 ** 127, "the case itself leaves the range"
    err, tol = np.abs(f64(got) - ref), OM.tolerance(f64(x), w, ref, act, mx)
    assert np.all(err <= tol), f"err/tol {np.nanmax(err / tol):.3f}, finite: {np.isfinite(err).all()}"


def randn(M, K, exponent, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn((M, K), generator=g, device="cuda", dtype=torch.float64) * 2.0 ** exponent).to(torch.bfloat16)


SHAPES = [(1, 264, 416), (4, 128, 96), (8, 264, 416), (24, 40, 2240), (70, 136, 544)]


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("lo,hi,exponent", [(240, 255, -40), (245, 246, -40), (254, 255, -100), (130, 255, -60), (1, 12, 100), (1, 2, 120),
                                            (1, 255, -60)])
def test_mxfp4_scales_against_x(B, M, N, K, lo, hi, exponent):
    rng = np.random.default_rng(M + N + lo)
    q = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
    sf = rng.integers(lo, hi, (N, K // 32), dtype=np.uint8)
    w = oracle.mxfp4_dequantize(q, sf)
    x = randn(M, K, exponent, M + K)
    check(B.mxfp4_matvec(x, dev(q), dev(oracle.mx_sf_swizzle(sf, K))), x, w, True)


@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("exponent,log2_t", [(120, -20), (124, -40), (-120, 110), (-80, 120), (100, -110), (0, -130), (0, 100)])
def test_nvfp4_tensor_scale_against_x(B, M, N, K, exponent, log2_t):
    rng = np.random.default_rng(M + N)
    q = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
    sf = rng.integers(0, 127, (N, K // 16), dtype=np.uint8)
    T = np.float32(1.37 * 2.0 ** log2_t)
    w = oracle.dequantize(q, sf, 1.0) * float(T)
    x = randn(M, K, exponent, M + K)
    bias = randn(1, N, max(exponent + log2_t, -100), 5)[0]
    sf, ts = dev(oracle.sf_swizzle(sf, K)), torch.tensor([T], device="cuda")
    check(B.nvfp4_matvec(x, dev(q), sf, ts), x, w, False)
    check(B.nvfp4_matvec(x, dev(q), sf, ts, bias), x, w, False, bias)


@pytest.mark.parametrize("M", [2, 8])
def test_zero_rows_and_zero_weights_stay_zero_under_any_scale(B, M):
    # the factors that undo the scaling may be infinite by themselves: zero times them is not a number
    N, K = 136, 320
    x = randn(M, K, 100, 3)
    x[1] = 0
    for byte, log2_t in ((254, 126), (1, -126)):
        y = B.mxfp4_matvec(x, torch.zeros((N, K // 2), dtype=torch.uint8, device="cuda"),
                           dev(oracle.mx_sf_swizzle(np.full((N, K // 32), byte, np.uint8), K)))
        assert torch.all(y == 0)
        y = B.nvfp4_matvec(x, torch.zeros((N, K // 2), dtype=torch.uint8, device="cuda"),
                           dev(oracle.sf_swizzle(np.full((N, K // 16), 126, np.uint8), K)), torch.tensor([2.0 ** log2_t], device="cuda"))
        assert torch.all(y == 0)
        q = dev(np.random.default_rng(1).integers(0, 256, (N, K // 2), dtype=np.uint8))
        y = B.nvfp4_matvec(x[1:2], q, dev(oracle.sf_swizzle(np.full((N, K // 16), 126, np.uint8), K)), torch.tensor([2.0 ** log2_t], device="cuda"))
        assert torch.all(y == 0)
