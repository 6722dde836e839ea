"""GPU parity: weight-only 4-bit linears (nvfp4_matvec, mxfp4_matvec) through the C ABI against the FP64 oracle.

Weights are random codes under random scale bytes, so every code, subnormal and zero scales and wide ranges occur; the
tolerance is derived in oracle.matvec.tolerance.
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
    return None if t is None else t.detach().to(torch.float64).cpu().numpy()


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Weight:
    def __init__(self, fmt, N, K, seed, spread=None):
        rng = np.random.default_rng(seed)
        self.fmt, self.N, self.K = fmt, N, K
        q = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
        if fmt == "nv":
            sf = rng.integers(0, 127, (N, K // 16), dtype=np.uint8)        # every finite E4M3 magnitude
            T = np.float32(2.0 ** -9 * rng.uniform(0.5, 1.0))
            self.w = oracle.dequantize(q, sf, T)
            self.sf, self.ts = dev(oracle.sf_swizzle(sf, K)), torch.tensor([T], device="cuda")
        else:
            lo, hi = spread or (115, 128)
            sf = rng.integers(lo, hi, (N, K // 32), dtype=np.uint8)
            self.w = oracle.mxfp4_dequantize(q, sf)
            self.sf, self.ts = dev(oracle.mx_sf_swizzle(sf, K)), None
        self.q = dev(q)

    def call(self, B, x, bias=None, act=0, out=None):
        if self.fmt == "nv":
            return B.nvfp4_matvec(x, self.q, self.sf, self.ts, bias, act, out=out)
        return B.mxfp4_matvec(x, self.q, self.sf, bias, act, out=out)


def check(B, W, x, bias=None, act=0):
    y = W.call(B, x, bias, act)
    ref = OM.linear(f64(x), W.w, f64(bias), bool(act))
    tol = OM.tolerance(f64(x), W.w, ref, bool(act), W.fmt == "mx")
    err = np.abs(f64(y) - ref)
    assert y.shape == ref.shape and np.all(err <= tol), \
        f"err/tol {np.max(err / tol):.3f} at {np.unravel_index((err / tol).argmax(), err.shape)}"
    return y


def rows(M, K, seed, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return workloads.make_activation("outlier", M, K + pad, g, "cuda")[:, :K]


SHAPES = [(1, 8, 32), (1, 128, 128), (2, 136, 96), (3, 1000, 160), (8, 256, 512), (9, 264, 544), (16, 128, 1056), (17, 640, 2240),
          (24, 72, 320), (25, 128, 4128), (32, 2432, 1216), (33, 200, 640), (64, 512, 1024), (70, 88, 256), (5, 128, 24576), (32, 136, 15360), (48, 64, 32), (130, 40, 288), (1, 9216, 3072), (4, 4104, 3072), (2, 72, 2240), (3, 16, 992), (4, 256, 3104), (1, 40000, 64)]


@pytest.mark.parametrize("fmt", ["nv", "mx"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_against_the_oracle(B, fmt, M, N, K):
    W = Weight(fmt, N, K, M + N + K)
    x = rows(M, K, N, pad=8 * (M % 3))
    bias = (0.5 * torch.randn(N, device="cuda")).to(torch.bfloat16)
    check(B, W, x, bias, B.ACT_NONE)
    check(B, W, x, None, B.ACT_SILU)


@pytest.mark.parametrize("fmt", ["nv", "mx"])
def test_quantized_weights_and_the_linear_of_quantized_rows(B, fmt):
    # the weight as the library quantizes it; the token linear on the same weight agrees within what quantizing x costs
    M, N, K = 24, 768, 1536
    g = torch.Generator(device="cuda").manual_seed(3)
    w = (torch.randn((N, K), generator=g, device="cuda") * K ** -0.5).to(torch.bfloat16)
    x = torch.randn((M, K), generator=g, device="cuda").to(torch.bfloat16)
    if fmt == "nv":
        q, sf, ts = B.nvfp4_quantize_weight(w)
        y = B.nvfp4_matvec(x, q, sf, ts)
        token = B.nvfp4_quantize_linear(x, q, sf, ts)
        _, sfr, _ = B.nvfp4_quantize_weight(w, B.SF_ROW_MAJOR)
        deq = oracle.dequantize(q.cpu().numpy(), sfr.cpu().numpy().reshape(N, K // 16), np.float32(ts.item()))
    else:
        q, sf = B.mxfp4_quantize(w)
        y = B.mxfp4_matvec(x, q, sf)
        token = B.mxfp4_linear(*B.mxfp4_quantize(x), q, sf)
        _, sfr = B.mxfp4_quantize(w, B.SF_ROW_MAJOR)
        deq = oracle.mxfp4_dequantize(q.cpu().numpy(), sfr.cpu().numpy().reshape(N, K // 32))
    ref = OM.linear(f64(x), deq)
    assert np.all(np.abs(f64(y) - ref) <= OM.tolerance(f64(x), deq, ref, mx=fmt == "mx"))
    rel = ((y.float() - token.float()).norm() / y.float().norm()).item()
    assert 0.01 < rel < 0.3, rel


def test_powers_of_two_are_exact(B):
    # one element per row, any exponent: y = x w exactly, from 2^-100 to 2^100
    N, K = 128, 256
    for fmt in ("nv", "mx"):
        W = Weight(fmt, N, K, 5)
        x = torch.zeros((32, K), dtype=torch.bfloat16, device="cuda")
        for m in range(32):
            x[m, (37 * m) % K] = (-1.0) ** m * 2.0 ** (-100 + m * 200 / 31 // 1)
        got = f64(W.call(B, x))
        want = torch.from_numpy(f64(x) @ W.w.T).to(torch.bfloat16).to(torch.float64).numpy()
        # FP32 holds the product; NVFP4's T multiplies after the sum: one FP32 rounding before the BF16 one
        assert np.all(np.abs(got - want) <= 2.0 ** -7 * np.abs(want))
        if fmt == "mx":
            assert np.array_equal(got, want)


@pytest.mark.parametrize("lo,hi", [(0, 40), (100, 140), (90, 165), (200, 214)])
def test_mxfp4_scales_of_any_size(B, lo, hi):
    # whole rows of tiny or huge scales, and rows that mix scales 2^75 apart; sums stay within FP32
    W = Weight("mx", 264, 416, lo + hi, spread=(lo, hi))
    x = rows(3, 416, 7)
    check(B, W, (x.float() * 2.0 ** (60 if hi <= 40 else -20 if lo >= 200 else 0)).to(torch.bfloat16))


def test_rows_far_apart_do_not_disturb_each_other(B):
    # scales of x rows and of weight rows are kept row by row
    W = Weight("mx", 128, 512, 11, spread=(120, 124))
    sf = np.full((128, 16), 60, np.uint8)
    sf[::2] = 180
    W.sf = dev(oracle.mx_sf_swizzle(sf, 512))
    W.w = oracle.mxfp4_dequantize(W.q.cpu().numpy(), sf)
    x = rows(8, 512, 13)
    x = (x.float() * torch.tensor([2.0 ** (8 * i - 30) for i in range(8)], device="cuda")[:, None]).to(torch.bfloat16)
    check(B, W, x)


def test_silu_extremes(B):
    K = 128
    W = Weight("nv", 64, K, 17)
    x = torch.zeros((6, K), dtype=torch.bfloat16, device="cuda")
    x[0] = -60.0                      # silu = -5e-25: the row's own scale keeps it
    x[1] = 300.0
    x[2] = -1e4                       # underflows to -0
    x[3, ::2] = 30.0
    x[3, 1::2] = -30.0
    x[4] = torch.linspace(-8, 8, K, device="cuda")
    y = check(B, W, x, None, B.ACT_SILU)
    assert torch.all(y[2] == 0) and torch.all(y[5] == 0)


def test_output_pitch_bias_and_rows_behind(B):
    W = Weight("nv", 200, 320, 19)
    x = rows(11, 320, 3, pad=40)
    bias = torch.randn(200, device="cuda").to(torch.bfloat16)
    want = W.call(B, x, bias)
    wide = torch.full((14, 256), 9.0, dtype=torch.bfloat16, device="cuda")
    got = W.call(B, x, bias, out=wide[1:12, 8:208])
    assert torch.equal(got, want)
    assert torch.all(wide[0] == 9) and torch.all(wide[12:] == 9) and torch.all(wide[:, :8] == 9) and torch.all(wide[:, 208:] == 9)
    one = W.call(B, x[3:4], bias)
    assert torch.equal(one, want[3:4])            # a row's result does not depend on its neighbours
    col = torch.empty((320, 1), dtype=torch.bfloat16, device="cuda")
    col[:, 0] = x[3]
    with pytest.raises(TypeError):
        W.call(B, col.t()[:, ::2])


@pytest.mark.parametrize("fmt,M,N,K", [("nv", 8, 1024, 3200), ("mx", 40, 512, 2432)])
def test_repeatable_on_another_stream_and_captured(B, fmt, M, N, K):
    W = Weight(fmt, N, K, 23)
    x = rows(M, K, 5)
    want = W.call(B, x, act=B.ACT_SILU)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = W.call(B, x, act=B.ACT_SILU)
    side.synchronize()
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = W.call(B, x, act=B.ACT_SILU)
    got.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_workspaces_of_two_streams_and_a_small_one(B):
    # two calls at once, each with a workspace of its own; and one that is too small is refused
    W = Weight("nv", 4096, 1024, 31)
    a, b = rows(8, 1024, 41), rows(20, 1024, 42)
    wa, wb = W.call(B, a), W.call(B, b)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for i in range(20):
        with torch.cuda.stream(s1):
            got.append((W.call(B, a), wa))
        with torch.cuda.stream(s2):
            got.append((W.call(B, b), wb))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in got)
    ws = torch.empty(B.matvec_workspace_bytes(8, 1024), dtype=torch.uint8, device="cuda")
    assert torch.equal(B.nvfp4_matvec(a, W.q, W.sf, W.ts, workspace=ws), wa)
    with pytest.raises(B.SolError):
        B.nvfp4_matvec(a, W.q, W.sf, W.ts, workspace=ws[:-256])


def test_weight_beyond_32_bit_offsets(B):
    # 2^32 bytes of codes and more: rows near the end are addressed in 64 bits
    N, K = 720896, 12288                           # 4.4 GB of codes
    q = torch.zeros((N, K // 2), dtype=torch.uint8, device="cuda")
    sf = torch.zeros(B.scale_bytes(N, K), dtype=torch.uint8, device="cuda")
    small = Weight("nv", 128, K, 29)
    q[-128:] = small.q
    sf[-small.sf.numel():] = small.sf.reshape(-1)
    x = rows(2, K, 9)
    y = B.nvfp4_matvec(x, q, sf, small.ts)
    assert torch.equal(y[:, -128:], small.call(B, x)) or (y[:, -128:].float() - small.call(B, x).float()).abs().max() <= 2.0 ** -7 * y.float().abs().max()
    ref = OM.linear(f64(x), small.w)
    assert np.all(np.abs(f64(y[:, -128:]) - ref) <= OM.tolerance(f64(x), small.w, ref))
    assert torch.all(y[:, :-128] == 0)
