"""GPU parity: layer norm with modulation or a weight and its gradients through the C ABI against the FP64 oracle.

Tolerances.  An output in BF16 is off by at most half a step, 2^-8 of its value; everything else is FP32, each rounding 2^-24 of
the magnitudes that the oracle returns as `bound`.  Sums over a row: a lane adds K / 64 values one after the other (up to three
levels inside a piece of eight), then 6 steps over two halves and the warp and up to 16 over warps: chain(K) = K / 64 + 26
roundings, once for the mean, once for the variance (the gradients: for both means).  The elementwise part adds fewer than 16.
Gradients of scale and shift: a thread adds at most all rows of its sample one after the other, `rows` roundings, up to 12 groups
and FP64 over the blocks; xhat itself has the statistics' error, chain(K) + 8 roundings.
"""
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


def chain(K):
    return K / 64 + 26


def make(M, K, rows, seed, pitch=0, offset=0.3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    S = -(-M // rows)
    wide = lambda: torch.randn((M, K + pitch), generator=g, device="cuda")[:, :K]  # noqa: E731
    x = (wide() * torch.exp(0.5 * torch.randn(K, generator=g, device="cuda")) + offset * torch.randn(K, generator=g, device="cuda"))
    x = torch.cat((x, x.new_full((M, pitch), 7.0)), dim=1).to(torch.bfloat16)[:, :K]
    dy = torch.randn((M, K + pitch), generator=g, device="cuda").to(torch.bfloat16)[:, :K]
    scale = (0.3 * torch.randn((S, K), generator=g, device="cuda")).to(torch.bfloat16)
    shift = (0.3 * torch.randn((S, K), generator=g, device="cuda")).to(torch.bfloat16)
    return x, dy, scale, shift


def check_forward(x, scale, shift, rows, one, eps, y, stats):
    M, K = x.shape
    zero = np.zeros((-(-M // rows), K))
    gain = N.rows_of(zero + 1.0 if scale is None else f64(scale) + one, M, rows)
    ref, bound, mean, rstd = N.forward(f64(x), gain, N.rows_of(zero if shift is None else f64(shift), M, rows), eps)
    tol = 2.0 ** -8 * np.abs(ref) + (2 * chain(K) + 16) * U * bound + 1e-38
    err = np.abs(f64(y) - ref)
    assert np.all(err <= tol), f"err/tol {np.max(err / tol):.3f} at {np.unravel_index((err / tol).argmax(), err.shape)}"
    if stats is not None:
        s = f64(stats)
        size = np.abs(f64(x)).mean(axis=1, keepdims=True)
        assert np.all(np.abs(s[:, :1] - mean) <= (chain(K) + 2) * U * size + 1e-38)
        assert np.all(np.abs(s[:, 1:] / rstd - 1.0) <= (2 * chain(K) + 8) * U * (1.0 + rstd * size))


def check_backward(dy, x, scale, rows, one, eps, dx, dscale, dshift):
    M, K = x.shape
    gain = N.rows_of(np.ones((-(-M // rows), K)) if scale is None else f64(scale) + one, M, rows)
    ref = N.backward(f64(dy), f64(x), gain, eps, rows)
    tol = 2.0 ** -8 * np.abs(ref[0]) + (4 * chain(K) + 32) * U * ref[3] + 1e-38
    err = np.abs(f64(dx) - ref[0])
    assert np.all(err <= tol), f"dx err/tol {np.max(err / tol):.3f} at {np.unravel_index((err / tol).argmax(), err.shape)}"
    for got, want, bound in ((dscale, ref[1], ref[4]), (dshift, ref[2], ref[5])):
        if got is not None:
            assert got.dtype == torch.float32 and got.shape == want.shape
            tol = (min(rows, M) + 2 * chain(K) + 24) * U * bound + 1e-38
            err = np.abs(f64(got) - want)
            assert np.all(err <= tol), f"sum err/tol {np.max(err / tol):.3f}"


SHAPES = [  # M, K, rows per sample
    (1, 8, 1), (1, 64, 1), (1, 3072, 1), (2, 16384, 2), (3, 104, 2), (37, 264, 37), (5, 4104, 2), (333, 2432, 333), (129, 4096, 43),
    (70, 8200, 23), (9, 12296, 9), (64, 512, 1), (700, 96, 100), (1025, 768, 512),
]


@pytest.mark.parametrize("M,K,rows", SHAPES)
@pytest.mark.parametrize("one", [1.0, 0.0])
def test_forward_and_gradients(B, M, K, rows, one):
    x, dy, scale, shift = make(M, K, rows, M + K)
    y, stats = B.sol_layernorm(x, scale, shift, rows, scale_offset=one, with_stats=True)
    check_forward(x, scale, shift, rows, one, 1e-6, y, stats)
    dx, dscale, dshift = B.sol_layernorm_backward(dy, x, stats, scale, rows, scale_offset=one)
    check_backward(dy, x, scale, rows, one, 1e-6, dx, dscale, dshift)


@pytest.mark.parametrize("with_scale,with_shift", [(False, False), (True, False), (False, True)])
def test_absent_parts(B, with_scale, with_shift):
    x, dy, scale, shift = make(75, 520, 30, 5)
    scale, shift = scale if with_scale else None, shift if with_shift else None
    y, stats = B.sol_layernorm(x, scale, shift, 30, eps=1e-3, with_stats=True)
    check_forward(x, scale, shift, 30, 1.0, 1e-3, y, stats)
    assert torch.equal(B.sol_layernorm(x, scale, shift, 30, eps=1e-3), y)
    dx, dscale, dshift = B.sol_layernorm_backward(dy, x, stats, scale, 30, with_scale=with_scale, with_shift=with_shift)
    assert (dscale is None) == (not with_scale) and (dshift is None) == (not with_shift)
    check_backward(dy, x, scale, 30, 1.0, 1e-3, dx, dscale, dshift)


def test_pitches_and_in_place(B):
    x, dy, scale, shift = make(201, 1160, 67, 6, pitch=24)
    y, stats = B.sol_layernorm(x, scale, shift, 67, with_stats=True)
    check_forward(x, scale, shift, 67, 1.0, 1e-6, y, stats)
    wide = torch.full((201, 1200), 3.0, dtype=torch.bfloat16, device="cuda")
    B.sol_layernorm(x, scale, shift, 67, out=wide[:, 16:1176])
    assert torch.equal(wide[:, 16:1176], y) and (wide[:, :16] == 3.0).all() and (wide[:, 1176:] == 3.0).all()
    got = B.sol_layernorm_backward(dy, x, stats, scale, 67)
    check_backward(dy, x, scale, 67, 1.0, 1e-6, *got)
    dy2, x2 = dy.clone(), x.clone()
    for out in (dy2, x2):
        again = B.sol_layernorm_backward(dy2, x2, stats, scale, 67, out=out)
        assert all(torch.equal(a, b) for a, b in zip(again, got))
        dy2, x2 = dy.clone(), x.clone()
    x2 = x.clone()
    assert torch.equal(B.sol_layernorm(x2, scale, shift, 67, out=x2), y)


def test_large_means_constant_rows_and_values_that_are_not_numbers(B):
    x, dy, scale, shift = make(64, 1024, 64, 7)
    x = (x.float() + 300.0).to(torch.bfloat16)                 # the mean is far larger than the spread
    x[5] = 2.5                                                 # variance 0: xhat 0
    x[9, 17] = float("nan")
    x[11, 3] = float("inf")
    y, stats = B.sol_layernorm(x, scale, shift, 64, with_stats=True)
    fine = [m for m in range(64) if m not in (9, 11)]
    check_forward(x[fine], scale, shift, 64, 1.0, 1e-6, y[fine], stats[fine])
    assert torch.equal(y[5], shift[0])
    assert y[9].isnan().all() and y[11].isnan().all()
    dx = B.sol_layernorm_backward(dy, x, stats, scale, 64)[0]
    assert dx[fine].isfinite().all() and dx[9].isnan().all()
    # a plain eps of 0 is the formula's as well
    x, dy, scale, shift = make(16, 256, 16, 8)
    y, stats = B.sol_layernorm(x, scale, shift, 16, eps=0.0, with_stats=True)
    check_forward(x, scale, shift, 16, 1.0, 0.0, y, stats)


def test_same_bits_again_on_another_stream_and_captured(B):
    x, dy, scale, shift = make(2000, 640, 900, 9)
    y, stats = B.sol_layernorm(x, scale, shift, 900, with_stats=True)
    got = B.sol_layernorm_backward(dy, x, stats, scale, 900)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y2, stats2 = B.sol_layernorm(x, scale, shift, 900, with_stats=True)
        again = B.sol_layernorm_backward(dy, x, stats2, scale, 900)
    side.synchronize()
    assert torch.equal(y, y2) and torch.equal(stats, stats2) and all(torch.equal(a, b) for a, b in zip(got, again))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y3, stats3 = B.sol_layernorm(x, scale, shift, 900, with_stats=True)
        third = B.sol_layernorm_backward(dy, x, stats3, scale, 900)
    x2, dy2, scale2, shift2 = make(2000, 640, 900, 10)
    for a, b in ((x, x2), (dy, dy2), (scale, scale2), (shift, shift2)):
        a.copy_(b)
    graph.replay()
    torch.cuda.synchronize()
    check_forward(x2, scale2, shift2, 900, 1.0, 1e-6, y3, stats3)
    check_backward(dy2, x2, scale2, 900, 1.0, 1e-6, *third)


def test_rows_far_apart(B):
    """Element offsets past 32 bits: every row starts 2^26 elements behind the one before."""
    M, K, pitch = 70, 128, 1 << 26
    wide = torch.empty(M * pitch, dtype=torch.bfloat16, device="cuda").as_strided((M, K), (pitch, 1))
    x, dy, scale, shift = make(M, K, 35, 11)
    wide.copy_(x)
    y, stats = B.sol_layernorm(wide, scale, shift, 35, with_stats=True)
    check_forward(x, scale, shift, 35, 1.0, 1e-6, y, stats)
    got = B.sol_layernorm_backward(dy, wide, stats, scale, 35, out=wide)
    check_backward(dy, x, scale, 35, 1.0, 1e-6, wide, *got[1:])


def test_refused_tensors(B):
    x, dy, scale, shift = make(6, 64, 3, 12)
    stats = torch.zeros((6, 2), device="cuda")
    for bad in (dict(scale=scale[:1]), dict(scale=scale.float()), dict(shift=shift[:, :32]), dict(out=x.float()), dict(out=x[:5])):
        with pytest.raises((TypeError, ValueError)):
            B.sol_layernorm(x, rows_per_sample=3, **bad)
    with pytest.raises(ValueError):
        B.sol_layernorm(x.t())
    with pytest.raises((TypeError, ValueError)):
        B.sol_layernorm_backward(dy, x, stats[:5], scale, 3)
    with pytest.raises(B.SolError):
        B.sol_layernorm(x[:, 1:57])
    with pytest.raises(B.SolError):
        B.sol_layernorm(x, rows_per_sample=0)


@pytest.mark.parametrize("M,K,rows", [(41, 3080, 20), (37, 4096, 37), (33, 4608, 11), (29, 6144, 29), (50, 6152, 25), (31, 8192, 31), (23, 10000, 8), (21, 12288, 21), (600, 4000, 600)])
def test_every_form_of_the_gradients(B, M, K, rows):
    x, dy, scale, shift = make(M, K, rows, M + K)
    stats = B.sol_layernorm(x, scale, shift, rows, with_stats=True)[1]
    dx, dscale, dshift = B.sol_layernorm_backward(dy, x, stats, scale, rows)
    check_backward(dy, x, scale, rows, 1.0, 1e-6, dx, dscale, dshift)


def test_slices_of_one_modulation_tensor(B):
    """Scale and shift as columns of the modulation linear's output, six chunks a sample."""
    x, dy, _, _ = make(300, 328, 75, 21)
    g = torch.Generator(device="cuda").manual_seed(22)
    mod = (0.3 * torch.randn((4, 6 * 328), generator=g, device="cuda")).to(torch.bfloat16)
    shift, scale = mod.chunk(6, dim=1)[:2]
    y, stats = B.sol_layernorm(x, scale, shift, 75, with_stats=True)
    check_forward(x, scale, shift, 75, 1.0, 1e-6, y, stats)
    assert torch.equal(y, B.sol_layernorm(x, scale.contiguous(), shift.contiguous(), 75))
    got = B.sol_layernorm_backward(dy, x, stats, scale, 75)
    check_backward(dy, x, scale, 75, 1.0, 1e-6, *got)
    with pytest.raises(ValueError, match="pitch"):
        B.sol_layernorm(x, scale, shift.contiguous(), 75)
