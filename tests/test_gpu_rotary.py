"""GPU parity: head norm + rotary positions and their gradients through the C ABI against the FP64 oracle.

Tolerances.  An output is rounded once to BF16: at most 2^-8 of its value.  Before that it is FP32: the mean of
squares (at most 8 + log2(32) sequential roundings), root, quotient, two products for the norm, sine and cosine of an
angle reduced to half a turn (2 ulp, and the reduced angle's own rounding, at most pi 2^-24 absolute) and two
products and a sum: under 32 roundings of 2^-24, each relative to the magnitudes the output is made of (`bound`), so
2^-19 of those.  Gradients pass through two such chains, 2^-18.  A weight gradient also sums its terms in FP32 along
a lane's chain: `chain` more roundings of 2^-24.
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
    return None if t is None else t.detach().to(torch.float64).cpu().numpy()


def make(Bt, S, H, Hk, D, seed, fused=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if fused:   # slices of one projection output [B, S, (H + 2 Hk) D]
        x = torch.randn((Bt, S, (H + 2 * Hk) * D), generator=g, device="cuda").to(torch.bfloat16)
        q, k = x[:, :, :H * D].unflatten(2, (H, D)), x[:, :, H * D:(H + Hk) * D].unflatten(2, (Hk, D))
    else:
        q = torch.randn((Bt, S, H, D), generator=g, device="cuda").to(torch.bfloat16)
        k = torch.randn((Bt, S, Hk, D), generator=g, device="cuda").to(torch.bfloat16)
    qw = (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16)
    kw = (1 + 0.3 * torch.randn(D, generator=g, device="cuda")).to(torch.bfloat16)
    return q, k, qw, kw


def positions(rows, axes, seed, far=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 5)
    return far + torch.randint(0, 700, (rows, axes), generator=g, device="cuda", dtype=torch.int64)


def close(got, ref, bound, slack):
    err = np.abs(f64(got).reshape(ref.shape) - ref)
    tol = 2.0 ** -8 * np.abs(ref) + slack * bound + 1e-38
    assert np.all(err <= tol), f"err/tol {np.max(err / tol):.3f} at {np.unravel_index((err / tol).argmax(), err.shape)}"


def check_forward(B, q, k, pos, freqs, dims, half, qw, kw, scale=1.0, eps=1e-6, out=None):
    qo, ko = B.sol_qk_rotary(q, k, pos, freqs, dims, B.ROTARY_HALF if half else B.ROTARY_INTERLEAVED, qw, kw, eps, scale, out=out)
    M = None if pos is None else R.rotation(R.angles(f64(pos), f64(freqs), dims or [2 * len(freqs)]), q.shape[3], half, scale)
    for x, w, o in ((q, qw, qo), (k, kw, ko)):
        if x is not None and out is None:
            ref, bound = R.forward(f64(x).reshape(-1, x.shape[2], x.shape[3]), f64(w), M, eps)
            close(o, ref, bound, 2.0 ** -19)
    return qo, ko


def check_backward(B, dq, dk, q, k, pos, freqs, dims, half, qw, kw, scale=1.0, eps=1e-6, chain=16):
    got = B.sol_qk_rotary_backward(dq, dk, q, k, pos, freqs, dims, B.ROTARY_HALF if half else B.ROTARY_INTERLEAVED, qw, kw, eps, scale)
    M = None if pos is None else R.rotation(R.angles(f64(pos), f64(freqs), dims or [2 * len(freqs)]), dq.shape[3], half, scale)
    for i, (dy, x, w) in enumerate(((dq, q, qw), (dk, k, kw))):
        if dy is None:
            assert got[i] is None and got[2 + i] is None
            continue
        H, D = dy.shape[2], dy.shape[3]
        dx, dw, bound, wbound = R.backward(f64(dy).reshape(-1, H, D), None if w is None else f64(x).reshape(-1, H, D), f64(w), M, eps)
        close(got[i], dx, bound, 2.0 ** -18)
        if w is None:
            assert got[2 + i] is None
        else:
            assert got[2 + i].dtype == torch.float32
            assert np.all(np.abs(f64(got[2 + i]) - dw) <= (64 + chain) * 2.0 ** -24 * wbound + 1e-38)
    return got


GEOMETRIES = [
    # B, S, H, Hk, D, axis dims, half, far
    (1, 1, 1, 1, 32, [8], False, 0),
    (1, 1, 24, 24, 128, [16, 56, 56], False, 0),
    (2, 37, 24, 24, 128, [16, 56, 56], False, 0),
    (3, 5, 38, 19, 64, [32], True, 0),
    (1, 130, 7, 1, 64, [64], True, 3_999_000),
    (2, 9, 5, 5, 256, [128], False, 1 << 20),
    (1, 33, 3, 3, 256, [10, 14, 24, 16], True, 0),
    (4, 3, 33, 11, 32, [32], True, 100_000),
    (1, 11, 17, 17, 32, [6, 10], False, 0),
    (1, 300, 9, 3, 128, [128], True, 0),
]


@pytest.mark.parametrize("geo", GEOMETRIES, ids=lambda g: "x".join(map(str, g[:5])))
@pytest.mark.parametrize("normed", ["both", "none", "q"])
def test_forward(B, geo, normed):
    Bt, S, H, Hk, D, dims, half, far = geo
    q, k, qw, kw = make(Bt, S, H, Hk, D, sum(geo[:5]))
    freqs, _ = B.rotary_frequencies(dims)
    check_forward(B, q, k, positions(S, len(dims), 1, far), freqs, dims, half, qw if normed != "none" else None,
                  kw if normed == "both" else None, scale=1.25)


@pytest.mark.parametrize("geo", GEOMETRIES, ids=lambda g: "x".join(map(str, g[:5])))
@pytest.mark.parametrize("normed", ["both", "none", "k"])
def test_backward(B, geo, normed):
    Bt, S, H, Hk, D, dims, half, far = geo
    q, k, qw, kw = make(Bt, S, H, Hk, D, 3 * sum(geo[:5]))
    dq, dk, _, _ = make(Bt, S, H, Hk, D, 7 * sum(geo[:5]), fused=False)
    freqs, _ = B.rotary_frequencies(dims)
    check_backward(B, dq, dk, q, k, positions(S, len(dims), 2, far), freqs, dims, half, kw if normed == "both" else None,
                   kw if normed != "none" else None, scale=0.75)


def test_gradients_against_differences_of_the_kernel_itself(B):
    # d/dt of <forward(x + t e), dy> over bumps large enough to survive the BF16 outputs, at FP64 sums of many outputs
    q, k, qw, _ = make(1, 64, 4, 4, 64, 5, fused=False)
    dy = torch.randn_like(q.float()).to(torch.bfloat16)
    freqs, _ = B.rotary_frequencies([64])
    pos = positions(64, 1, 3)
    g = B.sol_qk_rotary_backward(dy, None, q, None, pos, freqs, q_weight=qw)[0].double()
    e = torch.randn_like(q.float())
    t = 2.0 ** -4
    hi, lo = (q.float() + t * e).to(torch.bfloat16), (q.float() - t * e).to(torch.bfloat16)
    f = lambda x: (B.sol_qk_rotary(x, None, pos, freqs, q_weight=qw)[0].double() * dy.double()).sum()  # noqa: E731
    slope, want = (f(hi) - f(lo)).item(), (g * (hi.double() - lo.double())).sum().item()
    # each of the 16384 outputs is off by at most 2^-8 of itself on each side, at random: 6 deviations of the sum; and
    # the third derivative of the norm, t^2 e^2 / x^2 of the slope
    y = B.sol_qk_rotary(q, None, pos, freqs, q_weight=qw)[0].double()
    noise = 6 * 2.0 ** -8 * (2 * (y * dy.double()).square().sum()).sqrt().item()
    assert abs(slope - want) <= noise + 0.03 * (g * (hi.double() - lo.double())).square().sum().sqrt().item() * 4
    assert abs(want) > 0


def test_norm_alone_and_no_key(B):
    q, k, qw, kw = make(2, 19, 6, 6, 64, 11)
    check_forward(B, q, k, None, None, None, False, qw, kw)
    qo, ko = check_forward(B, q, None, None, None, None, False, qw, None, eps=0.5)
    assert ko is None
    check_backward(B, q.contiguous(), None, q, None, None, None, None, False, qw, None, eps=0.5)
    check_backward(B, q.contiguous(), k.contiguous(), q, k, None, None, None, True, qw, kw)
    with pytest.raises(B.SolError):
        B.sol_qk_rotary(q, None, None, None)


def test_far_positions_keep_their_angle(B):
    # position p and p + 2^20 turn by angles that differ by an exact number of turns where freq = 2 pi j / 2^20
    S, D = 64, 32
    j = torch.arange(1, D // 2 + 1, device="cuda", dtype=torch.float64) * 977
    freqs = j * (2 * np.pi / 2 ** 20)
    q, _, _, _ = make(1, S, 2, 2, D, 13, fused=False)
    pos = torch.arange(S, device="cuda")[:, None]
    near = B.sol_qk_rotary(q, None, pos, freqs)[0].float()
    far = B.sol_qk_rotary(q, None, pos + (1 << 22), freqs)[0].float()
    # FP64: 2^22 * 0.1 rad carries 2^-53 relative = 5e-11 rad: only BF16 ties can fall the other way
    assert (near - far).abs().max() <= 2.0 ** -7 * near.abs().max()
    assert (near != far).float().mean() < 1e-2
    big = B.sol_qk_rotary(q, None, pos - (1 << 22), freqs)[0].float()     # negative positions as well
    assert (near != big).float().mean() < 1e-2


def test_position_tables_shared_and_per_token(B):
    Bt, S, H, D = 3, 20, 4, 64
    q, k, qw, kw = make(Bt, S, H, H, D, 17)
    freqs, _ = B.rotary_frequencies([64])
    shared = positions(S, 1, 9)
    a = B.sol_qk_rotary(q, k, shared, freqs, q_weight=qw, k_weight=kw)
    b = B.sol_qk_rotary(q, k, shared.repeat(Bt, 1), freqs, q_weight=qw, k_weight=kw)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    check_forward(B, q, k, positions(Bt * S, 1, 10), freqs, None, True, qw, kw)
    check_forward(B, q, k, positions(1, 1, 10), freqs, None, True, qw, kw)      # one row for every token
    with pytest.raises(ValueError):
        B.sol_qk_rotary(q, k, positions(S + 1, 1, 10), freqs)


@pytest.mark.parametrize("half", [False, True])
def test_in_place_and_into_a_wider_buffer(B, half):
    Bt, S, H, Hk, D = 2, 31, 6, 2, 128
    q, k, qw, kw = make(Bt, S, H, Hk, D, 19)
    freqs, _ = B.rotary_frequencies([96])
    pos, lay = positions(S, 1, 4), B.ROTARY_HALF if half else B.ROTARY_INTERLEAVED
    want = B.sol_qk_rotary(q, k, pos, freqs, layout=lay, q_weight=qw, k_weight=kw)
    dwant = B.sol_qk_rotary_backward(want[0], want[1], q, k, pos, freqs, layout=lay, q_weight=qw, k_weight=kw)
    wide = torch.full((Bt, S, 2048), 3.0, dtype=torch.bfloat16, device="cuda")
    oq, ok = wide[:, :, 64:64 + H * D].unflatten(2, (H, D)), wide[:, :, 1024:1024 + Hk * D].unflatten(2, (Hk, D))
    got = B.sol_qk_rotary(q, k, pos, freqs, layout=lay, q_weight=qw, k_weight=kw, out=(oq, ok))
    assert got[0] is oq and torch.equal(oq, want[0]) and torch.equal(ok, want[1])
    assert torch.all(wide[:, :, :64] == 3) and torch.all(wide[:, :, 64 + H * D:1024] == 3) and torch.all(wide[:, :, 1024 + Hk * D:] == 3)
    # gradients into the buffers of the incoming ones
    dq, dk = want[0].clone(), want[1].clone()
    got = B.sol_qk_rotary_backward(dq, dk, q, k, pos, freqs, layout=lay, q_weight=qw, k_weight=kw, out=(dq, dk))
    assert all(torch.equal(x, y) for x, y in zip(got, dwant))
    base = q._base.clone()
    v = base[:, :, (H + Hk) * D:].clone()
    q2, k2 = base[:, :, :H * D].unflatten(2, (H, D)), base[:, :, H * D:(H + Hk) * D].unflatten(2, (Hk, D))
    B.sol_qk_rotary(q2, k2, pos, freqs, layout=lay, q_weight=qw, k_weight=kw, out=(q2, k2))
    assert torch.equal(q2, want[0]) and torch.equal(k2, want[1]) and torch.equal(base[:, :, (H + Hk) * D:], v)


def test_zero_rows_large_and_non_finite_values(B):
    q, _, qw, _ = make(1, 8, 2, 2, 64, 23, fused=False)
    freqs, _ = B.rotary_frequencies([64])
    pos = positions(8, 1, 6)
    q[0, 0] = 0
    q[0, 1] *= 2.0 ** 60            # squares near 2^120: still FP32
    q[0, 2] *= 2.0 ** -50
    check_forward(B, q, None, pos, freqs, None, False, qw, None)
    q[0, 3, 0, 5] = float("inf")
    q[0, 4, 1, 6] = float("nan")
    out = B.sol_qk_rotary(q, None, pos, freqs, q_weight=qw)[0]
    assert torch.isnan(out[0, 4, 1]).all() and not torch.isfinite(out[0, 3, 0]).all()
    keep = torch.ones((8, 2), dtype=torch.bool, device="cuda")
    keep[3, 0] = keep[4, 1] = False
    assert torch.isfinite(out[0][keep]).all()      # other heads of the same tokens are not touched


def test_repeatable_on_another_stream_and_captured(B):
    q, k, qw, kw = make(2, 500, 24, 24, 128, 29)
    dq, dk = q.contiguous(), k.contiguous()
    freqs, _ = B.rotary_frequencies([16, 56, 56])
    pos = positions(500, 3, 8)
    args = (pos, freqs, [16, 56, 56], B.ROTARY_INTERLEAVED, qw, kw)
    want, dwant = B.sol_qk_rotary(q, k, *args), B.sol_qk_rotary_backward(dq, dk, q, k, *args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, dgot = B.sol_qk_rotary(q, k, *args), B.sol_qk_rotary_backward(dq, dk, q, k, *args)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want + dwant, got + dgot))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.sol_qk_rotary(q, k, *args)
        dgot = B.sol_qk_rotary_backward(dq, dk, q, k, *args)
    for t in got + dgot:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want + dwant, got + dgot))


def test_offsets_beyond_32_bits(B):
    # a pitch that puts the last token past 2^32 elements of its buffer
    S, H, D = 5, 2, 64
    pitch = (1 << 30) + 64
    big = torch.empty((S - 1) * pitch + H * D, dtype=torch.bfloat16, device="cuda")
    view = big.as_strided((1, S, H, D), (S * pitch, pitch, D, 1))
    q, _, qw, _ = make(1, S, H, H, D, 31, fused=False)
    view.copy_(q)
    freqs, _ = B.rotary_frequencies([64])
    pos = positions(S, 1, 6)
    want = B.sol_qk_rotary(q, None, pos, freqs, q_weight=qw)[0]
    assert torch.equal(B.sol_qk_rotary(view, None, pos, freqs, q_weight=qw)[0], want)
    dwant = B.sol_qk_rotary_backward(want, None, q, None, pos, freqs, q_weight=qw)
    dgot = B.sol_qk_rotary_backward(want, None, view, None, pos, freqs, q_weight=qw)
    assert torch.equal(dwant[0], dgot[0]) and torch.equal(dwant[2], dgot[2])
    B.sol_qk_rotary(view, None, pos, freqs, q_weight=qw, out=(view, None))
    assert torch.equal(view, want)


def test_weight_gradients_of_many_tokens(B):
    q, k, qw, kw = make(2, 3000, 12, 4, 64, 37)
    dq, dk, _, _ = make(2, 3000, 12, 4, 64, 41, fused=False)
    freqs, _ = B.rotary_frequencies([64])
    # 6000 tokens x 2 groups over 592 blocks of 8 warps: at most 3 tasks of 4 heads in a lane's chain
    check_backward(B, dq, dk, q, k, positions(3000, 1, 12), freqs, None, True, qw, kw, chain=16)


def test_refusals_on_the_device(B):
    q, k, qw, kw = make(1, 4, 2, 2, 64, 43)
    freqs, _ = B.rotary_frequencies([64])
    pos = positions(4, 1, 1)
    with pytest.raises(ValueError):
        B.sol_qk_rotary(q, k[:, :3], pos, freqs)
    with pytest.raises(ValueError):
        B.sol_qk_rotary(q, k, pos.cpu(), freqs)
    with pytest.raises(TypeError):
        B.sol_qk_rotary(q, k, pos, freqs, q_weight=qw.float())
    with pytest.raises(TypeError):
        B.sol_qk_rotary(q, k, pos, freqs, q_weight=qw[:32])
    with pytest.raises(ValueError):
        B.sol_qk_rotary_backward(q.contiguous(), None, None, None, pos, freqs, q_weight=qw)
    with pytest.raises(B.SolError):
        B.sol_qk_rotary(torch.zeros((1, 4, 2, 48), dtype=torch.bfloat16, device="cuda"), None, pos, freqs[:24])
    with pytest.raises(B.SolError):
        B.sol_qk_rotary_backward(q.contiguous(), None, q, None, pos, freqs, q_weight=qw,
                                 workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
