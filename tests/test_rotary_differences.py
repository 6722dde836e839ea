"""The rotary step's gradients against differences, element by element and along directions in which a missing term shows.

CPU: the oracle's closed form against central differences of the oracle's forward in FP64, and the same comparison on gradients
with one term left out, which must fail.  GPU: the kernel's gradients against those differences, and against differences of
the kernel's own outputs.

Tolerances.  Central differences in FP64 with a step of 2^-13 of a unit value: cut off at about 2^-26 of the slope's third
derivative, rounding 2^-52 2^13 of the function; 2^-20 of the magnitudes covers both.  The kernel's gradient: 2^-8 of itself
(BF16) and 2^-18 of its magnitudes (FP32 roundings), its weight gradient (64 + 16) 2^-24 of its magnitudes.
"""
import numpy as np
import pytest
import torch

from oracle import rotary as R

STEP = 2.0 ** -13
CASES = [  # rows, heads, head_dim, rotated columns, half, eps
    (3, 2, 32, 32, False, 1e-6), (2, 3, 64, 32, True, 1e-6), (3, 1, 128, 128, False, 0.5), (2, 2, 64, 0, False, 1e-6), (1, 3, 256, 64, True, 0.0)]


def make(case, seed):
    rows, H, D, rot, half, _ = case
    rng = np.random.default_rng(seed)
    bf16 = lambda a: torch.from_numpy(a).to(torch.bfloat16)  # noqa: E731
    x, dy, w = bf16(rng.normal(size=(rows, H, D))), bf16(rng.normal(size=(rows, H, D))), bf16(rng.uniform(0.5, 2.5, D))
    pos = torch.arange(5, 5 + rows)[:, None]
    freqs = torch.from_numpy(10000.0 ** (-np.arange(rot // 2) * 2.0 / max(rot, 1)))
    M = R.rotation(R.angles(pos.numpy(), freqs.numpy(), [rot]), D, half, 1.25) if rot else None
    return x, dy, w, pos, freqs, M


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def differences(x, dy, w, M, eps):
    """d <forward(x, w), dy> / dx and / dw, one element at a time."""
    f = lambda x, w: R.forward(x, w, M, eps)[0]  # noqa: E731
    dx, dw = np.zeros_like(x), np.zeros_like(w)
    for j in range(x.shape[2]):
        e = np.zeros(x.shape[2])
        e[j] = STEP
        dx[:, :, j] = ((f(x + e, w) - f(x - e, w)) * dy).sum(axis=2) / (2 * STEP)
        dw[j] = ((f(x, w + e) - f(x, w - e)) * dy).sum() / (2 * STEP)
    return dx, dw


def agree(dx, dw, fd, bounds, slack, wslack):
    ok_x = np.all(np.abs(dx - fd[0]) <= slack[0] * np.abs(fd[0]) + slack[1] * bounds[0] + 2.0 ** -20 * bounds[0])
    return bool(ok_x and np.all(np.abs(dw - fd[1]) <= wslack * bounds[1] + 2.0 ** -20 * bounds[1]))


@pytest.mark.parametrize("case", CASES, ids=str)
def test_differences_see_every_term(case):
    x, dy, w, _, _, M = make(case, 1)
    x, dy, w, eps = f64(x), f64(dy), f64(w), case[5]
    fd = differences(x, dy, w, M, eps)
    dx, dw, bx, bw = R.backward(dy, x, w, M, eps)
    assert agree(dx, dw, fd, (bx, bw), (0, 0), 0)
    kernel = ((2.0 ** -8, 2.0 ** -18), 80 * 2.0 ** -24)      # the room that the kernel's gradients are given
    r = 1.0 / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps)
    dn = dy if M is None else np.einsum("mji,mhj->mhi", M, dy)
    proj = x * r * (dn * w * x * r).mean(axis=2, keepdims=True)
    wrong = {"projection": r * dn * w, "weight": r * (dn - x * r * (dn * x * r).mean(axis=2, keepdims=True)), "root": dn * w - proj,
             "projection's weight": r * (dn * w - x * r * (dn * x * r).mean(axis=2, keepdims=True)), "zero": 0 * dx, "sign": r * (dn * w + proj)}
    if M is not None:
        wrong["turn"] = R.backward(dy, x, w, None, eps)[0]
        wrong["inverse"] = R.backward(dy, x, w, np.swapaxes(M, 1, 2), eps)[0]
    for name, bad in wrong.items():
        assert not agree(bad, dw, fd, (bx, bw), *kernel), name
    assert not agree(dx, (dn * x).sum(axis=(0, 1)), fd, (bx, bw), *kernel)
    assert not agree(dx, (dn * x * r)[:, 1:].sum(axis=(0, 1)), fd, (bx, bw), *kernel)


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES, ids=str)
def test_kernel_against_differences(B, case):
    rows, H, D, rot, half, eps = case
    x, dy, w, pos, freqs, M = make(case, 2)
    got = B.sol_qk_rotary_backward(dy[None].cuda(), None, x[None].cuda(), None, pos.cuda() if rot else None, freqs.cuda() if rot else None,
                                   layout=B.ROTARY_HALF if half else B.ROTARY_INTERLEAVED, q_weight=w.cuda(), eps=eps, scale=1.25)
    fd = differences(f64(x), f64(dy), f64(w), M, eps)
    _, _, bx, bw = R.backward(f64(dy), f64(x), f64(w), M, eps)
    assert agree(f64(got[0])[0], f64(got[2]), fd, (bx, bw), (2.0 ** -8, 2.0 ** -18), 80 * 2.0 ** -24)


@pytest.mark.gpu
@pytest.mark.parametrize("half", [False, True])
def test_kernel_against_its_own_differences(B, half):
    S, H, D = 64, 4, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.randn((1, S, H, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    w = torch.randint(8, 40, (D,), generator=g, device="cuda").to(torch.bfloat16) / 16
    pos, (freqs, _) = torch.arange(S, device="cuda")[:, None], B.rotary_frequencies([D])
    lay = B.ROTARY_HALF if half else B.ROTARY_INTERLEAVED
    f = lambda x, w: B.sol_qk_rotary(x, None, pos, freqs, layout=lay, q_weight=w)[0].double()  # noqa: E731
    dx, _, dw, _ = B.sol_qk_rotary_backward(dy, None, x, None, pos, freqs, layout=lay, q_weight=w)
    dx, y = dx.double(), f(x, w)
    # Along x itself the norm does not change (eps is 1e-6 of it): twice and half of x give the same outputs but for BF16's rounding,
    # so <dx, x> of every head vanishes but for dx's own rounding.  Without the projection it would be <dy, y>.
    assert torch.all((f(2 * x, w) - f(x / 2, w)).abs() <= (2.0 ** -7 + 1e-5) * y.abs())
    M = R.rotation(R.angles(f64(pos), f64(freqs), [D]), D, half, 1.0)
    bound = torch.from_numpy(R.backward(f64(dy)[0], f64(x)[0], f64(w), M, 1e-6)[2]).cuda()[None]
    along = (dx * x.double()).sum(dim=3).abs()
    room = ((2.0 ** -8 * dx.abs() + 2.0 ** -18 * bound) * x.double().abs()).sum(dim=3) + 2e-6 * (dy.double() * y).abs().sum(dim=3)
    assert torch.all(along <= room)
    assert (dy.double() * y).sum(dim=3).abs().median() > 10 * room.median()       # the term would show
    # The outputs are linear in w: differences have no remainder, only the outputs' roundings, 2^-8 of each at most and at random:
    # six deviations of their sum.  (w +- 1/4 is exact.)
    e = torch.where(torch.rand(D, generator=g, device="cuda") < 0.5, -0.25, 0.25).to(torch.bfloat16)
    hi, lo = f(x, w + e), f(x, w - e)
    slope, want = ((hi - lo) * dy.double()).sum().item(), 2 * (dw.double() * e.double()).sum().item()
    noise = 6 * 2.0 ** -8 / 3 ** 0.5 * ((hi.square() + lo.square()) * dy.double().square()).sum().sqrt().item()
    assert abs(slope - want) <= noise
    e = dw.sign().to(torch.bfloat16) / 4                                           # the direction in which it is largest
    hi, lo = f(x, w + e), f(x, w - e)
    slope, want = ((hi - lo) * dy.double()).sum().item(), 2 * (dw.double() * e.double()).sum().item()
    assert abs(slope - want) <= noise < 0.05 * abs(want)
