"""BF16 parameters are rounded up or down by chance, in proportion: by the 16 bits that seed, step, tensor and place give, and so that the
average moves as FP32 parameters would.

Value by value: the FP32 value in front of the rounding is known to the tolerance of an FP32 parameter (the moments are those of the
oracle, bit for bit; root and quotient 2^-22 each, four more roundings of the update, two of the sum: 2^-24 (2 |p| + 16 |update|)).  Rounding by
chance does not fall when the value grows, so what leaves lies between the oracle's roundings of both ends, and is the one value where these agree.
On average: the mean over n values of what is rounded, in steps, minus where the values lie, has a variance of at most 1 / 4 n: five of
its deviations, 2.5 / sqrt(n), and 2^-17 for the random bits' places.  Always down or to nearest on these values is off by 0.3 and more.
"""
import numpy as np
import pytest
import torch

from oracle import adamw as A

U = 2.0 ** -24
LR, B1, B2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01


def noise16(seed, step, tensor, n):
    """The parameter's 16 bits: those of the states' hash, multiplied once more."""
    h = A.noise(seed, step, tensor, np.arange(n)).astype(np.uint64)
    return (h * np.uint64(0x9E3779B1) & np.uint64(0xFFFFFFFF)) >> np.uint64(16)


def away(p, size):
    """FP32 values next to the ends p - size and p + size, outside, ordered by magnitude (rounding by chance works on magnitudes)."""
    lo, hi = np.abs(p) - size, np.abs(p) + size
    lo, hi = np.nextafter(lo.astype(np.float32), np.float32(0)), np.nextafter(hi.astype(np.float32), np.float32(np.inf))
    return np.copysign(np.maximum(lo, 0), p).astype(np.float32), np.copysign(hi, p).astype(np.float32)


def expected(p, g, m, v, t, seed, tensor):
    """What may leave: the two ends' roundings, and the FP64 value in front of it."""
    m, v = A.moments(m, v, g, B1, B2)
    ref, size = A.parameters(p.astype(np.float64), m.astype(np.float64), v.astype(np.float64), t, LR, B1, B2, EPS, DECAY)
    lo, hi = away(ref, U * (2 * np.abs(p) + 16 * size * np.abs(m)))
    bits = noise16(seed, t, tensor, p.size)
    return A.bf16_by_chance(lo, bits), A.bf16_by_chance(hi, bits), ref


def inputs(sizes, seed):
    rng = np.random.default_rng(seed)
    bf = lambda v: torch.from_numpy(v.astype(np.float32)).to(torch.bfloat16)  # noqa: E731
    ps = [bf(0.05 * rng.standard_normal(n)) for n in sizes]
    gs = [bf(1e-3 * rng.standard_normal(n)) for n in sizes]
    ms = [torch.from_numpy((1e-4 * rng.standard_normal(n)).astype(np.float32)) for n in sizes]
    vs = [torch.from_numpy(((1e-3 * rng.standard_normal(n)) ** 2).astype(np.float32)) for n in sizes]
    return ps, gs, ms, vs


def inside(got, lo, hi):
    return (np.abs(got) >= np.abs(lo)) & (np.abs(got) <= np.abs(hi)) & (np.signbit(got) == np.signbit(lo))


def test_other_roundings_would_be_seen():
    """The check on the oracle: down, up, to nearest and by other random bits are outside for a good part of the values."""
    (p,), (g,), (m,), (v,) = inputs([20000], 1)
    lo, hi, ref = expected(p.float().numpy(), g.float().numpy(), m.numpy(), v.numpy(), 8, 77, 0)
    assert np.mean(lo == hi) > 0.95
    value = ref.astype(np.float32)
    n = np.uint64(p.numel())
    assert inside(A.bf16_by_chance(value, noise16(77, 8, 0, int(n))), lo, hi).all()
    zeros = np.zeros(int(n), np.uint64)
    for bits in (zeros, zeros + np.uint64(0xFFFF), zeros + np.uint64(0x8000), noise16(78, 8, 0, int(n)), noise16(77, 8, 1, int(n)), noise16(77, 9, 0, int(n))):
        assert np.mean(~inside(A.bf16_by_chance(value, bits), lo, hi)) > 0.05


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("g16", [True, False])
def test_value_by_value(B, bits, g16):
    sizes, seed, step = [1, 31, 2049, 0, 70001], 77, 7
    ps, gs, ms, vs = inputs(sizes, 2)
    states = {"m": ms, "v": vs}
    if bits == 8:
        em, ev = [A.encode(m.numpy(), 3, None) for m in ms], [A.encode(v.numpy(), 2, None) for v in vs]
        ms, vs = ([torch.from_numpy(A.decode(*e, k)) for e in es] for es, k in ((em, 3), (ev, 2)))
        states = {name: [torch.from_numpy(e[i]) for e in es] for name, es, i in (("m", em, 0), ("m_scale", em, 1), ("v", ev, 0), ("v_scale", ev, 1))}
    plan = B.sol_adamw_plan([p.cuda() for p in ps], [(g if g16 else g.float()).cuda() for g in gs], state_bits=bits, step=step,
                            states={k: [t.cuda() for t in v] for k, v in states.items()})
    B.sol_adamw_step(plan, LR, B1, B2, EPS, DECAY, seed=seed)
    for i, (p, g, m, v) in enumerate(zip(ps, gs, ms, vs)):
        lo, hi, _ = expected(p.float().numpy(), g.float().numpy(), m.numpy(), v.numpy(), step + 1, seed, i)
        got = plan.params[i].float().cpu().numpy()
        good = inside(got, lo, hi)
        assert good.all(), f"tensor {i}: {np.mean(~good):.3g} of the values, the first at {np.argmin(good)}"


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [32, 8])
def test_on_average(B, bits):
    """Equal parameters and gradients: every value in front of the rounding is the same but for its place's random bits."""
    n = 1 << 20
    for start, grad in ((0.25, 1e-3), (-0.25, 1e-3), (0.3125, -1e-3)):
        p = torch.full((n,), start, dtype=torch.bfloat16, device="cuda")
        plan = B.sol_adamw_plan([p], [torch.full((n,), grad, device="cuda")], state_bits=bits)
        B.sol_adamw_step(plan, 3e-4, B1, B2, EPS, DECAY, seed=5)
        m, v = A.moments(np.zeros(1, np.float32), np.zeros(1, np.float32), np.full(1, grad, np.float32), B1, B2)
        ref, _ = A.parameters(np.full(1, start), m.astype(np.float64), v.astype(np.float64), 1, 3e-4, B1, B2, EPS, DECAY)
        step = 2.0 ** (np.floor(np.log2(abs(ref[0]))) - 7)
        place = abs(ref[0]) / step % 1.0
        assert 0.1 < place < 0.9
        mean = float(p.double().mean())
        assert abs(mean - ref[0]) <= (2.5 / n ** 0.5 + 2.0 ** -17 + U * 4 / 2.0 ** -8) * step, (mean - ref[0]) / step
        assert p.unique().numel() == 2
