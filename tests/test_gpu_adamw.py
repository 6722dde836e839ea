"""GPU parity: the AdamW step over many tensors through the C ABI against the oracle.

Moments, 8-bit codes and exponent bytes are compared bit for bit: the definition rounds every operation.  Parameters (FP64 in the
oracle, from the same FP32 moments): root and quotient are the hardware's approximate ones (at most 2^-22 and 2^-22 relative), root,
bias correction and eps enter with three more roundings, the numerator with two, the sum with two of the parameter's size: 2^-24 (2 |p|
+ 16 |update|), and 2^-8 of the value where it leaves as BF16 to nearest, 2^-7 where by chance (a whole step).
"""
import numpy as np
import pytest
import torch

from oracle import adamw as A

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


def host(t):
    return t.detach().cpu().numpy() if t.dtype != torch.bfloat16 else t.detach().float().cpu().numpy()


class Run:
    """A plan over random tensors, and the oracle's copy of everything in it."""

    def __init__(self, B, sizes, bits, p16, g16, copy, seed, step=0, warm=True):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda n: torch.randn(n, generator=g, device="cuda")  # noqa: E731
        self.B, self.sizes, self.bits = B, sizes, bits
        ps = [(0.05 * randn(n)).to(torch.bfloat16 if p16 else torch.float32) for n in sizes]
        self.gs = [(1e-3 * randn(n) * torch.exp(2 * randn(n))).to(torch.bfloat16 if g16 else torch.float32) for n in sizes]
        states = None
        if warm:
            m = [1e-4 * randn(n) for n in sizes]
            v = [(1e-3 * randn(n)).square() for n in sizes]
            if bits == 8:
                em, ev = ([A.encode(host(x), k, None) for x in s] for s, k in ((m, 3), (v, 2)))
                up = lambda parts, i: [torch.from_numpy(x[i]).cuda() for x in parts]  # noqa: E731
                states = {"m": up(em, 0), "m_scale": up(em, 1), "v": up(ev, 0), "v_scale": up(ev, 1)}
            else:
                states = {"m": m, "v": v}
        self.plan = B.sol_adamw_plan(ps, self.gs, copies=[p.to(torch.bfloat16) for p in ps] if copy else None, state_bits=bits, states=states, step=step)
        self.t = step

    def check_step(self, seed=None, lr=1e-3, lr_factor=1.0, g_factor=1.0, only=None, step=None, **kw):
        """One step (or `step`, a callable), checked on all tensors or `only` some."""
        plan, bits = self.plan, self.bits
        names = ("m", "v") if bits == 32 else ("m", "v", "m_scale", "v_scale")
        some = range(len(self.sizes)) if only is None else only
        before = {i: [host(plan.params[i]).astype(np.float64)] + [host(getattr(plan, n)[i]).copy() for n in names] for i in some}
        if step is None:
            self.B.sol_adamw_step(plan, lr, seed=seed, **kw)
        else:
            step()
        self.t += 1
        torch.cuda.synchronize()
        assert plan.step.tolist() == [self.t, 0]
        b1, b2, eps, decay = kw.get("beta1", 0.9), kw.get("beta2", 0.999), kw.get("eps", 1e-8), kw.get("weight_decay", 0.01)
        for i in some:
            p, m, v = before[i][:3]
            g = host(plan.grads[i]) * np.float32(g_factor)
            if bits == 8:
                m, v = A.decode(m, before[i][3], 3), A.decode(v, before[i][4], 2)
            m, v = A.moments(m, v, g, b1, b2)
            r = None if seed is None else A.noise(seed, self.t, i, np.arange(self.sizes[i]))
            if bits == 8:
                for name, value, k, shift in (("m", m, 3, 0), ("v", v, 2, 16)):
                    code, scale = A.encode(value, k, None if r is None else (r >> shift) & 0xFFFF)
                    assert np.array_equal(host(getattr(plan, name)[i]), code), f"{name} of tensor {i}"
                    assert np.array_equal(host(getattr(plan, name + "_scale")[i]), scale), f"{name} scale of tensor {i}"
            else:
                assert np.array_equal(host(plan.m[i]), m) and np.array_equal(host(plan.v[i]), v)
            ref, size = A.parameters(p, m.astype(np.float64), v.astype(np.float64), self.t, lr * lr_factor, b1, b2, eps, decay)
            tol = U * (2 * np.abs(p) + 16 * size * np.abs(m))
            got = host(plan.params[i]).astype(np.float64)
            if plan.params[i].dtype == torch.bfloat16:
                tol = tol + (2.0 ** -8 if seed is None else 2.0 ** -7) * np.abs(ref)
            assert np.all(np.abs(got - ref) <= tol), f"parameter {i}: err/tol {np.max(np.abs(got - ref) / tol)}"
            if plan.copies is not None:
                assert torch.equal(plan.copies[i], plan.params[i].to(torch.bfloat16))


SIZES = [1, 7, 8, 31, 32, 33, 63, 200, 2047, 2048, 2049, 6151, 100003, 0, 5]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p16,g16,copy", [(False, False, True), (False, True, False), (True, True, False), (True, False, False)])
@pytest.mark.parametrize("seed", [None, 1234567890123456789])
def test_two_steps(B, bits, p16, g16, copy, seed):
    run = Run(B, SIZES, bits, p16, g16, copy, 3)
    run.check_step(seed)
    run.check_step(seed, lr=3e-4, beta1=0.8, beta2=0.95, eps=1e-6, weight_decay=0.1)


@pytest.mark.parametrize("bits", [32, 8])
def test_from_zero_states(B, bits):
    run = Run(B, [40, 4096, 3], bits, False, False, False, 4, warm=False)
    run.gs[1].zero_()                                   # v = 0: 0 / eps
    run.check_step(11)
    run.check_step(11)


def test_more_tensors_than_a_launch_takes(B):
    sizes = [(37 * i) % 1500 for i in range(1000)]
    run = Run(B, sizes, 8, False, False, True, 5, step=1000)
    run.check_step(2 ** 63 + 5)


def test_late_steps_and_steps_past_32_bits(B):
    for step in (9999, 2 ** 32 + 6):
        run = Run(B, [100, 77], 8, True, True, False, 6, step=step)
        run.check_step(17)


@pytest.mark.parametrize("bits", [32, 8])
def test_values_that_are_not_finite(B, bits):
    run = Run(B, [96, 40], bits, False, False, False, 7)
    run.gs[0][5], run.gs[0][40], run.gs[0][41] = float("nan"), float("inf"), -float("inf")
    plan = run.plan
    old = plan.params[0].clone()
    B.sol_adamw_step(plan, 1e-3, seed=1)
    bad = torch.tensor([5, 40, 41], device="cuda")
    fine = torch.ones(96, dtype=torch.bool, device="cuda")
    fine[bad] = False
    assert plan.params[0][bad].isnan().all() and plan.params[0][fine].isfinite().all() and not torch.equal(plan.params[0], old)
    assert plan.params[1].isfinite().all()
    if bits == 8:
        assert ((plan.m[0][bad] & 127) == 127).all() and (plan.v[0][bad] == 127).all()
        assert ((plan.m[0][fine] & 127) < 127).all() and (plan.v[0][fine] < 124).all()
    run.gs[0][bad] = 1e-3
    B.sol_adamw_step(plan, 1e-3, seed=1)
    assert plan.params[0][bad].isnan().all() and plan.params[0][fine].isfinite().all()


def test_tiny_and_huge_values(B):
    run = Run(B, [64, 64, 64], 8, False, False, False, 8, warm=False)
    run.gs[0].mul_(1e-33)                               # squares vanish, first moments are subnormal
    run.gs[1].mul_(1e18)
    run.gs[2][:32] = torch.logspace(-18, 3, 32, device="cuda")     # one block over many powers of two
    run.check_step(5, eps=1e-3)
    run.check_step(5, eps=1e-3)


@pytest.mark.parametrize("eps", [1e-9, 2e-10, 1e-12, 1e-16])
def test_squares_below_the_normal_range(B, eps):
    run = Run(B, [256], 32, False, False, False, 12, warm=False)
    run.gs[0].copy_(torch.logspace(-21, -15, 256, device="cuda"))       # squares from 1e-42 on, times 1 - beta2
    run.check_step(None, eps=eps, weight_decay=0.0)
    run.check_step(None, eps=eps, weight_decay=0.0, beta2=0.9999)


def test_factors_on_the_device_capture_and_replay(B):
    run = Run(B, [5000, 321], 8, False, False, True, 9)
    lr_scale, grad_scale = torch.tensor([0.5], device="cuda"), torch.tensor(0.25, device="cuda")
    call = lambda: B.sol_adamw_step(run.plan, 1e-3, seed=99, lr_scale=lr_scale, grad_scale=grad_scale)  # noqa: E731
    run.check_step(99, lr_factor=0.5, g_factor=0.25, step=call)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    assert run.plan.step.tolist() == [run.t, 0]         # a capture does not run
    for factor in (1.0, 0.125):
        lr_scale.fill_(factor)
        grad_scale.fill_(2 * factor)
        run.gs[0].neg_()
        run.check_step(99, lr_factor=factor, g_factor=2 * factor, step=graph.replay)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def on_side():
        with torch.cuda.stream(side):
            call()
        side.synchronize()

    run.check_step(99, lr_factor=0.125, g_factor=0.25, step=on_side)


def test_other_gradients_and_parameters_without_one(B):
    run = Run(B, [300, 40, 64], 32, False, False, False, 10)
    plan = run.plan
    keep = [t.clone() for t in (plan.params[1], plan.m[1], plan.v[1])]
    plan.set_grads([g.to(torch.bfloat16) if i != 1 else None for i, g in enumerate(run.gs)])
    run.check_step(None, only=[0, 2])
    assert all(torch.equal(a, b) for a, b in zip(keep, (plan.params[1], plan.m[1], plan.v[1])))
    plan.set_grads([None] * 3)
    B.sol_adamw_step(plan, 1e-3)
    assert plan.step.tolist() == [2, 0]


@pytest.mark.parametrize("bits", [32, 8])
def test_tensors_on_16_byte_boundaries(B, bits):
    g = torch.Generator(device="cuda").manual_seed(13)
    ps, gs = ([torch.randn(n, generator=g, device="cuda")[4:] for n in (3004, 68)] for _ in range(2))
    other = [torch.cat((torch.zeros(4, device="cuda"), p)) for p in ps]
    plan = B.sol_adamw_plan(ps, gs, state_bits=bits)
    same = B.sol_adamw_plan([p[4:].clone() for p in other], [x.clone() for x in gs], state_bits=bits)
    for _ in range(2):
        B.sol_adamw_step(plan, 1e-3, seed=4)
        B.sol_adamw_step(same, 1e-3, seed=4)
    assert all(torch.equal(a, b) for n in ("params", "m", "v") for a, b in zip(getattr(plan, n), getattr(same, n)))


def test_a_tensor_past_32_bits(B):
    n, tail = 2 ** 32 + 100, 100 + 4096
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    p[-tail:] = 0.05 * torch.randn(tail, device="cuda")
    g[-tail:] = 1e-3 * torch.randn(tail, device="cuda")
    plan = B.sol_adamw_plan([p], [g], state_bits=8)
    B.sol_adamw_step(plan, 1e-3, seed=21)
    m, v = A.moments(np.zeros(tail, np.float32), np.zeros(tail, np.float32), host(g[-tail:]), 0.9, 0.999)
    r = A.noise(21, 1, 0, np.arange(n - tail, n))
    for name, value, k, shift in (("m", m, 3, 0), ("v", v, 2, 16)):
        first = (n - tail) % 32                          # blocks are the tensor's: fill the tail's first one up
        pad = np.append(np.zeros(first, np.float32), value)
        code, scale = A.encode(pad, k, np.append(np.zeros(first, np.int64), (r >> shift) & 0xFFFF))
        assert np.array_equal(host(getattr(plan, name)[0][-tail:]), code[first:])
        assert np.array_equal(host(getattr(plan, name + "_scale")[0][-scale.size:]), scale)
    assert (p[:1000] == 0).all() and (plan.m[0][:1 << 20] == 0).all()


def test_refused_plans(B):
    p, g = torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
    for bad in (lambda: B.sol_adamw_plan([p, p], [g, g]), lambda: B.sol_adamw_plan([p], [g[:32]]), lambda: B.sol_adamw_plan([p], [g, g]),
                lambda: B.sol_adamw_plan([p.half()], [g]), lambda: B.sol_adamw_plan([p], [g.half()]), lambda: B.sol_adamw_plan([p[::2]], [g[:32]]),
                lambda: B.sol_adamw_plan([p], [g], state_bits=16), lambda: B.sol_adamw_plan([p], [g], step=-1), lambda: B.sol_adamw_plan([p], [g], copies=[p]),
                lambda: B.sol_adamw_plan([p.bfloat16()], [g], copies=[p.bfloat16()]), lambda: B.sol_adamw_plan([p], [g.cpu()]),
                lambda: B.sol_adamw_plan([p], [g], states={"m": [p], "v": [p[:3]]})):
        with pytest.raises((TypeError, ValueError)):
            bad()
    plan = B.sol_adamw_plan([p[4:]], [g[4:]])
    assert plan.step.tolist() == [0, 0]
    plan = B.sol_adamw_plan([p[1:]], [g[1:]])
    with pytest.raises(B.SolError):                     # not on a 16-byte boundary
        B.sol_adamw_step(plan, 1e-3)
    with pytest.raises(B.SolError):
        B.sol_adamw_step(B.sol_adamw_plan([p], [g]), -1.0)


def test_large_steps_in_chunks_of_several(B):
    run = Run(B, [39000037, 5, 8191, 8193, 8192, 100], 32, False, True, True, 14)
    run.check_step(None)


@pytest.mark.parametrize("p16", [True, False])
def test_large_and_small_plans_agree(B, p16):
    """To nearest the place in a tensor does not count: a large tensor's slices (on blocks of 32) give what it gives."""
    n, cut = 40000007, 1000000
    g = torch.Generator(device="cuda").manual_seed(15)
    p = (0.05 * torch.randn(n, generator=g, device="cuda")).to(torch.bfloat16 if p16 else torch.float32)
    grad = (1e-3 * torch.randn(n, generator=g, device="cuda")).to(torch.bfloat16 if p16 else torch.float32)
    other = p.clone()
    whole = B.sol_adamw_plan([p], [grad], state_bits=8)
    for _ in range(2):
        B.sol_adamw_step(whole, 1e-3)
    for first in (0, 17 * cut, 39 * cut, 40 * cut - cut):
        part = slice(first, min(n, first + cut))
        small = B.sol_adamw_plan([other[part].clone()], [grad[part].clone()], state_bits=8)
        for _ in range(2):
            B.sol_adamw_step(small, 1e-3)
        assert torch.equal(small.params[0], p[part]) and torch.equal(small.m[0], whole.m[0][part]) and torch.equal(small.v[0], whole.v[0][part])
        assert torch.equal(small.m_scale[0], whole.m_scale[0][first // 32:first // 32 + small.m_scale[0].numel()])
    last = slice(40 * cut, n)
    small = B.sol_adamw_plan([other[last].clone()], [grad[last].clone()], state_bits=8)
    for _ in range(2):
        B.sol_adamw_step(small, 1e-3)
    assert torch.equal(small.params[0], p[last]) and torch.equal(small.v[0], whole.v[0][last])
