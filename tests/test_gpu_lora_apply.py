"""GPU parity: adapters of many requests and their gradients through the C ABI against the FP64 oracle.

Tolerances.  The tensor core adds sixteen products to an FP32 sum at a time; a sum of n products is off by at most steps(n) = n / 16 + 24
times 2^-23 (a truncation) of the sum of their sizes, the joining of up to 16 slices in FP32 included in the 24.  t and dt enter the
second product in two BF16 parts: 2^-17 of their value (half a step of the second part, 2^-9 of at most 2^-8 of the first).  So an update has
steps(first sum) 2^-23 + 2^-17 + steps(2 r) 2^-23 of its magnitude; a BF16 result 2^-8 of its value on top, and 2^-24 of the sum.
"""
import numpy as np
import pytest
import torch

from oracle import lora_apply as L

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def steps(n):
    return (n / 16 + 24) * 2.0 ** -23


class Case:
    def __init__(self, offsets, ids, n, r, K, N, M, seed=1, pitch=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        bf = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
        self.x, self.y, self.dy, self.dx = (bf(M, c + pitch)[:, :c] for c in (K, N, N, K))
        self.a, self.b = bf(n, r, K), (0.1 * torch.randn((n, N, r), generator=g, device="cuda")).to(torch.bfloat16)
        self.s = torch.rand(n, generator=g, device="cuda") * 2 - 0.5
        self.o = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        self.i = torch.tensor(ids, dtype=torch.int32, device="cuda")
        self.r, self.K, self.N, self.M = r, K, N, M

    def stacks(self):
        return self.a, self.b, self.s, self.o, self.i

    def reference(self):
        return [f64(t) for t in (self.a, self.b, self.s)] + [self.o.tolist(), self.i.tolist()]

    def t_error(self):
        return steps(self.K) + 2.0 ** -17

    def check_forward(self, B, y0, y, t=None):
        ref, size, t_ref, t_size = L.apply(f64(self.x), *self.reference(), f64(y0))
        tol = 2.0 ** -8 * np.abs(ref) + (self.t_error() + steps(2 * self.r) + 2.0 ** -24) * size
        tol[size == 0] = 0                                   # rows without an adapter keep their bits
        err = np.abs(f64(y) - ref)
        assert np.all(err <= tol), f"y: err {err.max()} at {np.unravel_index((err - tol).argmax(), err.shape)}"
        if t is not None:
            there = t_size[:, 0] > 0
            got = f64(t[:, :self.r]) + f64(t[:, self.r:])
            assert np.all((np.abs(got - t_ref) <= self.t_error() * t_size)[there])

    def check_backward(self, B, dx=True):
        t = torch.full((self.M, 2 * self.r), float("nan"), dtype=torch.bfloat16, device="cuda")
        t_ref = L.apply(f64(self.x), *self.reference(), f64(self.y))[2]
        t64 = torch.from_numpy(t_ref).cuda()
        rows = t64.abs().sum(1) > 0
        hi = t64.to(torch.bfloat16)
        t[rows] = torch.cat((hi, (t64 - hi.double()).to(torch.bfloat16)), dim=1)[rows]
        dx0 = self.dx.clone()
        da, db = B.sol_lora_backward(self.dy, self.x, t, *self.stacks(), dx=self.dx if dx else None)
        used = f64(torch.where(rows[:, None], t[:, :self.r].double() + t[:, self.r:].double(), 0.0))
        ref = L.backward(f64(self.dy), f64(self.x), used, *self.reference(), f64(dx0))
        dt_error = steps(self.N) + 2.0 ** -17
        for name, got, want, size, error in (("dA", da, ref[0], ref[3], dt_error + steps(2 * self.M)), ("dB", db, ref[1], ref[4], steps(2 * self.M))):
            err = np.abs(f64(got) - want)
            assert got.dtype == torch.float32 and np.all(err <= error * size + 1e-30), f"{name}: {np.max(err / (error * size + 1e-30))}"
        if dx:
            tol = 2.0 ** -8 * np.abs(ref[2]) + (dt_error + steps(2 * self.r) + 2.0 ** -24) * ref[5]
            tol[ref[5] == 0] = 0
            err = np.abs(f64(self.dx) - ref[2])
            assert np.all(err <= tol), f"dx: err {err.max()}"
        else:
            assert torch.equal(self.dx, dx0)
        return da, db


CASES = [  # offsets, ids, adapters, r, K, N, M
    ([0, 1], [0], 1, 8, 8, 8, 1),
    ([0, 1], [0], 1, 16, 64, 64, 1),
    ([0, 128], [0], 1, 32, 256, 128, 128),
    ([0, 300], [0], 1, 32, 512, 320, 300),
    ([0, 1, 2, 3, 4, 5], [2, 0, 1, 2, -1], 3, 16, 192, 328, 5),
    ([3, 40, 40, 200, 331, 460], [1, 0, -1, 0, 9], 2, 64, 136, 72, 500),
    ([0, 129, 257, 1000], [1, 1, 0], 2, 24, 1000, 648, 1003),
    ([0, 700], [3], 5, 56, 2432, 1032, 700),
    ([0, 64, 2048], [0, 1], 2, 40, 320, 4104, 2049),
]


@pytest.mark.parametrize("offsets,ids,n,r,K,N,M", CASES)
def test_forward(B, offsets, ids, n, r, K, N, M):
    c = Case(offsets, ids, n, r, K, N, M)
    y0 = c.y.clone()
    y, t = B.sol_lora_apply(c.x, *c.stacks(), c.y, with_t=True)
    assert y is c.y
    B.sol_last_device_status()
    c.check_forward(B, y0, y, t)
    again = B.sol_lora_apply(c.x, *c.stacks(), y0)
    assert torch.equal(again, y)


@pytest.mark.parametrize("offsets,ids,n,r,K,N,M", CASES)
def test_gradients(B, offsets, ids, n, r, K, N, M):
    c = Case(offsets, ids, n, r, K, N, M, seed=2)
    first = c.check_backward(B)
    B.sol_last_device_status()
    second = c.check_backward(B, dx=False)
    assert all(torch.equal(a, b) for a, b in zip(first, second))


def test_many_requests_of_one_row_and_of_none(B):
    n = 1024
    lens = np.random.default_rng(3).integers(0, 3, n)
    offsets = np.concatenate(([0], np.cumsum(lens)))
    c = Case(offsets.tolist(), [(7 * i) % 130 - 1 for i in range(n)], 128, 16, 128, 192, int(offsets[-1]) + 2)
    y0 = c.y.clone()
    c.check_forward(B, y0, B.sol_lora_apply(c.x, *c.stacks(), c.y))
    c.check_backward(B)


def test_offsets_outside_the_rows_and_backwards(B):
    """Held to the rows that exist; a request that would end before it begins has none."""
    c = Case([-5, 20, 70, 60, 2000], [0, 1, 0, 1], 2, 16, 64, 64, 100)
    y0 = c.y.clone()
    y = B.sol_lora_apply(c.x, *c.stacks(), c.y)
    B.sol_last_device_status()
    c.o = torch.tensor([0, 20, 60, 60, 60], dtype=torch.int32, device="cuda")        # rows that one request alone has
    keep = slice(0, 60)
    ref, size, _, _ = L.apply(f64(c.x), *c.reference(), f64(y0))
    tol = 2.0 ** -8 * np.abs(ref) + (c.t_error() + steps(2 * c.r) + 2.0 ** -24) * size
    assert np.all((np.abs(f64(y) - ref) <= tol)[keep])


def test_rows_of_others_may_hold_anything(B):
    c = Case([10, 75, 200], [0, 1], 2, 32, 320, 448, 230)
    y0 = c.y.clone()
    for t in (c.x, c.y, c.dy, c.dx, y0):
        t[:10] = float("nan")
        t[200:] = float("inf")
    y = B.sol_lora_apply(c.x, *c.stacks(), c.y)
    same = torch.equal(y[:10].isnan(), y0[:10].isnan()) and torch.equal(y[200:], y0[200:])
    assert same and y[10:200].isfinite().all()
    inside = Case([0, 65, 190], [0, 1], 2, 32, 320, 448, 190)
    for name in ("x", "y", "dy", "dx"):
        setattr(inside, name, {"x": c.x, "y": y0, "dy": c.dy, "dx": c.dx}[name][10:200].clone())
    inside.a, inside.b, inside.s = c.a, c.b, c.s
    z0 = inside.y.clone()
    z, t = B.sol_lora_apply(inside.x, *inside.stacks(), inside.y, with_t=True)
    inside.check_forward(B, z0, z, t)
    wide = torch.full((230, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[10:200] = t
    da, db = B.sol_lora_backward(c.dy, c.x, wide, *c.stacks(), dx=c.dx)
    assert da.isfinite().all() and db.isfinite().all() and c.dx[10:200].isfinite().all() and c.dx[:10].isnan().all()
    # a value that is not finite in one request's row reaches that row and its adapter, nobody else
    inside.x[3, 5] = float("nan")
    z = B.sol_lora_apply(inside.x, *inside.stacks(), z0)
    assert z[3].isnan().all() and z[torch.arange(190, device="cuda") != 3].isfinite().all()


def test_pitches_capture_and_another_stream(B):
    c = Case([0, 150, 333], [1, 0], 2, 32, 264, 520, 340, pitch=24)
    y0 = c.y.clone()
    y, t = B.sol_lora_apply(c.x, *c.stacks(), c.y, with_t=True)
    c.check_forward(B, y0, y, t)
    c.check_backward(B)
    graph = torch.cuda.CUDAGraph()
    other = torch.empty_like(y0)
    with torch.cuda.graph(graph):
        other.copy_(y0)
        z, t2 = B.sol_lora_apply(c.x, *c.stacks(), other, with_t=True)
        grads = B.sol_lora_backward(c.dy, c.x, t2, *c.stacks())
    c2 = Case([0, 40, 340], [0, 1], 2, 32, 264, 520, 340, seed=8)
    for name in ("x", "dy", "a", "b", "s", "o", "i"):
        getattr(c, name).copy_(getattr(c2, name))
    graph.replay()
    torch.cuda.synchronize()
    c.check_forward(B, y0, other, t2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = B.sol_lora_backward(c.dy, c.x, t2, *c.stacks())
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(grads, again))


def test_rows_far_apart(B):
    """Element offsets past 32 bits: rows of x and y 2^24 elements apart."""
    M, pitch = 260, 1 << 24
    c = Case([0, 130, 260], [0, 1], 2, 16, 64, 128, M)
    wide = torch.empty(2 * M * pitch, dtype=torch.bfloat16, device="cuda")
    x, y = wide.as_strided((M, 64), (pitch, 1)), wide.as_strided((M, 128), (pitch, 1), 256)
    x.copy_(c.x)
    y.copy_(c.y)
    y0 = c.y.clone()
    B.sol_lora_apply(x, *c.stacks(), y)
    c.check_forward(B, y0, y)


def test_a_wait_that_runs_out_is_reported(B):
    c = Case([0, 300], [0], 1, 32, 512, 320, 300)
    y0 = c.y.clone()
    B.sol_lora_apply(c.x, *c.stacks(), c.y)
    torch.cuda.synchronize()
    try:
        B.sol_set_wait_limit_cycles(1000000)
        B.sol_test_hold_loads(True)
        c.y.copy_(y0)
        B.sol_lora_apply(c.x, *c.stacks(), c.y)
        with pytest.raises(B.SolError):
            B.sol_last_device_status()
        assert torch.equal(c.y, y0)
        B.sol_lora_backward(c.dy, c.x, torch.zeros((300, 64), dtype=torch.bfloat16, device="cuda"), *c.stacks(), dx=c.dx)
        with pytest.raises(B.SolError):
            B.sol_last_device_status()
    finally:
        B.sol_test_hold_loads(False)
        B.sol_set_wait_limit_cycles(0)
    c.check_forward(B, y0, B.sol_lora_apply(c.x, *c.stacks(), c.y))


def test_refused_tensors(B):
    c = Case([0, 40], [0], 1, 16, 64, 96, 40)
    a, b, s, o, i = c.stacks()
    for bad in ((a[:, :8], b, s, o, i), (a, b[:, :88], s, o, i), (a, b, s.double(), o, i), (a, b, s, o[:1], i), (a, b, s, o.long(), i), (a, b, s, o, i.float()),
                (a.float(), b, s, o, i), (a[0], b, s, o, i)):
        with pytest.raises((TypeError, ValueError)):
            B.sol_lora_apply(c.x, *bad, c.y)
    with pytest.raises(ValueError):
        B.sol_lora_apply(c.x[:39], *c.stacks(), c.y)
    with pytest.raises(B.SolError):
        B.sol_lora_apply(c.x, *c.stacks(), c.y, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
