"""CPU: the layer norm oracle against hand values and differences, and the refusals of the entry points (nothing reaches CUDA)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import layernorm as N


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding, build

    build.build()
    binding.lib()
    return binding


def test_a_row_by_hand():
    # mean 3, centred -2 0 2, variance 8/3; with eps 1/3 the root is sqrt(3)
    y, _, mean, rstd = N.forward(np.array([[1.0, 3.0, 5.0]]), np.array([[2.0, 2.0, 0.0]]), np.array([[0.0, 1.0, 7.0]]), 1.0 / 3.0)
    assert np.allclose(mean, 3.0) and np.allclose(rstd, 3.0 ** -0.5)
    assert np.allclose(y, [[-4.0 / 3.0 ** 0.5, 1.0, 7.0]])


@pytest.mark.parametrize("rows_per_sample", [5, 2, 1])
def test_gradients_against_differences(rows_per_sample):
    rng = np.random.default_rng(7)
    rows, K, eps = 5, 6, 1e-2
    samples = -(-rows // rows_per_sample)
    x, dy = rng.normal(size=(rows, K)), rng.normal(size=(rows, K))
    scale, shift = rng.normal(size=(samples, K)), rng.normal(size=(samples, K))

    def loss(x, scale, shift):
        g, b = (N.rows_of(t, rows, rows_per_sample) for t in (1.0 + scale, shift))
        return float((N.forward(x, g, b, eps)[0] * dy).sum())

    got = N.backward(dy, x, N.rows_of(1.0 + scale, rows, rows_per_sample), eps, rows_per_sample)[:3]
    args, h = [x, scale, shift], 1e-5
    for i, grad in enumerate(got):
        for at in np.ndindex(*grad.shape):
            d = np.zeros_like(args[i])
            d[at] = h
            up, down = (loss(*(a + s * d if j == i else a for j, a in enumerate(args))) for s in (1.0, -1.0))
            assert abs((up - down) / (2 * h) - grad[at]) < 1e-7


def test_refusals(B):
    L = B.lib()
    buf = ctypes.create_string_buffer(8192)
    p = (ctypes.addressof(buf) + 255) & ~255
    NULLP, SHAPE, ALIGN, WS = 1, 2, 3, 4

    def forward(x=p, M=4, K=64, ldx=64, scale=p, shift=p, ld_mod=64, rows=4, offset=1.0, eps=1e-6, y=p, ldy=64, stats=p):
        return L.sol_layernorm(x, M, K, ldx, scale, shift, ld_mod, rows, offset, eps, y, ldy, stats, None)

    assert forward(x=None) == NULLP and forward(y=None) == NULLP
    for bad in (dict(M=0), dict(K=0), dict(K=60), dict(K=16392, ldx=16392, ldy=16392, ld_mod=16392), dict(ld_mod=56), dict(ldx=56), dict(ldy=56), dict(rows=0), dict(eps=-1.0),
                dict(eps=float("nan")), dict(offset=float("inf")), dict(M=2 ** 31)):
        assert forward(**bad) == SHAPE, bad
    for bad in (dict(x=p + 8), dict(y=p + 8), dict(scale=p + 2), dict(shift=p + 8), dict(stats=p + 4), dict(ldx=68), dict(ldy=66), dict(ld_mod=76)):
        assert forward(**bad) == ALIGN, bad

    def backward(dy=p, ld_dy=64, x=p, ldx=64, stats=p, scale=p, ld_scale=64, M=400, K=64, rows=400, offset=1.0, dx=p, ld_dx=64, ds=p, db=p, ws=p, size=1 << 22):
        return L.sol_layernorm_backward(dy, ld_dy, x, ldx, stats, scale, ld_scale, M, K, rows, offset, dx, ld_dx, ds, db, ws, size, None)

    need = L.sol_layernorm_backward_workspace_bytes(400, 64, 400)
    assert need > 0 and L.sol_layernorm_backward_workspace_bytes(400, 60, 400) == 0
    assert L.sol_layernorm_backward_workspace_bytes(8192, 64, 1) == 0            # a sample to a row: nothing to add up
    for bad in (dict(dy=None), dict(x=None), dict(stats=None), dict(dx=None), dict(ws=None)):
        assert backward(**bad) == NULLP, bad
    for bad in (dict(M=0), dict(K=4), dict(ld_dy=32), dict(ldx=32), dict(ld_dx=32), dict(ld_scale=8), dict(rows=-1), dict(offset=float("nan"))):
        assert backward(**bad) == SHAPE, bad
    for bad in (dict(dy=p + 8), dict(x=p + 2), dict(dx=p + 8), dict(scale=p + 8), dict(ds=p + 8), dict(db=p + 4), dict(stats=p + 4), dict(ld_dx=68), dict(ld_scale=68),
                dict(ws=p + 16)):
        assert backward(**bad) == ALIGN, bad
    assert backward(size=need - 1) == WS


@pytest.mark.parametrize("name", ["sol_layernorm", "sol_layernorm_backward"])
def test_host_tensors_are_refused(B, name):
    with pytest.raises(TypeError, match="CUDA"):
        getattr(B, name)(torch.zeros((4, 64), dtype=torch.bfloat16), *[None] * (2 if name.endswith("backward") else 0))
