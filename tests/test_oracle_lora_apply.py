"""CPU: the oracle of many requests' adapters against hand values and differences, and the refusals of the entry points."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import lora_apply as L


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding, build

    build.build()
    binding.lib()
    return binding


def test_two_requests_by_hand():
    x = np.array([[1.0, 2.0], [3.0, 4.0], [5.0, 6.0], [7.0, 8.0]])
    A, Bm = np.array([[[1.0, 0.0]], [[0.0, 1.0]]]), np.array([[[1.0], [10.0]], [[-1.0], [0.5]]])
    y, _, t, _ = L.apply(x, A, Bm, np.array([2.0, 1.0]), [1, 2, 2, 3], [1, 0, 0], np.ones((4, 2)))
    assert np.allclose(y, [[1, 1], [-3, 3], [11, 101], [1, 1]])          # row 1: adapter 1; row 2: adapter 0; the others none
    assert np.allclose(t[:, 0], [0, 4, 5, 0])


def test_gradients_against_differences():
    rng = np.random.default_rng(5)
    M, K, N, r, n = 7, 4, 3, 2, 3
    x, A, Bm, y, dy = (rng.normal(size=s) for s in ((M, K), (n, r, K), (n, N, r), (M, N), (M, N)))
    scaling, offsets, ids = np.array([0.5, 2.0, -1.0]), [0, 2, 3, 6], [2, 7, 0]

    def loss(x, A, Bm):
        return float((L.apply(x, A, Bm, scaling, offsets, ids, y)[0] * dy).sum())

    t = L.apply(x, A, Bm, scaling, offsets, ids, y)[2]
    da, db, dx = L.backward(dy, x, t, A, Bm, scaling, offsets, ids, np.zeros((M, K)))[:3]
    args, h = [x, A, Bm], 1e-5
    for i, grad in enumerate((dx, da, db)):
        for at in np.ndindex(*grad.shape):
            d = np.zeros_like(args[i])
            d[at] = h
            up, down = (loss(*(a + s * d if j == i else a for j, a in enumerate(args))) for s in (1.0, -1.0))
            assert abs((up - down) / (2 * h) - grad[at]) < 1e-7
    assert (da[1] == 0).all() and (db[1] == 0).all() and (dx[2] == 0).all()


def test_refusals(B):
    lib = B.lib()
    buf = ctypes.create_string_buffer(4096)
    p = (ctypes.addressof(buf) + 255) & ~255
    NULLP, SHAPE, ALIGN, WS = 1, 2, 3, 4
    base = dict(x=p, ldx=64, a=p, b=p, s=p, o=p, i=p, requests=3, n=2, y=p, ldy=96, t=p, M=50, K=64, N=96, r=16, ws=p, size=1 << 30)

    def forward(**kw):
        return lib.sol_lora_apply(*{**base, **kw}.values(), None)

    need = lib.sol_lora_workspace_bytes(50, 64, 96, 16, 2, 3, 0)
    assert need >= 50 * 16 * 4 and lib.sol_lora_workspace_bytes(50, 64, 96, 16, 2, 3, 1) > need
    assert lib.sol_lora_workspace_bytes(50, 60, 96, 16, 2, 3, 0) == 0
    for name in ("x", "a", "b", "s", "o", "i", "y", "ws"):
        assert forward(**{name: None}) == NULLP, name
    for bad in (dict(M=0), dict(K=60), dict(N=100), dict(r=12), dict(r=72), dict(r=0), dict(requests=0), dict(requests=1025), dict(n=0), dict(n=1025),
                dict(ldx=56), dict(ldy=88), dict(M=2 ** 31)):
        assert forward(**bad) == SHAPE, bad
    for bad in (dict(x=p + 8), dict(y=p + 8), dict(a=p + 2), dict(b=p + 8), dict(s=p + 2), dict(o=p + 1), dict(i=p + 2), dict(t=p + 8), dict(ldx=68),
                dict(ldy=100), dict(ws=p + 16)):
        assert forward(**bad) == ALIGN, bad
    assert forward(size=need - 1) == WS

    base2 = dict(dy=p, ld_dy=96, x=p, ldx=64, t=p, a=p, b=p, s=p, o=p, i=p, requests=3, n=2, dx=p, ld_dx=64, da=p, db=p, M=50, K=64, N=96, r=16, ws=p,
                 size=1 << 30)

    def backward(**kw):
        return lib.sol_lora_backward(*{**base2, **kw}.values(), None)

    for name in ("dy", "x", "t", "a", "b", "s", "o", "i", "da", "db", "ws"):
        assert backward(**{name: None}) == NULLP, name
    for bad in (dict(M=0), dict(K=4), dict(ld_dy=88), dict(ldx=56), dict(ld_dx=56), dict(r=4)):
        assert backward(**bad) == SHAPE, bad
    for bad in (dict(dy=p + 8), dict(t=p + 8), dict(da=p + 4), dict(db=p + 8), dict(dx=p + 8), dict(ld_dx=68)):
        assert backward(**bad) == ALIGN, bad
    assert backward(size=lib.sol_lora_workspace_bytes(50, 64, 96, 16, 2, 3, 1) - 1) == WS


@pytest.mark.parametrize("name,arguments", [("sol_lora_apply", 7), ("sol_lora_backward", 8)])
def test_host_tensors_are_refused(B, name, arguments):
    with pytest.raises(TypeError, match="CUDA"):
        getattr(B, name)(torch.zeros((4, 64), dtype=torch.bfloat16), *[None] * (arguments - 1))
