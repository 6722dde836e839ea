"""CPU: the AdamW oracle's 8-bit formats against torch's, its rounding by chance on average, and the refusals of the entry point."""
import ctypes
import struct

import numpy as np
import pytest
import torch

from oracle import adamw as A


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding, build

    build.build()
    binding.lib()
    return binding


@pytest.mark.parametrize("mantissa,dtype", [(3, torch.float8_e4m3fn), (2, torch.float8_e5m2)])
def test_codes_are_those_of_the_formats(mantissa, dtype):
    codes = np.arange(125 if mantissa == 2 else 127, dtype=np.uint8)
    want = torch.from_numpy(codes).view(dtype).double().numpy()
    if mantissa == 2:
        codes, want = codes[:124], want[:124]              # 124 is the format's infinity
    assert np.array_equal(A.table(mantissa)[codes], want)
    rng = np.random.default_rng(1)
    v = (rng.normal(size=64) * np.exp(3 * rng.normal(size=64))).astype(np.float32)
    v = v if mantissa == 3 else v * v
    code, scale = A.encode(v, mantissa, None)
    y = v.astype(np.float64) * np.repeat(2.0 ** (127.0 - scale), 32)
    assert np.array_equal(torch.from_numpy(y).float().to(dtype).double().numpy(), A.decode(code, np.full(2, 127), mantissa))
    top = np.abs(y).reshape(2, 32).max(axis=1)
    lo = 2.0 ** (7 if mantissa == 3 else 14)
    assert np.all((top >= lo) & (top < 2 * lo))


def test_rounding_by_chance_keeps_the_average():
    v = np.float32(1.0) + np.arange(32, dtype=np.float32) / 40
    total, n = np.zeros(32), 4000
    for s in range(n):
        code, scale = A.encode(v, 2, A.noise(7, s, 0, np.arange(32)) & 0xFFFF)
        total += A.decode(code, scale, 2)
    # a value lies in steps of 1/4 (1/2 above 2): deviation of the mean at most 1/4 / sqrt(n); five of them
    assert np.all(np.abs(total / n - v) < 5 * 0.25 / n ** 0.5)


def test_the_second_moment_moves_by_chance_and_not_to_nearest():
    """beta2 = 0.999 changes v by a thousandth of it a step, a fraction of a step of the format."""
    for seed, lo, hi in ((None, 0.99, 1.01), (3, 0.45, 0.75)):
        code, scale = A.encode(np.ones(2048, np.float32), 2, None)
        for t in range(500):
            _, v = A.moments(np.zeros(2048, np.float32), A.decode(code, scale, 2), np.zeros(2048, np.float32), 0.9, 0.999)
            code, scale = A.encode(v, 2, None if seed is None else A.noise(seed, t, 0, np.arange(2048)) & 0xFFFF)
        assert lo < A.decode(code, scale, 2).mean() < hi       # exact: 0.999^500 = 0.61


def test_refusals(B):
    L = B.lib()
    buf = ctypes.create_string_buffer(8192)
    p = (ctypes.addressof(buf) + 255) & ~255
    NULLP, SHAPE, ALIGN, LAYOUT = 1, 2, 3, 8

    def call(count=1, tensors=True, state=p, options=True, **kw):
        o = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.0, lr_scale=0, grad_scale=0, seed=0, chance=0, p16=0, g16=0, bits=32)
        t = dict(param=p, copy=0, grad=p, m=p, v=p, ms=0, vs=0, n=64)
        for k, v in kw.items():
            (o if k in o else t)[k] = v
        ob = struct.pack("@dddddPPQiiii", *o.values())
        tb = struct.pack("@PPPPPPPq", *t.values()) * max(count, 1)
        return L.sol_adamw_step(tb if tensors else None, count, ob if options else None, state, None)

    assert call(tensors=False) == NULLP and call(options=False) == NULLP and call(state=None) == NULLP
    for name in ("param", "grad", "m", "v"):
        assert call(**{name: 0}) == NULLP
        assert call(**{name: p + 8}) == ALIGN
    assert call(bits=8) == NULLP and call(bits=8, ms=p) == NULLP
    assert call(bits=16) == LAYOUT and call(p16=1, copy=p) == LAYOUT
    for bad in (dict(count=-1), dict(n=-1), dict(lr=-1.0), dict(lr=float("nan")), dict(beta1=1.0), dict(beta2=1.0), dict(beta1=-0.1), dict(eps=-1e-8),
                dict(decay=float("inf"))):
        assert call(**bad) == SHAPE, bad
    assert call(copy=p + 2) == ALIGN and call(state=p + 4) == ALIGN and call(lr_scale=p + 2) == ALIGN and call(grad_scale=p + 1) == ALIGN


def test_plans_of_host_tensors_are_refused(B):
    with pytest.raises(TypeError, match="CUDA"):
        B.sol_adamw_plan([torch.zeros(8)], [torch.zeros(8)])
    with pytest.raises(ValueError):
        B.sol_adamw_plan([], [])
    with pytest.raises(TypeError, match="plan"):
        B.sol_adamw_step(torch.zeros(8), 1e-3)
