"""CPU: the rotary oracle against hand values and finite differences, the frequency entry point against the published
formulas, and the refusals of the entry points (nothing reaches CUDA)."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import rotary as R


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding, build

    build.build()
    binding.lib()
    return binding


def test_a_quarter_turn_by_hand():
    theta = np.array([[math.pi / 2]])
    x = np.array([[[3.0, 4.0, 7.0, 9.0]]])
    y, _ = R.forward(x, None, R.rotation(theta, 4, False, 1.0), 0.0)
    assert np.allclose(y, [[[-4.0, 3.0, 7.0, 9.0]]])
    y, _ = R.forward(x, None, R.rotation(np.array([[math.pi / 2, 0.0]]), 4, True, 2.0), 0.0)
    assert np.allclose(y, [[[-14.0, 8.0, 6.0, 18.0]]])     # pairs (0, 2) and (1, 3), scaled by 2


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("weighted", [False, True])
def test_gradients_against_differences(half, weighted):
    rng = np.random.default_rng(3)
    rows, H, D, rot = 3, 2, 8, 6
    x, dy = rng.normal(size=(rows, H, D)), rng.normal(size=(rows, H, D))
    w = rng.normal(size=D) if weighted else None
    M = R.rotation(rng.normal(size=(rows, rot // 2)), D, half, 1.3)
    dx, dw, _, _ = R.backward(dy, x, w, M, 1e-3)
    loss = lambda a, b: float((R.forward(a, b, M, 1e-3)[0] * dy).sum())  # noqa: E731
    h = 1e-6
    for idx in [(0, 0, 0), (1, 1, 5), (2, 0, 7), (0, 1, 3)]:
        e = np.zeros_like(x)
        e[idx] = h
        assert abs((loss(x + e, w) - loss(x - e, w)) / (2 * h) - dx[idx]) < 1e-7
    for c in (0, 4, 7) if weighted else ():
        e = np.zeros_like(w)
        e[c] = h
        assert abs((loss(x, w + e) - loss(x, w - e)) / (2 * h) - dw[c]) < 1e-7


def test_frequencies_follow_the_published_formulas(B):
    f, s = B.rotary_frequencies([16, 56, 56], device="cpu")
    want = np.concatenate([10000.0 ** (-2.0 * np.arange(d // 2) / d) for d in (16, 56, 56)])
    assert s == 1.0 and np.allclose(f.numpy(), want, rtol=1e-14)
    f, s = B.rotary_frequencies([64], theta=500000.0, scaling="linear", factor=4.0, device="cpu")
    base = 500000.0 ** (-2.0 * np.arange(32) / 64)
    assert s == 1.0 and np.allclose(f.numpy(), base / 4.0, rtol=1e-14)
    f, _ = B.rotary_frequencies([64], scaling="ntk", factor=4.0, device="cpu")
    assert np.allclose(f.numpy(), (10000.0 * 4.0 ** (64 / 62)) ** (-2.0 * np.arange(32) / 64), rtol=1e-13)
    assert abs(f.numpy()[-1] * 4.0 / 10000.0 ** (-62 / 64) - 1.0) < 1e-12    # the slowest pair slows by the factor
    f, s = B.rotary_frequencies([64], scaling="yarn", factor=16.0, original_length=4096, device="cpu")
    plain = 10000.0 ** (-2.0 * np.arange(32) / 64)
    turns = 4096 * plain / (2 * math.pi)
    fast, slow = turns > 40, turns < 0.7
    assert fast.any() and slow.any()
    assert np.allclose(f.numpy()[fast], plain[fast], rtol=1e-13)             # many turns: left alone
    assert np.allclose(f.numpy()[slow], plain[slow] / 16.0, rtol=1e-13)      # less than a turn: interpolated
    assert np.all(np.diff(f.numpy()) < 0) and abs(s - (0.1 * math.log(16.0) + 1.0)) < 1e-15


@pytest.mark.parametrize("kw", [dict(axis_dims=[3]), dict(axis_dims=[0]), dict(axis_dims=[8], theta=0.0), dict(axis_dims=[8], theta=math.nan),
                                dict(axis_dims=[8], scaling="linear", factor=0.5), dict(axis_dims=[2], scaling="ntk", factor=2.0),
                                dict(axis_dims=[8], scaling="yarn", factor=2.0), dict(axis_dims=[8], scaling="yarn", factor=math.inf, original_length=9.0),
                                dict(axis_dims=[8], scaling="yarn", factor=2.0, original_length=9.0, beta_fast=1.0, beta_slow=2.0)])
def test_frequencies_refuse(B, kw):
    with pytest.raises(B.SolError):
        B.rotary_frequencies(device="cpu", **kw)


def test_frequencies_refuse_what_is_not_named(B):
    with pytest.raises(ValueError):
        B.rotary_frequencies([8], scaling="longer", device="cpu")
    with pytest.raises(ValueError):
        B.rotary_frequencies([], device="cpu")


def test_entry_points_refuse_bad_arguments(B):
    L = B.lib()
    buf = ctypes.create_string_buffer(4096)
    p = (ctypes.addressof(buf) + 255) & ~255   # aligned fake pointer, never dereferenced
    NULLP, SHAPE, ALIGN, WS, LAYOUT = 1, 2, 3, 4, 8

    def rot(**kw):
        d = dict(positions=p, freqs=p, position_rows=4, axes=1, axis_dims=(64,), layout=0, scale=1.0)
        d.update(kw)
        dims = d["axis_dims"] + (0,) * (4 - len(d["axis_dims"]))
        return B._ROTARY.pack(d["positions"] or 0, d["freqs"] or 0, d["position_rows"], d["axes"], *dims, d["layout"], d["scale"])

    def heads(x=p, out=p, weight=None, heads=2, ld_in=128, ld_out=128):
        return B._HEAD_TENSOR.pack(x or 0, out or 0, weight or 0, heads, ld_in, ld_out)

    def fwd(q=None, k=None, rows=4, D=64, r=None, eps=1e-6, no_q=False, no_rot=False):
        return L.sol_qk_rotary(None if no_q else q or heads(), k, rows, D, None if no_rot else r or rot(), eps, None)

    assert fwd(no_q=True) == NULLP
    assert fwd(q=heads(x=None)) == NULLP and fwd(k=heads(out=None)) == NULLP
    assert fwd(no_rot=True) == NULLP                                  # neither positions nor a weight: nothing to do
    assert fwd(r=rot(positions=None)) == NULLP and fwd(r=rot(freqs=None)) == NULLP
    assert fwd(rows=0) == SHAPE and fwd(rows=1 << 31) == SHAPE and fwd(D=96) == SHAPE and fwd(D=512) == SHAPE
    assert fwd(eps=-1.0) == SHAPE and fwd(eps=math.nan) == SHAPE
    assert fwd(q=heads(heads=0)) == SHAPE and fwd(q=heads(ld_in=64)) == SHAPE and fwd(q=heads(ld_out=120)) == SHAPE
    assert fwd(r=rot(axis_dims=(60,))) == SHAPE                       # 60 % 8
    assert fwd(r=rot(axis_dims=(72,))) == SHAPE                       # more than the head
    assert fwd(r=rot(axes=2, axis_dims=(9, 7))) == SHAPE and fwd(r=rot(axes=2, axis_dims=(16, 0))) == SHAPE
    assert fwd(r=rot(axes=0)) == SHAPE and fwd(r=rot(axes=5)) == SHAPE and fwd(r=rot(position_rows=0)) == SHAPE
    assert fwd(r=rot(scale=math.inf)) == SHAPE and fwd(r=rot(layout=2)) == LAYOUT
    assert fwd(r=rot(positions=p + 4)) == ALIGN and fwd(r=rot(freqs=p + 4)) == ALIGN
    assert fwd(q=heads(x=p + 8)) == ALIGN and fwd(q=heads(ld_in=132)) == ALIGN and fwd(q=heads(weight=p + 4)) == ALIGN
    assert fwd(q=heads(out=p + 2)) == ALIGN and fwd(k=heads(ld_out=129)) == ALIGN

    need = L.sol_qk_rotary_backward_workspace_bytes(64)
    assert need > 0 and L.sol_qk_rotary_backward_workspace_bytes(48) == 0

    def grad(dy=p, x=p, dx=p, weight=p, dweight=p, heads=2, ld_dy=128, ld_x=128, ld_dx=128):
        return B._HEAD_GRAD.pack(dy or 0, x or 0, dx or 0, weight or 0, dweight or 0, heads, ld_dy, ld_x, ld_dx)

    def bwd(q=None, k=None, rows=4, D=64, r=None, eps=1e-6, ws=p, size=need, no_q=False, no_rot=False):
        return L.sol_qk_rotary_backward(None if no_q else q or grad(), k, rows, D, None if no_rot else r or rot(), eps, ws,
                                        size, None)

    assert bwd(no_q=True) == NULLP and bwd(q=grad(dy=None)) == NULLP and bwd(q=grad(dx=None)) == NULLP
    assert bwd(q=grad(x=None)) == NULLP and bwd(q=grad(dweight=None)) == NULLP and bwd(ws=None) == NULLP
    assert bwd(q=grad(weight=None), no_rot=True) == NULLP
    assert bwd(size=need - 1) == WS and bwd(ws=p + 128) == ALIGN
    assert bwd(rows=0) == SHAPE and bwd(D=80) == SHAPE and bwd(q=grad(ld_x=64)) == SHAPE and bwd(k=grad(heads=3)) == SHAPE
    assert bwd(q=grad(dweight=p + 2)) == ALIGN and bwd(q=grad(ld_dx=130)) == ALIGN and bwd(q=grad(x=p + 8)) == ALIGN
    assert bwd(r=rot(layout=7)) == LAYOUT


def test_binding_refuses_before_the_library(B):
    q = torch.zeros((1, 4, 2, 64), dtype=torch.bfloat16)
    pos, f = torch.zeros((4, 1), dtype=torch.int64), torch.zeros(32, dtype=torch.float64)
    with pytest.raises(TypeError):                                   # host tensors
        B.sol_qk_rotary(q, None, pos, f)
    with pytest.raises(TypeError):
        B.sol_qk_rotary_backward(q, None, None, None, pos, f)
    shape = (1, 4, 2, 64)
    assert B._head_view("q", q, shape, -1) == 128 and B._head_view("q", q[:, :, :1], (1, 4, 1, 64), -1) == 128
    with pytest.raises(TypeError):
        B._head_view("q", q.float(), shape, -1)
    with pytest.raises(ValueError):
        B._head_view("q", q, (1, 4, 4, 64), -1)
    with pytest.raises(ValueError):
        B._head_view("q", q, shape, 0)                               # another device
    with pytest.raises(ValueError):
        B._head_view("q", q.transpose(1, 2), (1, 2, 4, 64), -1)
    with pytest.raises(ValueError):                                  # batches not densely stacked
        B._head_view("q", torch.zeros((2, 8, 2, 64), dtype=torch.bfloat16)[:, :4], (2, 4, 2, 64), -1)
    assert B._rotary_of(None, None, None, 0, 1.0, 4, -1) is None and B._rotary_of(pos, f, None, 0, 1.0, 8, -1) is not None
    for bad in [(pos.int(), f, None), (pos[:, 0], f, None), (pos, f.float(), None), (pos, None, None), (None, f, None),
                (pos, f, [32, 32]), (pos, f, [32]), (pos[:3], f, None)]:
        with pytest.raises((TypeError, ValueError)):
            B._rotary_of(*bad, 0, 1.0, 4, -1)
