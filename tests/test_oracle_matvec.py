"""CPU: the weight-only linear's oracle on hand values, and the refusals of the entry points and the binding."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from oracle import matvec as OM


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding, build

    build.build()
    binding.lib()
    return binding


def test_by_hand():
    # one row, one block: codes 1 (0.5), 9 (-0.5), 7 (6) under scale 2 and T = 0.25
    q = np.zeros((1, 16), np.uint8)
    q[0, 0], q[0, 1] = 0x91, 0x07
    sf = np.zeros((1, 2), np.uint8)
    sf[0, 0] = 0x40                       # E4M3 2.0
    w = oracle.dequantize(q, sf, 0.25)
    assert w[0, :4].tolist() == [0.25, -0.25, 3.0, 0.0]
    x = np.zeros((1, 32))
    x[0, :3] = [4.0, 8.0, -1.0]
    assert OM.linear(x, w, np.array([10.0]))[0, 0] == 1.0 - 2.0 - 3.0 + 10.0
    assert abs(OM.linear(x, w, act=True)[0, 0] - (0.25 * 4 / (1 + np.exp(-4.0)) - 0.25 * 8 / (1 + np.exp(-8.0)) - 3.0 / (1 + np.e))) < 1e-12
    assert OM.silu(np.array([-800.0, 800.0])).tolist() == [0.0, 800.0]


def test_entry_points_refuse_bad_arguments(B):
    L = B.lib()
    buf = ctypes.create_string_buffer(4096)
    p = (ctypes.addressof(buf) + 255) & ~255   # aligned fake pointer, never dereferenced
    NULLP, SHAPE, ALIGN, WS, LAYOUT = 1, 2, 3, 4, 8
    big = 1 << 40

    def nv(x=p, ldx=64, wq=p, wsf=p, ts=p, bias=None, act=0, y=p, ldy=8, M=4, N=8, K=64, ws=p, size=big):
        return L.nvfp4_matvec(x, ldx, wq, wsf, ts, bias, act, y, ldy, M, N, K, ws, size, None)

    def mx(x=p, ldx=64, wq=p, wsf=p, bias=None, act=0, y=p, ldy=8, M=4, N=8, K=64, ws=p, size=big):
        return L.mxfp4_matvec(x, ldx, wq, wsf, bias, act, y, ldy, M, N, K, ws, size, None)

    assert nv(ts=None) == NULLP
    assert nv(ts=p + 2) == ALIGN
    for f in (nv, mx):
        for name in ("x", "wq", "wsf", "y"):
            assert f(**{name: None}) == NULLP
            assert f(**{name: p + 8}) == ALIGN
        assert f(bias=p + 8) == ALIGN and f(ldx=68) == ALIGN and f(ldy=12) == ALIGN
        assert f(act=1) == LAYOUT and f(act=3) == LAYOUT                    # GELU is an output activation elsewhere
        assert f(M=0) == SHAPE and f(N=12, ldy=16) == SHAPE and f(K=48) == SHAPE and f(N=0) == SHAPE
        assert f(ldx=56) == SHAPE and f(N=16) == SHAPE                      # pitches too small
        assert f(M=(1 << 18) + 1) == SHAPE and f(N=1 << 23, ldy=1 << 23) == SHAPE
        assert f(M=8, ws=None) == NULLP and f(ws=p + 128) == ALIGN
        assert f(M=8, size=L.sol_matvec_workspace_bytes(8, 64) - 1) == WS
    assert L.sol_matvec_workspace_bytes(0, 64) == 0 and L.sol_matvec_workspace_bytes(4, 48) == 0
    # x padded to sixteen rows and 256 columns in FP16, and a float per row
    assert L.sol_matvec_workspace_bytes(8, 64) == 16 * 256 * 2 + 16 * 4
    assert L.sol_matvec_workspace_bytes(4, 3072) == 0 and L.sol_matvec_workspace_bytes(5, 3072) > 0      # the blocks' own
    assert L.sol_matvec_workspace_bytes(1, 3104) == 16 * 3328 * 2 + 16 * 4
    assert L.sol_matvec_workspace_bytes(65, 544) == 128 * 768 * 2 + 128 * 4
    # the input activation is refused where an output activation is asked for
    assert L.nvfp4_linear_quantized_out(p, p, p, p, p, p, None, 2, p, p, p, None, 4, 64, 64, None) == LAYOUT


def test_binding_refuses_before_the_library(B):
    x = torch.zeros((2, 64), dtype=torch.bfloat16)
    wq, wsf = torch.zeros((8, 32), dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8)
    with pytest.raises(TypeError):                                          # host tensors
        B.nvfp4_matvec(x, wq, wsf, torch.ones(1))
    with pytest.raises(TypeError):
        B.mxfp4_matvec(x, wq, wsf)
    bad = [dict(x=x.float()), dict(x=x[0]), dict(x=x.t()), dict(wq=wq.int()), dict(wq=wq[:, ::2]), dict(wq=wq[:, :16].contiguous()),
           dict(wsf=wsf[:256]), dict(wsf=wsf.int()), dict(bias=torch.zeros(8)), dict(bias=torch.zeros(4, dtype=torch.bfloat16)),
           dict(out=torch.zeros((2, 8))), dict(out=torch.zeros((2, 16), dtype=torch.bfloat16)),
           dict(workspace=torch.zeros((4, 4), dtype=torch.uint8)[:, :2])]
    for kw in bad:
        args = dict(x=x, wq=wq, wsf=wsf, bias=None, out=None, workspace=None)
        args.update(kw)
        with pytest.raises((TypeError, ValueError)):
            B._matvec(None, "mxfp4_matvec", args["x"], args["wq"], args["wsf"], None, args["bias"], 0, args["out"], args["workspace"], 64)
