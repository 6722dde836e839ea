"""CPU: the block-sparse oracle on hand cases, and the refusals of the entry points and the binding."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import block_sparse as S


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding, build

    build.build()
    binding.lib()
    return binding


def test_choice_by_hand():
    assert S.choose([1.0, 5.0, 5.0, 2.0], 2, 0) == [1, 2]
    assert S.choose([1.0, 5.0, 5.0, 2.0], 1, 0) == [1]          # the lower of equals
    assert S.choose([1.0, 5.0, 6.0, 2.0], 2, 1) == [0, 2]       # the first is forced
    assert S.choose([1.0, 5.0], 7, 2) == [0, 1]
    assert S.choose([], 3, 1) == []
    x = np.arange(300.0)[:, None]
    assert S.means(x, 256)[:, 0].tolist() == [127.5, 277.5]     # a ragged block's mean is over its own rows


def test_all_blocks_listed_is_dense_attention():
    rng = np.random.default_rng(1)
    q, k, v = (rng.normal(size=(1, n, 2, 16)) for n in (300, 200, 200))
    lists = np.tile(np.array([0, 1], np.int32), (1, 2, 2, 1))
    counts = np.full((1, 2, 2), 2, np.int32)
    assert np.allclose(S.attend(q, k, v, lists, counts), OA.attention(q, k, v), atol=1e-12)
    counts[0, 1, 1] = 0
    got = S.attend(q, k, v, lists, counts)
    assert np.all(got[0, 256:, 1] == 0) and np.all(got[0, :256, 1] != 0)
    assert np.allclose(S.attend(q, k, v, lists, np.full_like(counts, 2), lens=[130]), OA.attention(q, k[:, :130], v[:, :130]), atol=1e-12)


def test_entry_points_refuse_bad_arguments(B):
    L = B.lib()
    buf = ctypes.create_string_buffer(4096)
    p = (ctypes.addressof(buf) + 255) & ~255   # aligned fake pointer, never dereferenced
    NULLP, SHAPE, ALIGN, WS = 1, 2, 3, 4

    def sel(q=p, k=p, batch=1, sq=300, skv=300, H=4, Hk=2, D=64, ld_q=256, ld_k=128, count=2, first=1, lens=None, blocks=p, counts=p,
            scores=None, ws=p, size=1 << 40):
        return L.sol_select_blocks(q, k, batch, sq, skv, H, Hk, D, ld_q, ld_k, count, first, lens, blocks, counts, scores, ws, size, None)

    def att(q=p, k=p, v=p, out=p, batch=1, sq=300, skv=300, H=4, Hk=2, D=64, ld_q=256, ld_k=128, ld_v=128, ld_out=256, blocks=p, counts=p,
            n=2, lens=None):
        return L.sol_attention_blocks(q, k, v, out, batch, sq, skv, H, Hk, D, ld_q, ld_k, ld_v, ld_out, blocks, counts, n, lens, None)

    for name in ("q", "k", "blocks", "counts", "ws"):
        assert sel(**{name: None}) == NULLP
    for name in ("q", "k", "v", "out", "blocks", "counts"):
        assert att(**{name: None}) == NULLP
    for f in (sel, att):
        assert f(batch=0) == SHAPE and f(sq=0) == SHAPE and f(skv=0) == SHAPE and f(H=0) == SHAPE and f(Hk=0) == SHAPE and f(Hk=3) == SHAPE
        assert f(D=32) == SHAPE and f(D=96) == SHAPE and f(skv=1048577) == SHAPE and f(sq=(1 << 24) + 1) == SHAPE and f(batch=65536) == SHAPE
        assert f(ld_q=248) == SHAPE and f(ld_k=64) == SHAPE
        assert f(ld_q=260) == ALIGN and f(ld_k=132) == ALIGN and f(q=p + 8) == ALIGN and f(k=p + 2) == ALIGN
        assert f(blocks=p + 2) == ALIGN and f(counts=p + 1) == ALIGN and f(lens=p + 2) == ALIGN
    assert sel(count=0) == SHAPE and sel(count=8193) == SHAPE and sel(first=-1) == SHAPE and sel(first=3) == SHAPE
    assert sel(scores=p + 2) == ALIGN and sel(ws=p + 64) == ALIGN
    assert att(n=0) == SHAPE and att(n=8193) == SHAPE and att(ld_v=120) == SHAPE and att(ld_out=128) == SHAPE
    assert att(v=p + 8) == ALIGN and att(out=p + 8) == ALIGN and att(ld_out=258) == ALIGN
    need = L.sol_select_blocks_workspace_bytes(1, 300, 300, 4, 2, 64)
    assert need == 8 * 64 * (4 * 2 + 2 * 3) and sel(size=need - 1) == WS
    assert L.sol_select_blocks_workspace_bytes(1, 300, 300, 4, 3, 64) == 0


def test_binding_refuses_before_the_library(B):
    q = torch.zeros((1, 8, 4, 64), dtype=torch.bfloat16)
    k = torch.zeros((1, 8, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError):                       # host tensors
        B.sol_select_blocks(q, k, 1)
    with pytest.raises(TypeError):
        B.sol_attention_blocks(q, k, k, None, None)
    assert B._kv_of(q, k, -1) == (1, 8, 8, 4, 2, 64, 256, 128)
    for bad in (k[:, :, :, :32], k.repeat(2, 1, 1, 1), torch.zeros((1, 8, 3, 64), dtype=torch.bfloat16), k.float(), k[0]):
        with pytest.raises((TypeError, ValueError)):
            B._kv_of(q, bad, -1)
    assert B._lens_ptr(None, 1, -1) is None
    for bad in (torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int64), torch.zeros((1, 1), dtype=torch.int32)):
        with pytest.raises(TypeError):
            B._lens_ptr(bad, 1, -1)
