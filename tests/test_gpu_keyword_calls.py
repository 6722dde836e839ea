"""GPU: the entries that run on their first argument's device give the same bits for keyword calls as for calls by place."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


def same(a, b):
    a, b = (t if isinstance(t, tuple) else (t,) for t in (a, b))
    return len(a) == len(b) and all((x is None and y is None) or torch.equal(x, y) for x, y in zip(a, b))


def test_every_argument_by_name(B):
    g = torch.Generator(device="cuda").manual_seed(1)
    randn = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    x, w, bias = randn(3, 96), randn(40, 96), randn(40)
    q, sf, ts = B.nvfp4_quantize_weight(w)
    assert same(B.nvfp4_matvec(x=x, wq=q, wsf=sf, w_tscale=ts, bias=bias, activation=B.ACT_SILU), B.nvfp4_matvec(x, q, sf, ts, bias, B.ACT_SILU))
    q, sf = B.mxfp4_quantize(w)
    assert same(B.mxfp4_matvec(wq=q, x=x, wsf=sf, bias=bias), B.mxfp4_matvec(x, q, sf, bias))
    q, k, v = randn(2, 300, 4, 64), randn(2, 300, 2, 64), randn(2, 300, 2, 64)
    pos, weight = torch.arange(300, device="cuda")[:, None], randn(64)
    freqs, _ = B.rotary_frequencies(axis_dims=[64])
    assert same(B.sol_qk_rotary(q=q, k=k, positions=pos, freqs=freqs, q_weight=weight), B.sol_qk_rotary(q, k, pos, freqs, q_weight=weight))
    assert same(B.sol_qk_rotary_backward(dq=q, dk=k, q=q, k=k, positions=pos, freqs=freqs, k_weight=weight),
                B.sol_qk_rotary_backward(q, k, q, k, pos, freqs, k_weight=weight))
    lists = B.sol_select_blocks(q, k, 2)
    assert same(B.sol_select_blocks(q=q, k=k, count=2), lists)
    assert same(B.sol_attention_blocks(q=q, k=k, v=v, blocks=lists[0], counts=lists[1]), B.sol_attention_blocks(q, k, v, *lists))
