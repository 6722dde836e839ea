"""The operators between the quantized linears, run as a DiT block's first half runs them: the modulation vectors
from the conditioning (weight-only linear), layer norm + modulation + quantizer, the fused q/k/v linear, head norm +
rotary positions in place on its output, block selection, block-sparse attention, and the output projection.

Every new stage is held to its own FP64 oracle on the inputs that the chain gave it; the chain as a whole is captured
into a graph and replayed on new inputs.  Then the gradients of the q/k step, as the training phase takes them.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import attention as OA
from oracle import block_sparse as OS
from oracle import matvec as OM
from oracle import rotary as OR

pytestmark = pytest.mark.gpu

BATCH, TOKENS, HEADS, D = 2, 1100, 4, 128
WIDTH = HEADS * D
AXES = [16, 56, 56]


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


class Block:
    def __init__(self, B, seed):
        self.B = B
        g = torch.Generator(device="cuda").manual_seed(seed)
        rand = lambda *s, k=1.0: (torch.randn(s, generator=g, device="cuda") * k).to(torch.bfloat16)  # noqa: E731
        self.cond, self.x = rand(BATCH, WIDTH), rand(BATCH * TOKENS, WIDTH)
        self.w_mod, self.b_mod = rand(2 * WIDTH, WIDTH, k=0.3 * WIDTH ** -0.5), rand(2 * WIDTH, k=0.05)
        self.mod = B.nvfp4_quantize_weight(self.w_mod)
        self.qkv = B.nvfp4_quantize_weight(rand(3 * WIDTH, WIDTH, k=WIDTH ** -0.5))
        self.proj = B.nvfp4_quantize_weight(rand(WIDTH, WIDTH, k=WIDTH ** -0.5))
        self.qw, self.kw = (1 + 0.2 * rand(D).float()).to(torch.bfloat16), (1 + 0.2 * rand(D).float()).to(torch.bfloat16)
        self.freqs, self.scale = B.rotary_frequencies(AXES)
        n = torch.arange(TOKENS, device="cuda")
        self.pos = torch.stack((torch.zeros_like(n), n // 33, n % 33), dim=1).contiguous()
        self.lens = torch.tensor([TOKENS, 777], dtype=torch.int32, device="cuda")
        self.T = torch.tensor([4.0 / 2688], device="cuda")

    def run(self):
        B, s = self.B, {}
        s["mod"] = B.nvfp4_matvec(self.cond, *self.mod, self.b_mod, activation=B.ACT_SILU)
        shift, scale = s["mod"][:, :WIDTH].contiguous(), s["mod"][:, WIDTH:].contiguous()
        hq, hsf = B.nvfp4_layernorm_quantize(self.x, scale, shift, TOKENS, self.T)
        s["fused"] = B.nvfp4_linear(hq, hsf, self.T, *self.qkv).view(BATCH, TOKENS, 3 * WIDTH)
        q, k, v = (s["fused"][:, :, i * WIDTH:(i + 1) * WIDTH].unflatten(2, (HEADS, D)) for i in range(3))
        s["q_raw"], s["k_raw"] = q.clone(), k.clone()
        B.sol_qk_rotary(q, k, self.pos, self.freqs, AXES, q_weight=self.qw, k_weight=self.kw, scale=self.scale, out=(q, k))
        s["q"], s["k"], s["v"] = q, k, v
        s["blocks"], s["counts"] = B.sol_select_blocks(q, k, 4, 1, self.lens)
        s["attention"] = B.sol_attention_blocks(q, k, v, s["blocks"], s["counts"], self.lens)
        s["out"] = B.nvfp4_quantize_linear(s["attention"].view(BATCH * TOKENS, WIDTH), *self.proj)
        return s


def check(block, s):
    B = block.B
    q, _, _ = B.nvfp4_quantize_weight(block.w_mod, B.SF_ROW_MAJOR)
    _, sf, ts = B.nvfp4_quantize_weight(block.w_mod, B.SF_ROW_MAJOR)
    w = oracle.dequantize(q.cpu().numpy(), sf.cpu().numpy().reshape(2 * WIDTH, WIDTH // 16), np.float32(ts.item()))
    ref = OM.linear(f64(block.cond), w, f64(block.b_mod), True)
    assert np.all(np.abs(f64(s["mod"]) - ref) <= OM.tolerance(f64(block.cond), w, ref, True))

    M = OR.rotation(OR.angles(f64(block.pos), f64(block.freqs), AXES), D, False, block.scale)
    for name, weight in (("q", block.qw), ("k", block.kw)):
        ref, bound = OR.forward(f64(s[name + "_raw"]).reshape(-1, HEADS, D), f64(weight), M, 1e-6)
        got = f64(s[name]).reshape(ref.shape)
        assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -19 * bound)

    lists, counts, _ = OS.select(f64(s["q"]), f64(s["k"]), 4, 1, block.lens.tolist())
    assert np.array_equal(s["blocks"].cpu().numpy(), lists) and np.array_equal(s["counts"].cpu().numpy(), counts)
    ref = OS.attend(f64(s["q"]), f64(s["k"]), f64(s["v"]), lists, counts, block.lens.tolist())
    assert np.all(np.abs(f64(s["attention"]) - ref) <= OA.attention_tolerance(ref, f64(s["v"])))
    assert torch.isfinite(s["out"]).all()
    assert B.sol_last_device_status() == 0


def test_first_half_of_a_block_stage_by_stage(B):
    block = Block(B, 1)
    check(block, block.run())


def test_captured_and_replayed_on_new_inputs(B):
    block = Block(B, 2)
    block.run()                                    # first calls outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = block.run()
    other = Block(B, 3)
    block.cond.copy_(other.cond)
    block.x.copy_(other.x)
    block.lens.copy_(torch.tensor([130, TOKENS], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    check(block, s)
    again = block.run()
    assert all(torch.equal(s[name], again[name]) for name in s)


def test_gradients_of_the_query_key_step_in_the_chain(B):
    block = Block(B, 4)
    s = block.run()
    g = torch.Generator(device="cuda").manual_seed(9)
    dq = torch.randn(s["q"].shape, generator=g, device="cuda").to(torch.bfloat16)
    dk = torch.randn(s["k"].shape, generator=g, device="cuda").to(torch.bfloat16)
    got = B.sol_qk_rotary_backward(dq, dk, s["q_raw"], s["k_raw"], block.pos, block.freqs, AXES, q_weight=block.qw, k_weight=block.kw,
                                   scale=block.scale)
    M = OR.rotation(OR.angles(f64(block.pos), f64(block.freqs), AXES), D, False, block.scale)
    for i, (dy, x, w) in enumerate(((dq, s["q_raw"], block.qw), (dk, s["k_raw"], block.kw))):
        dx, dw, bound, wbound = OR.backward(f64(dy).reshape(-1, HEADS, D), f64(x).reshape(-1, HEADS, D), f64(w), M, 1e-6)
        assert np.all(np.abs(f64(got[i]).reshape(dx.shape) - dx) <= 2.0 ** -8 * np.abs(dx) + 2.0 ** -18 * bound)
        assert np.all(np.abs(f64(got[2 + i]) - dw) <= 80 * 2.0 ** -24 * wbound)
