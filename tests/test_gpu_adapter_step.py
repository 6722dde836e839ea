"""One training step of adapters through the C ABI: modulated norm, frozen projection, adapters of two policies, the way back, AdamW and the
weight refresh that follows a policy update, stage by stage against the oracles, and its gradients against differences of the loss.

Stages are checked from the values that entered them, with the tolerances of their own tests.  The gradients' check against differences
is of the whole chain in FP64: h, y, dy and dh are BF16, each off by at most 2^-8 of its value, y's error reaches dy relative to y - target,
which is of y's size here; a directional derivative along the gradient's signs is a sum of absolute values, so five such roundings and
as much again for the size of y against y - target make 2^-4 of it, a bound that a missing or doubled term (a factor of 2, a sample's
rows) exceeds.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import adamw as OA
from oracle import layernorm as ON
from oracle import lora_apply as OL
from paper_2604_06916_b200 import workloads

pytestmark = pytest.mark.gpu

ROWS, K, N, R, POLICIES, SAMPLE = 420, 256, 384, 16, 2, 150
U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


class Step:
    """A user's program: what it keeps between steps and the step itself."""

    def __init__(self, B, seed, bits):
        g = torch.Generator(device="cuda").manual_seed(seed)
        randn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.B = B
        self.x, self.target = randn(ROWS, K).to(torch.bfloat16), randn(ROWS, N).to(torch.bfloat16)
        self.scale, self.shift = (0.2 * randn(3, K)).to(torch.bfloat16), (0.2 * randn(3, K)).to(torch.bfloat16)
        self.w, self.bias = (randn(N, K) * K ** -0.5).to(torch.bfloat16), (0.1 * randn(N)).to(torch.bfloat16)
        self.w_back = self.w.t().contiguous()
        self.scaling = torch.tensor([2.0, 0.5], device="cuda")
        self.offsets = torch.tensor([0, 150, 290, 291, 420], dtype=torch.int32, device="cuda")
        self.ids = torch.tensor([1, 0, -1, 1], dtype=torch.int32, device="cuda")
        self.a, self.b = randn(POLICIES, R, K) * R ** -0.5, 0.1 * randn(POLICIES, N, R)
        self.a16, self.b16 = self.a.to(torch.bfloat16), self.b.to(torch.bfloat16)
        self.plan = B.sol_adamw_plan([self.a, self.b], [torch.zeros_like(self.a), torch.zeros_like(self.b)], copies=[self.a16, self.b16], state_bits=bits)

    def run(self):
        B, s = self.B, {}
        s["a16"], s["b16"], s["a"], s["b"] = self.a16.clone(), self.b16.clone(), self.a.clone(), self.b.clone()
        s["h"], s["stats"] = B.sol_layernorm(self.x, self.scale, self.shift, SAMPLE, with_stats=True)
        s["base"] = B.bf16_linear(s["h"], self.w, self.bias)
        requests = (self.scaling, self.offsets, self.ids)
        s["y"], s["t"] = B.sol_lora_apply(s["h"], self.a16, self.b16, *requests, s["base"].clone(), with_t=True)
        s["dy"] = (s["y"].float() - self.target.float()).to(torch.bfloat16)          # of sum (y - target)^2 / 2
        s["shared"] = B.bf16_linear(s["dy"], self.w_back)
        s["dh"] = s["shared"].clone()
        s["da"], s["db"] = B.sol_lora_backward(s["dy"], s["h"], s["t"], self.a16, self.b16, *requests, dx=s["dh"])
        s["dx"], s["dscale"], s["dshift"] = B.sol_layernorm_backward(s["dh"], self.x, s["stats"], self.scale, SAMPLE)
        self.plan.set_grads([s["da"], s["db"]])
        B.sol_adamw_step(self.plan, lr=1e-2, seed=5)
        s["merged"], s["q"], s["sf"], s["T"] = B.nvfp4_requantize_lora(self.w, self.a16[0], self.b16[0], 2.0, layout=B.SF_ROW_MAJOR)
        return s

    def check(self, s, steps):
        rows = lambda t: ON.rows_of(f64(t), ROWS, SAMPLE)  # noqa: E731
        ref, bound, _, _ = ON.forward(f64(self.x), rows(self.scale) + 1.0, rows(self.shift), 1e-6)
        assert np.all(np.abs(f64(s["h"]) - ref) <= 2.0 ** -8 * np.abs(ref) + 100 * U * bound)
        requests = [f64(self.scaling), self.offsets.tolist(), self.ids.tolist()]
        factors = [f64(s["a16"]), f64(s["b16"])]
        ref, size, _, _ = OL.apply(f64(s["h"]), *factors, *requests, f64(s["base"]))
        assert np.all(np.abs(f64(s["y"]) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -16 * size)
        t = np.nan_to_num(f64(s["t"][:, :R]) + f64(s["t"][:, R:])) * (size[:, :1] > 0)
        da, db, dh, da_size, db_size, dh_size = OL.backward(f64(s["dy"]), f64(s["h"]), t, *factors, *requests, f64(s["shared"]))
        assert np.all(np.abs(f64(s["da"]) - da) <= 2.0 ** -16 * da_size) and np.all(np.abs(f64(s["db"]) - db) <= 2.0 ** -17 * db_size)
        assert np.all(np.abs(f64(s["dh"]) - dh) <= 2.0 ** -8 * np.abs(dh) + 2.0 ** -16 * dh_size)
        dx, dscale, dshift, *bounds = ON.backward(f64(s["dh"]), f64(self.x), rows(self.scale) + 1.0, 1e-6, SAMPLE)
        assert np.all(np.abs(f64(s["dx"]) - dx) <= 2.0 ** -8 * np.abs(dx) + 200 * U * bounds[0])
        assert np.all(np.abs(f64(s["dscale"]) - dscale) <= (SAMPLE + 120) * U * bounds[1])
        assert np.all(np.abs(f64(s["dshift"]) - dshift) <= (SAMPLE + 120) * U * bounds[2])
        if steps == 1:                                    # from zero states
            for p, before, grad, copy in ((self.a, s["a"], s["da"], self.a16), (self.b, s["b"], s["db"], self.b16)):
                g = grad.detach().cpu().numpy().reshape(-1)
                m, v = OA.moments(np.zeros_like(g), np.zeros_like(g), g, 0.9, 0.999)
                want, step = OA.parameters(f64(before).reshape(-1), m.astype(np.float64), v.astype(np.float64), 1, 1e-2, 0.9, 0.999, 1e-8, 0.01)
                assert np.all(np.abs(f64(p).reshape(-1) - want) <= U * (2 * np.abs(want) + 16 * step * np.abs(m) + 1e-3))
                assert torch.equal(copy, p.to(torch.bfloat16))
        merged, q, _, T = oracle.requantize_lora(workloads.to_bits(self.w), workloads.to_bits(self.a16[0]), workloads.to_bits(self.b16[0]), 2.0)
        assert np.array_equal(workloads.to_bits(s["merged"]), merged) and np.array_equal(s["q"].cpu().numpy(), q)
        assert self.plan.step.tolist() == [steps, 0]
        assert self.B.sol_last_device_status() == 0


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_stage_by_stage(B, bits):
    step = Step(B, 1, bits)
    step.check(step.run(), 1)
    step.check(step.run(), 2)


def test_captured_and_replayed_on_new_inputs(B):
    step = Step(B, 2, 8)
    step.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = step.run()
    other = Step(B, 3, 8)
    for name in ("x", "target", "scale", "shift"):
        getattr(step, name).copy_(getattr(other, name))
    step.offsets.copy_(torch.tensor([5, 100, 260, 300, 419], dtype=torch.int32))
    for n in (2, 3):
        graph.replay()
        torch.cuda.synchronize()
        step.check(s, n)


def test_gradients_against_differences_of_the_loss(B):
    step = Step(B, 4, 32)
    s = step.run()
    x, w, bias, target = (f64(t) for t in (step.x, step.w, step.bias, step.target))
    requests = [f64(step.scaling), step.offsets.tolist(), step.ids.tolist()]

    def loss(p):
        h = ON.forward(p["x"], ON.rows_of(1.0 + p["scale"], ROWS, SAMPLE), ON.rows_of(p["shift"], ROWS, SAMPLE), 1e-6)[0]
        y = OL.apply(h, p["a"], p["b"], *requests, h @ w.T + bias)[0]
        return 0.5 * float(((y - target) ** 2).sum())

    point = {"x": x, "scale": f64(step.scale), "shift": f64(step.shift), "a": f64(s["a16"]), "b": f64(s["b16"])}
    for name, grad in (("x", s["dx"]), ("scale", s["dscale"]), ("shift", s["dshift"]), ("a", s["da"]), ("b", s["db"])):
        g = f64(grad)
        for part in [slice(None)] if name == "x" else range(g.shape[0]):              # every sample and policy by itself
            d = np.zeros_like(g)
            d[part] = np.sign(g[part])
            e = 1e-5
            up, down = (loss({**point, name: point[name] + k * e * d}) for k in (1.0, -1.0))
            want, got = (up - down) / (2 * e), float((g * d).sum())
            assert abs(got - want) <= 2.0 ** -4 * got, (name, part, got, want)


def test_policies_unmerged_beside_a_quantized_projection(B):
    """The rollout's form: one NVFP4 projection for all candidates, each row's own adapter on top; the merged weight gives the same but
    for its rounding to BF16."""
    step = Step(B, 6, 32)
    wq, wsf, wts = B.nvfp4_quantize_weight(step.w)
    base = B.nvfp4_quantize_linear(step.x, wq, wsf, wts, step.bias)
    y = B.sol_lora_apply(step.x, step.a16, step.b16, step.scaling, step.offsets, step.ids, base.clone())
    ref, size, _, _ = OL.apply(f64(step.x), f64(step.a16), f64(step.b16), f64(step.scaling), step.offsets.tolist(), step.ids.tolist(), f64(base))
    assert np.all(np.abs(f64(y) - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -16 * size)
    one = B.sol_lora_apply(step.x[:1], step.a16, step.b16, step.scaling, step.offsets[:2].clamp(max=1), step.ids[:1], base[:1].clone())
    assert torch.equal(one, y[:1])
    assert torch.equal(y[290], base[290])


def test_two_streams_at_once(B):
    """Two steps that overlap, each with its own tensors and workspaces, give what they give alone."""
    alone = [Step(B, seed, 8).run() for seed in (7, 8)]
    torch.cuda.synchronize()
    steps = [Step(B, seed, 8) for seed in (7, 8)]
    streams = [torch.cuda.Stream() for _ in steps]
    torch.cuda.synchronize()
    got = []
    for step, stream in zip(steps, streams):
        with torch.cuda.stream(stream):
            got.append(step.run())
    torch.cuda.synchronize()
    for a, b in zip(alone, got):
        for name in a:
            if name == "t":        # the request without an adapter leaves its rows as they are
                rows = torch.ones(ROWS, dtype=torch.bool, device="cuda")
                rows[290] = False
                assert torch.equal(a[name][rows], b[name][rows])
            else:
                assert torch.equal(a[name], b[name]), name
