"""GPU: what gradients that are not finite, and finite ones whose squares are not, leave behind, as the C header says it."""
import pytest
import torch

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("eps", [1e-8, 1e-12])
@pytest.mark.parametrize("p16", [False, True])
def test_fp32_states(B, eps, p16):
    p = torch.full((64,), 0.5, device="cuda").to(torch.bfloat16 if p16 else torch.float32)
    g = torch.full((64,), 1e-3, device="cuda")
    g[3], g[20], g[21], g[40] = NAN, INF, -INF, 1e20
    plan = B.sol_adamw_plan([p], [g])
    fine = torch.ones(64, dtype=torch.bool, device="cuda")
    fine[[3, 20, 21, 40]] = False
    for step in range(2):
        B.sol_adamw_step(plan, 1e-3, eps=eps)
        assert p[[3, 20, 21]].isnan().all() and p[fine].isfinite().all() and (p[fine] < 0.5).all()
        assert abs(float(p[40]) - 0.5) <= 2 * 1e-5 + 2.0 ** -8          # no update but the decay
        g[fine.logical_not()] = 1e-3
    m, v = plan.m[0], plan.v[0]
    assert m[3].isnan() and v[3].isnan() and m[20] == INF and m[21] == -INF and (v[[20, 21, 40]] == INF).all() and m[40].isfinite()
    assert m[fine].isfinite().all() and v[fine].isfinite().all()


@pytest.mark.parametrize("seed", [None, 9])
def test_8_bit_states(B, seed):
    p, g = torch.full((96,), 0.5, device="cuda"), torch.full((96,), 1e-3, device="cuda")
    g[3], g[40], g[41], g[70] = NAN, INF, -INF, 1e20
    plan = B.sol_adamw_plan([p], [g], state_bits=8)
    bad = torch.tensor([3, 40, 41], device="cuda")
    B.sol_adamw_step(plan, 1e-3, seed=seed)
    assert p[bad].isnan().all() and abs(float(p[70]) - 0.5) <= 1e-5
    assert ((plan.m[0][bad] & 127) == 127).all() and (plan.v[0][[3, 40, 41, 70]] == 127).all() and (plan.m[0][70] & 127) != 127
    g[[3, 40, 41, 70]] = 1e-3
    B.sol_adamw_step(plan, 1e-3, seed=seed)
    fine = torch.ones(96, dtype=torch.bool, device="cuda")
    fine[[3, 40, 41, 70]] = False
    assert p[~fine].isnan().all() and p[fine].isfinite().all()


def test_a_factor_that_is_not_finite(B):
    p, g, factor = torch.ones(40, device="cuda"), torch.ones(40, device="cuda"), torch.tensor(NAN, device="cuda")
    B.sol_adamw_step(B.sol_adamw_plan([p], [g]), 1e-3, grad_scale=factor)
    assert p.isnan().all()
