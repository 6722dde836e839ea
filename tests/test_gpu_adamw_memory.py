"""GPU: a plan whose tensors' memory has been changed under it takes no step: it would go to memory that is somebody else's by then."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


@pytest.fixture
def parts():
    g = torch.Generator(device="cuda").manual_seed(3)
    tensors = lambda: [torch.randn(n, generator=g, device="cuda") for n in (64, 300, 0, 32)]  # noqa: E731
    params, grads = tensors(), tensors()
    return params, grads, [p.to(torch.bfloat16) for p in params]


def state(plan, tensors):
    return [t.clone() for t in (*tensors, *plan.m, *plan.v, plan.step)]


@pytest.mark.parametrize("which", ["params", "copies"])
def test_other_memory_is_refused(B, parts, which):
    plan = B.sol_adamw_plan(*parts)
    B.sol_adamw_step(plan, 1e-3)
    t = dict(zip(("params", "grads", "copies"), parts))[which][1]
    old = t.detach()                                     # the memory that the plan knows stays alive, so that this test is safe
    t.data = t.detach().clone()
    everything = [p for part in parts for p in part] + [old]
    before = state(plan, everything)
    with pytest.raises(ValueError, match=which):
        B.sol_adamw_step(plan, 1e-3)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, state(plan, everything)))
    t.data = old
    B.sol_adamw_step(plan, 1e-3)
    assert plan.step.tolist() == [2, 0]


def test_other_gradients_do_not_bring_other_parameters(B, parts):
    """A parameter that has become longer (at the same address) keeps the length that its states have; one at another address is refused."""
    flat = torch.zeros(512, device="cuda")
    params, grads = [flat[:64], torch.zeros(32, device="cuda")], [torch.ones(64, device="cuda"), torch.ones(32, device="cuda")]
    plan = B.sol_adamw_plan(params, grads)
    params[0].data = flat
    with pytest.raises(TypeError):
        plan.set_grads([torch.ones(512, device="cuda"), grads[1]])
    plan.set_grads([2.0 * g for g in grads])
    B.sol_adamw_step(plan, 1e-3)
    assert (flat[:64] != 0).all() and (flat[64:] == 0).all()
    params[1].data = torch.zeros(32, device="cuda")
    plan.set_grads(grads)
    with pytest.raises(ValueError, match="params"):
        B.sol_adamw_step(plan, 1e-3)


def test_lists_that_the_caller_changes(B, parts):
    """The plan's tensors are those that it was made of, also where a list that it was given or offers holds others by now."""
    params, grads, _ = parts
    plan = B.sol_adamw_plan(params, grads)
    states = [*plan.m, *plan.v]
    mine = list(params)
    params[0], plan.m[0], plan.v[0] = torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
    before = [t.clone() for t in (*mine, *states)]
    B.sol_adamw_step(plan, 1e-3)
    torch.cuda.synchronize()
    assert all(not torch.equal(a, b) for a, b in zip(before, (*mine, *states)) if a.numel())
    assert (params[0] == 0).all() and (plan.m[0] == 0).all()
