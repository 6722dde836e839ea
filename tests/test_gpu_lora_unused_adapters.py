"""GPU: adapters of the stack that no row of a batch has.  Whatever their factors and their scaling hold, their gradients are zeros and the
others' results stay as they are."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("M,offsets,ids", [(700, [0, 300, 300, 700], [2, 0, -1]), (3000, [0, 100, 3000, 3000], [4, 2, 1])])
@pytest.mark.parametrize("filler", [float("nan"), float("inf")])
def test_their_values_count_for_nothing(B, M, offsets, ids, filler):
    n, r, K, N = 5, 24, 328, 520
    g = torch.Generator(device="cuda").manual_seed(M)
    bf = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    x, y, dy, dx, a, b = bf(M, K), bf(M, N), bf(M, N), bf(M, K), bf(n, r, K), bf(n, N, r)
    scaling = torch.rand(n, generator=g, device="cuda") + 0.5
    requests = (torch.tensor(offsets, dtype=torch.int32, device="cuda"), torch.tensor(ids, dtype=torch.int32, device="cuda"))

    def step():
        z, t = B.sol_lora_apply(x, a, b, scaling, *requests, y.clone(), with_t=True)
        out = dx.clone()
        return (z, out, *B.sol_lora_backward(dy, x, t, a, b, scaling, *requests, dx=out))

    want = step()
    used = {i for s, e, i in zip(offsets, offsets[1:], ids) if e > s and i >= 0}
    unused = torch.tensor([i for i in range(n) if i not in used], device="cuda")
    for part in (a, b, scaling):
        part[unused] = filler
    got = step()
    B.sol_last_device_status()
    for grad in got[2:]:
        assert (grad[unused] == 0).all() and (grad[list(used)] != 0).any()
    assert all(torch.equal(p, q) for p, q in zip(want, got))
