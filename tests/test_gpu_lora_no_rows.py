"""GPU: adapters of a batch in which no request has both rows and an adapter.  Nothing of y and dx changes, the factors' gradients are
zeros, and they are there for what is launched next, also in a captured graph."""
import pytest
import torch

pytestmark = pytest.mark.gpu
M, K, N, R, ADAPTERS = 4000, 512, 1024, 32, 6


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


REQUESTS = [([0, 1500, 4000], [-1, ADAPTERS]), ([0, 0, 0, 0], [0, 3, 5]), ([4000, 4000, 4000], [1, 1]), ([0, 0, 2000, 2000], [2, -7, 4])]


@pytest.mark.parametrize("offsets,ids", REQUESTS)
@pytest.mark.parametrize("captured", [False, True])
def test_zeros_and_nothing_else(B, offsets, ids, captured):
    g = torch.Generator(device="cuda").manual_seed(1)
    bf = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    x, y, dy, dx, a, b = bf(M, K), bf(M, N), bf(M, N), bf(M, K), bf(ADAPTERS, R, K), bf(ADAPTERS, N, R)
    t = torch.full((M, 2 * R), float("nan"), dtype=torch.bfloat16, device="cuda")
    scaling = torch.ones(ADAPTERS, device="cuda")
    requests = (torch.tensor(offsets, dtype=torch.int32, device="cuda"), torch.tensor(ids, dtype=torch.int32, device="cuda"))
    y0, dx0 = y.clone(), dx.clone()

    def step():
        # what the gradients' memory held before is not zero
        torch.full((8 * ADAPTERS * R * (K + N),), float("nan"), device="cuda")
        B.sol_lora_apply(x, a, b, scaling, *requests, y)
        da, db = B.sol_lora_backward(dy, x, t, a, b, scaling, *requests, dx=dx)
        return da, db, da + 1.0, db + 1.0

    step()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        for _ in range(20):
            for v in out:
                v.fill_(float("nan"))
            graph.replay()
            assert all(bool((v == i // 2).all()) for i, v in enumerate(out))
    else:
        for _ in range(20):
            assert all(bool((v == i // 2).all()) for i, v in enumerate(step()))
    B.sol_last_device_status()
    assert torch.equal(y, y0) and torch.equal(dx, dx0)
