"""GPU: infinities among the values of one request.  They make its row (what is added to it), its adapter's gradients and its dx not
finite, and reach nobody else."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("where", ["x", "dy", "lora_a", "lora_b"])
def test_infinities_stay_with_their_request(B, where):
    M, n, r, K, N, bad = 450, 3, 16, 264, 392, 131
    g = torch.Generator(device="cuda").manual_seed(5)
    bf = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    v = {"x": bf(M, K), "dy": bf(M, N), "lora_a": bf(n, r, K), "lora_b": bf(n, N, r)}
    y, dx, scaling = bf(M, N), bf(M, K), torch.ones(n, device="cuda")
    requests = (torch.tensor([0, 130, 200, 450], dtype=torch.int32, device="cuda"), torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"))

    def step():
        out, add = dx.clone(), y.clone()
        z, t = B.sol_lora_apply(v["x"], v["lora_a"], v["lora_b"], scaling, *requests, add, with_t=True)
        da, db = B.sol_lora_backward(v["dy"], v["x"], t, v["lora_a"], v["lora_b"], scaling, *requests, dx=out)
        return z, out, da, db

    fine = step()
    v[where][1 if where.startswith("lora") else bad, 3] = float("inf")
    z, out, da, db = step()
    B.sol_last_device_status()
    rows = torch.zeros(M, dtype=torch.bool, device="cuda")
    rows[bad] = True
    if where.startswith("lora"):
        rows[130:200] = True
    for got, want in ((z, fine[0]), (out, fine[1])):
        assert torch.equal(got[~rows], want[~rows])
    for got, want in ((da, fine[2]), (db, fine[3])):
        assert torch.equal(got[[0, 2]], want[[0, 2]])
    if where in ("x", "lora_a"):
        assert not z[rows].isfinite().any()
    if where in ("dy", "lora_b"):
        assert not out[rows].isfinite().any()
    if where in ("x", "dy"):
        assert not (da[1].isfinite().all() or db[1].isfinite().all())
