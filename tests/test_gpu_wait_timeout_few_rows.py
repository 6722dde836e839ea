"""The bounded waits of the few-row 4-bit linears, run out for real: x is held back from the products by the test hook, the waits
expire after a short limit, the kernel leaves through its normal teardown with its copies landed and y untouched, the host
reads SOL_ERR_TIMEOUT, and the next ordinary call is right.  Every form: x prepared by the products' blocks or in a launch of its
own, K shared by a cluster or not, a ring that is refilled and one that is not.  No trap, no fault, no unbounded spin."""
import pytest
import torch

pytestmark = pytest.mark.gpu

SOL_ERR_TIMEOUT = 7
FEW_ROW_SITE = 0xC          # high byte of the status word of these kernels' waits


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("fmt", ["nv", "mx"])
@pytest.mark.parametrize("M,N,K", [(1, 40, 64), (4, 264, 3072), (3, 19072, 256), (2, 19072, 2048), (8, 264, 512), (16, 136, 15360), (70, 9600, 1536)])
def test_wait_that_runs_out(B, fmt, M, N, K):
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    w = (torch.randn((N, K), generator=g, device="cuda") * K ** -0.5).to(torch.bfloat16)
    x = torch.randn((M, K), generator=g, device="cuda").to(torch.bfloat16)
    weight = B.nvfp4_quantize_weight(w) if fmt == "nv" else B.mxfp4_quantize(w)
    entry = B.nvfp4_matvec if fmt == "nv" else B.mxfp4_matvec
    want = entry(x, *weight, activation=B.ACT_SILU)
    B.sol_last_device_status()
    wide = torch.full((M + 2, N + 16), 3.0, dtype=torch.bfloat16, device="cuda")
    try:
        B.sol_set_wait_limit_cycles(1_000_000)      # about half a millisecond
        B.sol_test_hold_loads(True)
        entry(x, *weight, activation=B.ACT_SILU, out=wide[1:1 + M, 8:8 + N])
        with pytest.raises(B.SolError) as info:
            B.sol_last_device_status()
    finally:
        B.sol_test_hold_loads(False)
        B.sol_set_wait_limit_cycles(0)
    assert info.value.code == SOL_ERR_TIMEOUT
    assert (info.value.detail >> 8) == FEW_ROW_SITE, hex(info.value.detail)
    assert torch.all(wide == 3.0)                   # the held launch wrote nothing
    B.sol_last_device_status()                      # the word was cleared by the read
    for _ in range(3):
        assert torch.equal(entry(x, *weight, activation=B.ACT_SILU), want)
    B.sol_last_device_status()
