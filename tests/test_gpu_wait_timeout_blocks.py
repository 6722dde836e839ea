"""The bounded waits of the block-sparse attention, run out for real: its loads are held back by the test hook, the waits expire after
a short limit, the kernel leaves through its normal teardown with the output untouched, the host reads SOL_ERR_TIMEOUT, and
the next ordinary call is right.  One item per CTA and several, lists of one block and of many, some of them empty (the walk
passes those before it stops).  No trap, no fault, no unbounded spin."""
import pytest
import torch

pytestmark = pytest.mark.gpu

SOL_ERR_TIMEOUT = 7
ATTENTION_SITE = 0xB        # high byte of the status word of the attention kernels' waits


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("batch,S,H,n", [(1, 1, 1, 1), (1, 300, 4, 3), (2, 1500, 40, 6)])
@pytest.mark.parametrize("empty", [False, True])
def test_wait_that_runs_out(B, D, batch, S, H, n, empty):
    g = torch.Generator(device="cuda").manual_seed(S + H + D)
    q, k, v = (torch.randn((batch, S, H, D), generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    nq = -(-S // 256)
    blocks = torch.randint(0, -(-S // 128), (batch, H, nq, n), generator=g, device="cuda").to(torch.int32)
    counts = torch.full((batch, H, nq), n, dtype=torch.int32, device="cuda")
    if empty:
        counts.view(-1)[1::3] = 0
    lens = torch.full((batch,), S, dtype=torch.int32, device="cuda")
    want = B.sol_attention_blocks(q, k, v, blocks, counts, lens)
    assert B.sol_last_device_status() == 0
    out = torch.full((batch, S, H, D), 3.0, dtype=torch.bfloat16, device="cuda")
    try:
        B.sol_set_wait_limit_cycles(1_000_000)      # about half a millisecond
        B.sol_test_hold_loads(True)
        B.sol_attention_blocks(q, k, v, blocks, counts, lens, out=out)
        with pytest.raises(B.SolError) as info:
            B.sol_last_device_status()
    finally:
        B.sol_test_hold_loads(False)
        B.sol_set_wait_limit_cycles(0)
    assert info.value.code == SOL_ERR_TIMEOUT
    assert (info.value.detail >> 8) == ATTENTION_SITE, hex(info.value.detail)
    listed = (counts > 0).repeat_interleave(256, dim=2)[:, :, :S].transpose(1, 2)       # [batch, S, H]
    assert torch.all(out[listed] == 3.0)            # no query with a list was written
    assert torch.all((out[~listed] == 3.0) | (out[~listed] == 0.0))
    B.sol_last_device_status()                      # the word was cleared by the read
    for _ in range(3):
        assert torch.equal(B.sol_attention_blocks(q, k, v, blocks, counts, lens), want)
    assert B.sol_last_device_status() == 0
