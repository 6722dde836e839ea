"""The gradient of lora_a keeps dt's 24 bits: dt enters its product with x in three BF16 parts, and two would not do.

Every sum is chosen so that FP32 holds it: a row of dy has ones at three places and zeros elsewhere, the factor's three values there are
b0 in [1, 2) with 8 bits, b1 = 2^-9 times 8 bits and b2 = 2^-18 times 3 bits, so dt = b0 + b1 + b2 is a multiple of 2^-20 below 2.01;
x holds powers of two in one row and the other rows' dy is zero, so the gradient is dt times a power of two.
Tolerance: an adder that aligns its terms to the largest and keeps 23 bits below it loses nothing; one place of 2^-23 is allowed
for each of the four additions on the way (two of dt, two of its parts): 2^-21 of the value.  Two parts lose up to 2^-17 of it.
"""
import pytest
import torch

TOLERANCE = 2.0 ** -21


def factor(n, r, N, places, seed):
    """lora_b [n, N, r] with the three values at `places`, anything at the others, and dt [n, r] in FP64."""
    g = torch.Generator().manual_seed(seed)
    whole = lambda lo, hi: torch.randint(lo, hi, (n, r), generator=g).double()  # noqa: E731
    parts = (whole(128, 256) * 2.0 ** -7, whole(128, 256) * 2.0 ** -16, whole(4, 8) * 2.0 ** -20)
    b = torch.randn((n, N, r), generator=g).to(torch.bfloat16)
    for at, part in zip(places, parts):
        b[:, at] = part.to(torch.bfloat16)
        assert torch.equal(b[:, at].double(), part)
    return b, sum(parts)


def in_parts(dt, count):
    """dt as the sum of `count` BF16 parts, each what the ones before it left."""
    left, total = dt.float(), torch.zeros_like(dt)
    assert torch.equal(left.double(), dt)
    for _ in range(count):
        part = left.to(torch.bfloat16)
        total, left = total + part.double(), left - part.float()
    return total


def test_two_parts_would_be_seen():
    dt = factor(8, 64, 16, (0, 5, 9), 1)[1]
    assert torch.equal(in_parts(dt, 3), dt)
    off = (in_parts(dt, 2) - dt).abs() / dt
    assert (off > 2 * TOLERANCE).double().mean() > 0.5 and off.max() <= 2.0 ** -17


@pytest.mark.gpu
@pytest.mark.parametrize("M,r,K,N", [(1, 8, 64, 16), (1, 32, 3000, 328), (300, 24, 264, 1000), (2500, 64, 520, 4104), (129, 40, 72, 136)])
def test_gradient_of_lora_a(M, r, K, N):
    from paper_2604_06916_b200 import binding as B
    n, row = 2, M // 2
    places = (1, N // 2, N - 3)
    b, dt = factor(n, r, N, places, M + r)
    g = torch.Generator().manual_seed(r)
    x = torch.ldexp(torch.ones(M, K), torch.randint(-6, 7, (M, K), generator=g).float()).to(torch.bfloat16)
    dy = torch.zeros((M, N), dtype=torch.bfloat16)
    dy[row, list(places)] = 1.0
    a, t = torch.randn((n, r, K), generator=g).to(torch.bfloat16), torch.zeros((M, 2 * r), dtype=torch.bfloat16)
    requests = (torch.tensor([0, row, M], dtype=torch.int32).cuda(), torch.tensor([0, 1], dtype=torch.int32).cuda())
    da, db = B.sol_lora_backward(dy.cuda(), x.cuda(), t.cuda(), a.cuda(), b.cuda(), torch.ones(n).cuda(), *requests)
    B.sol_last_device_status()
    want = dt[1][:, None] * x[row].double()
    off = (da[1].double().cpu() - want).abs() / want
    assert off.max() <= TOLERANCE, f"{float(off.max()):.3g} of the value"
    assert (da[0] == 0).all() and (db == 0).all()
