"""GPU parity: block selection (exact) and block-sparse attention through the C ABI against the FP64 oracle.

Lists are compared for equality: means and scores are FP64 on both sides, and the inputs are such that no two
scores near a cut agree to 2^-40.  Attention: the tolerance of the dense kernel (oracle.attention.attention_tolerance).
"""
import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import block_sparse as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding
    binding.lib()
    return binding


def f64(t):
    return None if t is None else t.detach().to(torch.float64).cpu().numpy()


def make(batch, sq, skv, H, Hk, D, seed, fused=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if fused and sq == skv:
        x = torch.randn((batch, sq, (H + 2 * Hk) * D), generator=g, device="cuda").to(torch.bfloat16)
        return (x[:, :, :H * D].unflatten(2, (H, D)), x[:, :, H * D:(H + Hk) * D].unflatten(2, (Hk, D)),
                x[:, :, (H + Hk) * D:].unflatten(2, (Hk, D)))
    mk = lambda s, h: torch.randn((batch, s, h, D), generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    return mk(sq, H), mk(skv, Hk), mk(skv, Hk)


def check_select(B, q, k, count, first=0, lens=None):
    blocks, counts, scores = B.sol_select_blocks(q, k, count, first, lens, with_scores=True)
    want, wcounts, wscores = S.select(f64(q), f64(k), count, first, None if lens is None else lens.tolist())
    assert np.array_equal(counts.cpu().numpy(), wcounts)
    assert np.array_equal(blocks.cpu().numpy(), want)
    got, live = f64(scores), want >= 0
    assert np.all(got[~live] == -np.inf)
    # FP64 sums rounded once to FP32, and 2^-52 of the magnitudes summed where they cancel
    assert np.all(np.abs(got[live] - wscores[live]) <= 2.0 ** -23 * np.abs(wscores[live]) + 1e-13)
    plain = B.sol_select_blocks(q, k, count, first, lens)
    assert len(plain) == 2 and torch.equal(plain[0], blocks) and torch.equal(plain[1], counts)
    return blocks, counts


def check_attend(B, q, k, v, blocks, counts, lens=None, out=None):
    got = B.sol_attention_blocks(q, k, v, blocks, counts, lens, out=out)
    torch.cuda.synchronize()
    assert B.sol_last_device_status() == 0
    ref = S.attend(f64(q), f64(k), f64(v), blocks.cpu().numpy(), counts.cpu().numpy(), None if lens is None else lens.tolist())
    vn = np.repeat(f64(v), q.shape[2] // k.shape[2], axis=2)
    err, tol = np.abs(f64(got) - ref), OA.attention_tolerance(ref, vn)
    assert np.all(err <= tol), f"err/tol {np.max(err / tol):.3f} at {np.unravel_index((err / tol).argmax(), err.shape)}"
    return got


@pytest.mark.parametrize("batch,sq,skv,H,Hk,D,count,first", [
    (1, 1, 1, 1, 1, 64, 1, 0), (1, 1, 1000, 4, 2, 128, 3, 0), (2, 256, 128, 1, 1, 128, 1, 1), (1, 257, 129, 3, 1, 64, 2, 0),
    (2, 700, 1500, 6, 3, 64, 5, 2), (1, 2000, 2000, 5, 5, 128, 4, 4), (3, 300, 4500, 2, 1, 64, 7, 1), (1, 513, 640, 2, 2, 128, 40, 0)])
def test_selection(B, batch, sq, skv, H, Hk, D, count, first):
    q, k, _ = make(batch, sq, skv, H, Hk, D, batch + sq + skv, fused=True)
    check_select(B, q, k, count, first)


def test_selection_over_many_blocks(B):
    q, k, _ = make(1, 300, 128 * 600 + 5, 1, 1, 64, 3)          # 601 key blocks: one query block per CTA
    check_select(B, q, k, 33, 2)
    check_select(B, q, k, 601)
    check_select(B, q, k, 700, 1)


def test_many_blocks_of_both_signs_equal_or_nearly(B):
    # the search over the keys' bits: signs apart, all upper halves alike, exact ties across the cut
    q, k, _ = make(1, 256, 128 * 200, 1, 1, 64, 4)
    q[:] = 0
    q[..., 0] = 1.0
    k[:] = 0
    k[0, ::128, 0, 0] = torch.linspace(-3, 3, 200, device="cuda").to(torch.bfloat16)      # one row per block decides its mean
    for count in (1, 7, 100, 199, 200):
        check_select(B, q, k, count)
    k[0, ::128, 0, 0] = 1.0                                          # all equal
    check_select(B, q, k, 50, 3)
    k[0, 1::128, 0, 0] = torch.arange(200, device="cuda").to(torch.bfloat16) * 2.0 ** -40   # apart by 2^-40 only
    check_select(B, q, k, 50)
    k[0, 1::128, 0, 0] = (torch.arange(200, device="cuda") // 9).to(torch.bfloat16) * 2.0 ** -40
    for count in (5, 9, 14, 197):
        check_select(B, q, k, count, 2)
    k[0, ::128, 0, 0] = -1.0
    check_select(B, q, k, 14)


def test_equal_scores_go_to_the_lower_index(B):
    q, k, _ = make(1, 300, 1280, 2, 2, 64, 5)
    k = k[:, :128].repeat(1, 10, 1, 1)                          # ten equal blocks
    blocks, counts = check_select(B, q, k, 4)
    assert torch.equal(blocks, torch.arange(4, device="cuda", dtype=torch.int32).expand_as(blocks))
    k[:, 512:640] *= 2                                          # one block apart: above all for some rows, below for others
    check_select(B, q, k, 4)
    check_select(B, q, k, 1)
    zero = torch.zeros_like(k)
    blocks, _ = check_select(B, q, zero, 3, 1)
    assert blocks[0, 0, 0].tolist() == [0, 1, 2]
    check_select(B, torch.zeros_like(q), -zero, 3)              # negative zeros are zeros


def test_selection_with_lengths(B):
    q, k, _ = make(5, 300, 900, 2, 1, 64, 7)
    lens = torch.tensor([900, 0, 1, 129, 640], dtype=torch.int32, device="cuda")
    blocks, counts = check_select(B, q, k, 3, 1, lens)
    assert counts[1].abs().max() == 0 and torch.all(blocks[1] == -1) and torch.all(counts[2] == 1)
    odd = torch.tensor([1 << 30, -5, 900, 901, 128], dtype=torch.int32, device="cuda")    # held to [0, 900]
    check_select(B, q, k, 3, 0, odd)
    k[3, 129:] = float("nan")                                   # keys behind the length are not read into any mean
    check_select(B, q[3:4], torch.nan_to_num(k[3:4]), 2, 0, lens[3:4])
    a = B.sol_select_blocks(q, k, 3, 1, lens)
    assert torch.equal(a[0][3], blocks[3])


def test_small_and_large_values_in_one_mean(B):
    q, k, _ = make(1, 256, 512, 1, 1, 64, 11)
    k[:, ::2] *= 2.0 ** 20
    k[:, 1::4] *= 2.0 ** -20
    q[:, ::3] *= 2.0 ** -100
    k[:, 5] = 0
    k[:, 9] = 1e-39                                             # a subnormal
    check_select(B, q, k, 2)


def random_lists(batch, H, nq, n, top, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    blocks = torch.randint(0, top, (batch, H, nq, n), generator=g, device="cuda").to(torch.int32)
    counts = torch.randint(0, n + 1, (batch, H, nq), generator=g, device="cuda").to(torch.int32)
    return blocks, counts


@pytest.mark.parametrize("batch,sq,skv,H,Hk,D,n", [
    (1, 1, 1, 1, 1, 128, 1), (1, 256, 128, 1, 1, 64, 2), (2, 300, 700, 4, 2, 128, 4), (1, 130, 1000, 3, 3, 64, 5),
    (1, 1000, 513, 6, 1, 128, 3), (2, 515, 515, 2, 2, 64, 9), (1, 1, 4000, 8, 4, 64, 20)])
def test_attention_over_random_lists(B, batch, sq, skv, H, Hk, D, n):
    # in any order, with repeats, some lists empty
    q, k, v = make(batch, sq, skv, H, Hk, D, sq + skv + H, fused=True)
    blocks, counts = random_lists(batch, H, -(-sq // 256), n, -(-skv // 128), 1)
    check_attend(B, q, k, v, blocks, counts)
    check_attend(B, q, k, v, blocks, torch.full_like(counts, n))


@pytest.mark.parametrize("D", [64, 128])
def test_all_blocks_in_order_is_the_dense_kernel(B, D):
    q, k, v = make(2, 600, 1111, 3, 3, D, 13)
    nk = -(-1111 // 128)
    blocks = torch.arange(nk, device="cuda", dtype=torch.int32).expand(2, 3, 3, nk).contiguous()
    counts = torch.full((2, 3, 3), nk, dtype=torch.int32, device="cuda")
    want = B.sol_attention_bf16(q, k, v)
    assert torch.equal(B.sol_attention_blocks(q, k, v, blocks, counts), want)
    # shared key heads: the same as repeating them
    k1, v1 = k[:, :, :1].contiguous(), v[:, :, :1].contiguous()
    rep = B.sol_attention_bf16(q, k1.expand(-1, -1, 3, -1).contiguous(), v1.expand(-1, -1, 3, -1).contiguous())
    assert torch.equal(B.sol_attention_blocks(q, k1, v1, blocks, counts), rep)


def test_bad_entries_counts_and_lengths(B):
    q, k, v = make(4, 520, 700, 2, 1, 128, 17)
    blocks, counts = random_lists(4, 2, 3, 6, 6, 2)
    counts.fill_(6)
    clean = check_attend(B, q, k, v, blocks, counts)
    # entries that name nothing, wherever they stand, are skipped
    wide = torch.full((4, 2, 3, 12), -1, dtype=torch.int32, device="cuda")
    wide[..., 1::2] = blocks
    wide[..., 2] = 6
    wide[..., 4] = 1 << 30
    wide[..., 6] = -(1 << 31)
    wide[..., 8] = 8191
    got = B.sol_attention_blocks(q, k, v, wide, torch.full_like(counts, 12))
    assert torch.equal(got, clean)
    assert torch.equal(B.sol_attention_blocks(q, k, v, blocks, torch.full_like(counts, 1 << 30)), clean)     # held to 6
    assert torch.all(B.sol_attention_blocks(q, k, v, blocks, torch.full_like(counts, -3)) == 0)
    assert torch.all(B.sol_attention_blocks(q, k, v, torch.full_like(blocks, 77), counts) == 0)
    lens = torch.tensor([0, 1, 700, 300], dtype=torch.int32, device="cuda")
    got = check_attend(B, q, k, v, blocks, counts, lens)
    assert torch.all(got[0] == 0)
    # what stands behind the lengths does not matter
    k2, v2 = k.clone(), v.clone()
    for b, n in enumerate(lens.tolist()):
        k2[b, n:], v2[b, n:] = 7.0, 3.0
    assert torch.equal(B.sol_attention_blocks(q, k2, v2, blocks, counts, lens), got)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -3.0e38])
def test_anything_may_stand_behind_the_lengths(B, D, junk):
    q, k, v = make(3, 520, 900, 2, 1, D, 37)
    lens = torch.tensor([899, 1, 390], dtype=torch.int32, device="cuda")
    blocks, counts = random_lists(3, 2, 3, 9, 8, 5)
    blocks[..., 0] = 7 - 4 * torch.tensor([0, 1, 1], device="cuda", dtype=torch.int32)[:, None, None]    # the ragged block: 7, 3, 3
    blocks[..., 4] = blocks[..., 0]                                                                     # twice
    counts.fill_(9)
    want = check_attend(B, q, k, v, blocks, counts, lens)
    for b, n in enumerate(lens.tolist()):
        k[b, n:], v[b, n:] = junk, junk
    assert torch.equal(B.sol_attention_blocks(q, k, v, blocks, counts, lens), want)
    a = B.sol_select_blocks(q, k, 3, 1, lens)
    for b, n in enumerate(lens.tolist()):
        k[b, n:] = 0
    c = B.sol_select_blocks(q, k, 3, 1, lens)
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pattern", ["2000102", "1000000", "0001000", "3010030", "0000000"])
def test_runs_of_empty_lists(B, D, pattern):
    # Blocks of the kernel stay and walk every sm_count-th list: those of one block go through `pattern`, others through it
    # begun elsewhere.
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    H = sms * len(pattern)
    q, k, v = make(1, 5, 300, H, H, D, len(pattern) + D)
    counts = torch.tensor([int(pattern[(h // sms + h % sms % 3) % len(pattern)]) for h in range(H)], dtype=torch.int32, device="cuda").view(1, H, 1)
    blocks = torch.tensor([2, 0, 1], dtype=torch.int32, device="cuda").expand(1, H, 1, 3).contiguous()
    got = check_attend(B, q, k, v, blocks, counts)
    assert torch.all(got[0, :, counts.view(H) == 0] == 0)


def test_sharp_scores_and_output_view(B):
    q, k, v = make(1, 400, 1400, 2, 2, 128, 19)
    q = (q.float() * 6).to(torch.bfloat16)
    blocks, counts = random_lists(1, 2, 2, 8, 11, 3)
    wide = torch.full((1, 402, 3 * 256), 5.0, dtype=torch.bfloat16, device="cuda")
    view = wide[:, 1:401, 256:512].unflatten(2, (2, 128))
    got = check_attend(B, q, k, v, blocks, counts, out=view)
    assert got is view
    assert torch.all(wide[:, :, :256] == 5) and torch.all(wide[:, :, 512:] == 5) and torch.all(wide[:, 0] == 5) and torch.all(wide[:, 401] == 5)


def test_longest_list(B):
    q, k, v = make(1, 20, 256, 1, 1, 128, 23)
    blocks = torch.randint(0, 2, (1, 1, 1, 8192), device="cuda").to(torch.int32)
    check_attend(B, q, k, v, blocks, torch.full((1, 1, 1), 300, dtype=torch.int32, device="cuda"))


def test_selection_then_attention_captured_and_on_another_stream(B):
    q, k, v = make(2, 1500, 1500, 4, 2, 128, 29, fused=True)
    lens = torch.tensor([1500, 1111], dtype=torch.int32, device="cuda")

    def run():
        blocks, counts = B.sol_select_blocks(q, k, 4, 1, lens)
        return blocks, counts, B.sol_attention_blocks(q, k, v, blocks, counts, lens)

    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for t in got:
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    # new data in the same buffers: the captured lists follow it
    q.copy_(q.flip(1))
    graph.replay()
    torch.cuda.synchronize()
    again = run()
    assert all(torch.equal(a, b) for a, b in zip(again, got))


def test_refusals_on_the_device(B):
    q, k, v = make(1, 300, 300, 4, 2, 64, 31)
    blocks, counts = random_lists(1, 4, 2, 3, 3, 4)
    for bad in (dict(blocks=blocks.long()), dict(blocks=blocks[:, :, :1]), dict(blocks=blocks[..., ::2]), dict(counts=counts[..., :1]),
                dict(counts=counts.long()), dict(v=v[:, :200]), dict(kv_lens=torch.zeros(2, dtype=torch.int32, device="cuda")),
                dict(out=torch.empty_like(k))):
        args = dict(q=q, k=k, v=v, blocks=blocks, counts=counts, kv_lens=None, out=None)
        args.update(bad)
        with pytest.raises((TypeError, ValueError)):
            B.sol_attention_blocks(args["q"], args["k"], args["v"], args["blocks"], args["counts"], args["kv_lens"], args["out"])
    with pytest.raises(ValueError):
        B.sol_select_blocks(q, k, 0)
    with pytest.raises(B.SolError):
        B.sol_select_blocks(q, k, 2, 3)
    with pytest.raises(B.SolError):
        B.sol_select_blocks(q, k, 2, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
