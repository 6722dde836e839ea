"""CPU: a scale or shift that is one vector expanded over the samples (row pitch 0) reaches the C entry with that pitch, which the
entry refuses: the kernel would read rows that the vector does not have."""
import types

import pytest
import torch

SAMPLES, K = 3, 64


@pytest.fixture(scope="module")
def B():
    from paper_2604_06916_b200 import binding, build

    build.build()
    binding.lib()
    return binding


@pytest.fixture
def passed(B, monkeypatch):
    """The arguments that the binding would hand to the library, from host tensors; nothing is launched."""
    calls = []
    entry = lambda *args: calls.append(args) or 0  # noqa: E731
    monkeypatch.setattr(B, "lib", lambda: types.SimpleNamespace(sol_layernorm=entry, sol_layernorm_backward=entry,
                                                                sol_layernorm_backward_workspace_bytes=lambda *a: 0))
    monkeypatch.setattr(B, "_raw_stream", lambda index: 0)
    return calls


def vectors():
    x = torch.zeros((6, K), dtype=torch.bfloat16)
    one = torch.zeros((1, K), dtype=torch.bfloat16)
    return x, one.expand(SAMPLES, K), torch.zeros((SAMPLES, 2 * K), dtype=torch.bfloat16)[:, :K]


@pytest.mark.parametrize("which", ["scale", "shift", "both"])
def test_forward_passes_pitch_0_on(B, passed, which):
    x, wide, _ = vectors()
    B.sol_layernorm.__wrapped__(x, wide if which != "shift" else None, wide if which != "scale" else None, 2)
    assert passed[0][6] == 0


def test_backward_passes_pitch_0_on(B, passed):
    x, wide, _ = vectors()
    B.sol_layernorm_backward.__wrapped__(x, x, torch.zeros((6, 2)), wide, 2)
    assert passed[0][6] == 0


def test_other_pitches(B, passed):
    x, _, slices = vectors()
    B.sol_layernorm.__wrapped__(x, slices, slices, 2)
    B.sol_layernorm.__wrapped__(x, None, None, 2)
    B.sol_layernorm.__wrapped__(x, slices[:1], slices[:1])
    assert [c[6] for c in passed] == [2 * K, K, K]


@pytest.mark.parametrize("pitch", [0, 8, K - 8])
def test_the_entries_refuse_rows_that_overlap(B, pitch):
    """With addresses that are never read: shapes are checked first."""
    at = 4096
    bad_shape = B.lib().sol_layernorm(at, 6, 0, K, None, None, K, 2, 1.0, 1e-6, at, K, None, None)
    assert bad_shape != 0
    for scale, shift in ((at, None), (None, at), (at, at)):
        assert B.lib().sol_layernorm(at, 6, K, K, scale, shift, pitch, 2, 1.0, 1e-6, at, K, None, None) == bad_shape
    assert B.lib().sol_layernorm_backward(at, K, at, K, at, at, pitch, 6, K, 2, 1.0, at, K, None, None, None, 0, None) == bad_shape


@pytest.mark.gpu
def test_expanded_vectors_are_refused_on_the_device(B):
    x, wide, _ = (t.cuda() if t.stride(0) else t[:1].cuda().expand(SAMPLES, K) for t in vectors())
    assert wide.stride(0) == 0
    for scale, shift in ((wide, None), (None, wide), (wide, wide)):
        with pytest.raises(B.SolError):
            B.sol_layernorm(x, scale, shift, 2)
    with pytest.raises(B.SolError):
        B.sol_layernorm_backward(x, x, torch.zeros((6, 2), device="cuda"), wide, 2)
    # the same vector for all rows is a single sample
    x.normal_()
    one = torch.randn((1, K), device="cuda").to(torch.bfloat16)
    y = B.sol_layernorm(x, one, one)
    assert torch.equal(y, B.sol_layernorm(x, one.repeat(SAMPLES, 1), one.repeat(SAMPLES, 1), 2))
