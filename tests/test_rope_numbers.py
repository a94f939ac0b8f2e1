"""Rotary positions: numbers that do not fit what the C entry points take."""
import pytest

from paper_2604_18616_amd import binding


def test_frequencies_of_numbers_beyond_32_bits_are_refused():
    """None is cut to its lower half: 2^32 + 4096 positions are not 4096."""
    pytest.importorskip("torch")
    for kw in (dict(original_len=(1 << 32) + 4096), dict(original_len=1 << 31), dict(original_len=-(1 << 32) + 4096)):
        with pytest.raises(ValueError, match="32 bits"):
            binding.rope_frequencies(64, factor=4.0, device="cpu", **kw)
    with pytest.raises(ValueError, match="32 bits"):
        binding.rope_frequencies((1 << 32) + 64, device="cpu")
    most = binding.rope_frequencies(64, factor=4.0, original_len=(1 << 31) - 1, device="cpu")
    assert most.shape == (32,) and float(most[0]) == 1.0


@pytest.mark.gpu
def test_more_frequencies_than_32_bits_count_are_refused():
    import torch
    q = torch.zeros((1, 1, 1, 64), dtype=torch.bfloat16, device="cuda")
    far = torch.empty((1 << 31) + 32, dtype=torch.float64, device="cuda")        # twice that is 64 in 32 bits
    with pytest.raises(ValueError, match="32 bits"):
        binding.rope_bf16(q, torch.zeros(1, dtype=torch.int32, device="cuda"), far)
