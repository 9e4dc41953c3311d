"""Checks of the clear binding that need no GPU: a handle without a device stands in, and no call gets past them."""

import pytest
import torch


@pytest.fixture
def handle():
    from paper_2609_16915_gb300 import clear
    c = clear.Clear.__new__(clear.Clear)
    c._h, c.device, c._L = None, -1, None          # (tensors of the CPU are on device -1; a call would fail on None)
    return c


@pytest.mark.parametrize("size,channels,inner", [(8192, 129, 64), (8192, 128, 65), (8191, 5, 5), (0, 1, 1)])
def test_packed_weights_of_another_size(handle, size, channels, inner):
    """A buffer that does not hold channels x inner would be read past its end."""
    from paper_2609_16915_gb300 import clear
    w = clear.PackedWeights(torch.zeros(size, dtype=torch.int8), channels, inner)
    q, s = torch.zeros((2, inner), dtype=torch.int8), torch.ones(2)
    with pytest.raises(ValueError, match="weights"):
        handle.linear(q, s, w, torch.ones(channels), torch.empty((2, channels)))
    with pytest.raises(ValueError, match="weights"):
        handle.linear_codes(q, s, w, torch.ones(channels), torch.empty((2, channels), dtype=torch.uint8), 4, 0.0, 1.0)


@pytest.mark.parametrize("channels,inner", [(1, 1), (128, 64), (129, 65), (1000, 768), (5, 131071)])
def test_packed_size_is_the_library_s(channels, inner):
    from paper_2609_16915_gb300 import build, clear, load
    build.build()
    assert clear.packed_size(channels, inner) == load().rosetta_clear_packed_bytes(channels, inner)
