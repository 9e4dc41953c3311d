"""Argument checks of rosetta_clear_* that need no GPU, and the definitions that the GPU
tests compare with, against hand-computed values."""

import ctypes

import numpy as np
import pytest
import torch

from tests import clear_util as U


@pytest.fixture(scope="module")
def lib():
    import shutil
    import os
    if not (shutil.which("nvcc") or os.path.exists("/usr/local/cuda/bin/nvcc")):
        pytest.skip("nvcc not available")
    from paper_2609_16915_gb300 import build
    build.build()
    import paper_2609_16915_gb300 as R
    return R.load()


def test_null_handles_and_sizes_out_of_range(lib):
    three = (ctypes.c_int64 * 3)(64, 64, 64)
    assert lib.rosetta_clear_init(None, 0, 0) == -1
    assert lib.rosetta_clear_norm(None, 0, None, 1, None, 0, None, 0.0, 0, 1, None, 0, None, 1, None, None) == -1
    assert lib.rosetta_clear_pack_weights(None, None, 1, 1, 1, None, None) == -1
    assert lib.rosetta_clear_linear(None, None, 1, None, 0, None, None, None, 1, 1, 0, None, 1, None) == -1
    assert lib.rosetta_clear_linear_codes(None, None, 1, None, 0, None, None, None, 1, 1, 4, 0.0, 1.0, None, 1, None, None, 0,
                                          None) == -1
    assert lib.rosetta_clear_cache_append(None, 0, None, three, None, three, 0, 0, 1, 64, None, None, three, None, None, 1, 16,
                                          None, 1, None, None) == -1
    assert lib.rosetta_clear_attention(None, 0, None, three, 0, 0, 1, 1, 64, None, None, three, None, None, 1, 16, None, 1, None,
                                       1.0, None, three, None) == -1
    assert lib.rosetta_clear_sync_status(None, None) == -1
    lib.rosetta_clear_destroy(None)


@pytest.mark.parametrize("channels,inner,size", [(1, 1, 8192), (128, 64, 8192), (129, 65, 4 * 8192), (3, 131071, 2048 * 8192),
                                                 (0, 5, 0), (5, 0, 0), (5, 131072, 0), ((1 << 24) + 1, 1, 0)])
def test_packed_bytes(lib, channels, inner, size):
    assert lib.rosetta_clear_packed_bytes(channels, inner) == size


def test_reference_norm_by_hand():
    y, scale, h = U.norm(torch.tensor([[3.0, -4.0]]), torch.tensor([[0.0, 8.0]]), torch.tensor([1.0, 2.0]), 0.0)
    assert h.tolist() == [[3.0, 4.0]]                          # rms sqrt(12.5)
    assert np.allclose(y.numpy(), [[3 / 12.5 ** 0.5, 8 / 12.5 ** 0.5]]) and np.allclose(scale.numpy(), 8 / 12.5 ** 0.5 / 127)


def test_reference_append_by_hand():
    """A page of four rows: two old ones at scale 1, a new one four times as large."""
    cache, scale = torch.zeros(2, 1, 4, 4, dtype=torch.int8), torch.ones(2, 1)
    cache[1, 0, 0], cache[1, 0, 1], cache[1, 0, 3] = 100, -6, 77
    x = torch.tensor([508.0, -4.0, 2.0, 0.0]).reshape(1, 1, 1, 4)
    c, s = U.append(x, cache, scale, torch.tensor([[1]]), [2])
    assert s.tolist() == [[1.0], [4.0]]
    # 100/4 = 25, -6/4 = -1.5 -> -2 (ties to even), 2/4 = 0.5 -> 0; the row behind stays
    assert c[1, 0].tolist() == [[25] * 4, [-2] * 4, [127, -1, 0, 0], [77] * 4]


def test_reference_attention_by_hand():
    """Two positions with equal scores: the mean of their values; the first token sees only the first."""
    k, v = torch.ones(1, 1, 4, 4, dtype=torch.int8), torch.zeros(1, 1, 4, 4, dtype=torch.int8)
    v[0, 0, 0], v[0, 0, 1] = 10, 30
    one = torch.ones(1, 1)
    out, size = U.attention(torch.ones(1, 3, 1, 4), k, v, one, 0.5 * one, torch.tensor([[0]]), [2], 1.0)
    assert np.allclose(out[0, :, 0].numpy(), [[0] * 4, [5] * 4, [10] * 4])
    assert torch.equal(out, size)


def test_reference_codes_by_hand():
    y = np.array([[-9.0, -4.0, -3.51, -3.5, 3.49, 3.5, 99.0, np.nan]], np.float32)
    assert U.codes(y, 4, -4.0, 4.0).tolist() == [[0, 0, 0, 1, 14, 15, 15, 0]]


def test_binding_refuses_tensors_of_the_cpu():
    from paper_2609_16915_gb300 import clear
    c = clear.Clear.__new__(clear.Clear)
    c._h, c.device = None, 0
    with pytest.raises(ValueError):
        c.norm(torch.ones(2, 4), torch.ones(4), torch.ones(2, 4, dtype=torch.int8), torch.ones(2))
    with pytest.raises(ValueError):
        c.linear(torch.ones(2, 4, dtype=torch.int8), torch.ones(2), torch.ones(8), torch.ones(8), torch.ones(2, 8))
