"""The layer's cache refuses tokens that it has no room for, before anything moves."""

import pytest
import torch

from paper_2609_16915_gb300 import clear_layer as L


def cache():
    return L.Cache(3, 40, 2, 64, page=16, device="cpu")        # three pages a sequence


def test_room_runs_out():
    c = cache()
    c.take(40)
    c.lengths += 40
    for _ in range(8):
        c.take(1)
        c.lengths += 1
    with pytest.raises(ValueError, match="48 positions"):
        c.take(1)
    with pytest.raises(ValueError):
        cache().take(49)
    cache().take(48)


def test_lengths_that_were_set():
    c = cache()
    c.take(48)
    c.lengths += 48
    c.lengths[0], c.lengths[1], c.lengths[2] = 5, 30, 0          # sequences cut short: 18 positions left
    c.take(18)
    c.lengths += 18
    with pytest.raises(ValueError):
        c.take(1)


def test_a_full_cache_stops_the_layer():
    """... before any operator is called (there is none here)."""
    layer = L.Layer.__new__(L.Layer)
    layer.heads, layer.kv_heads, layer.dim = 4, 2, 64
    c = cache()
    c.lengths += 48
    x = r = torch.zeros(3, 49, 8)
    with pytest.raises(ValueError):
        layer.before_table(x, r, c)
    assert c.lengths.tolist() == [48] * 3
