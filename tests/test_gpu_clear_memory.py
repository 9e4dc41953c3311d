"""The workspace of the layer in the clear where device memory is short."""

import pytest
import torch

from tests.test_gpu_memory_short import MIB, _Left

pytestmark = pytest.mark.gpu


def test_workspace_that_cannot_double():
    """Where memory for twice the last workspace is not there, what the call needs is enough."""
    from paper_2609_16915_gb300 import clear
    tokens, inner = 32768, 2048                  # 128 MiB as f16
    q = torch.ones((tokens, inner), dtype=torch.int8, device="cuda")
    scale, w_scale = torch.ones(tokens, device="cuda"), torch.ones(64, device="cuda")
    out = torch.empty((tokens, 64), device="cuda")
    lib = clear.Clear(workspace_bytes=100 * MIB)
    w = lib.pack_weights(torch.ones((64, inner), dtype=torch.int8, device="cuda"))
    lib.linear(q[:64], scale[:64], w, w_scale, out[:64])
    lib.sync_status()
    with _Left(160):
        lib.linear(q, scale, w, w_scale, out)    # (200 MiB are not there)
        lib.sync_status()
    assert bool((out == inner).all())
    lib.close()
