"""The append's 8-bit values of numbers so small that their scale is rounded in a few bits."""

import numpy as np
import pytest
import torch

from tests.test_gpu_clear import lib  # noqa: F401  (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("most", [100, 150, 189, 190, 191, 250, 317, 1000, 1 << 14])
@pytest.mark.parametrize("dim,off", [(64, 0), (64, 1), (20, 0)])
def test_append_of_the_smallest_numbers(lib, most, dim, off):
    """Multiples of 2^-149: max / 127 has few bits or none, and quotients reach 190; bytes stay within [-127, 127]."""
    units = np.arange(-16 * dim // 2, 16 * dim // 2).reshape(1, 16, 1, dim) % (2 * most + 1) - most
    x = torch.from_numpy(units.astype(np.float64) * 2.0 ** -149).float()
    wide = torch.zeros((1, 16, 1, dim + 1))
    wide[..., off:off + dim] = x
    cache = [torch.zeros((1, 1, 16, dim), dtype=torch.int8, device="cuda") for _ in range(2)]
    scale = [torch.zeros((1, 1), device="cuda") for _ in range(2)]
    table, first = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    k = (wide.cuda() if off or dim == 20 else x.cuda())[..., off:off + dim]
    lib.cache_append(k, k, *cache, *scale, table, first)
    lib.sync_status()
    top = int(np.abs(units).max())
    unit = int(np.rint(top / 127))               # (no tie: 127 is odd, halves of it are not reached)
    want = np.clip(np.rint(units / unit), -127, 127) if unit else np.clip(units * 0, -127, 127)
    for c, s in zip(cache, scale):
        assert float(s) == unit * 2.0 ** -149
        assert np.array_equal(c.cpu().numpy().reshape(units.shape), want.astype(np.int8))
