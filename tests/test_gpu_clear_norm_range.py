"""The norm over the whole range of single precision: rows that have no norm say so, rows whose
squares leave the range have theirs."""

import math

import pytest
import torch

from tests import clear_util as U
from tests.test_gpu_clear import FLOATS, check_norm, lib, run_norm  # noqa: F401  (lib: the fixture)

pytestmark = pytest.mark.gpu

# an eighth of a warp's lanes, a warp, and blocks with 2, 8 and 32 elements a thread; odd ones singly; beyond a block's registers
WIDTHS = [1, 7, 96, 255, 768, 1021, 4096, 8200, 16384, 40961]


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("width", WIDTHS)
def test_infinity_under_a_gamma_of_zero(lib, dtype, width):
    x, gamma = U.rand(1, 5, width), 1 + 0.2 * U.rand(2, width)
    last = width - 1
    gamma[last] = 0
    x[1, last] = math.inf
    x[2, last] = -math.inf
    x[3, last] = math.nan
    x = x.to(dtype)
    q, scale, total = run_norm(lib, x, None, gamma, 1e-6)
    assert torch.isnan(scale[1:4]).all()
    check_norm(x[[0, 4]], None, gamma, 1e-6, (q[[0, 4]], scale[[0, 4]], total[[0, 4]]))
    # the infinity in the residual
    r = x.clone()
    scale = run_norm(lib, torch.ones_like(x), r, gamma, 1e-6, alias=True)[1]
    assert torch.isnan(scale[1:4]).all() and torch.isfinite(scale[[0, 4]]).all()


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_gamma_without_a_number(lib, width, bad):
    gamma = torch.ones(width)
    gamma[width // 2] = bad
    assert torch.isnan(run_norm(lib, 1 + U.rand(1, 3, width).abs(), None, gamma, 1e-6)[1]).all()


def test_sum_beyond_single_precision(lib):
    x = torch.full((2, 64), 3e38)
    x[1] = 1
    scale = run_norm(lib, x, x.clone(), torch.ones(64), 1e-6)[1]
    assert torch.isnan(scale[0]) and torch.isfinite(scale[1])
