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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("width", WIDTHS)
def test_squares_beyond_single_precision(lib, dtype, width):
    """Rows from 2^57 to 2^121: their sums of squares pass 2^114 to 2^255; one large value among small ones; and rows
    far below, which have the same norm without eps."""
    powers = [57, 60, 63, 64, 80, 100, 121]
    x = torch.cat([U.rand(1, 1, width) * 2.0 ** p for p in powers] + [U.rand(2, 3, width)])
    x[len(powers), 0] = 1e30
    x[len(powers) + 1, -1] = -2e25
    gamma = 1 + 0.2 * U.rand(3, width)
    x = x.to(dtype)
    check_norm(x, None, gamma, 1e-6, run_norm(lib, x, None, gamma, 1e-6))
    r = (x.float() * 0.5).to(dtype)
    check_norm(x, r, gamma, 1e-6, run_norm(lib, x, r, gamma, 1e-6, alias=True))
    low = torch.cat([U.rand(4, 1, width) * 2.0 ** -p for p in (40, 52, 56, 63, 75, 100, 115)]).to(dtype)
    check_norm(low, None, gamma, 0.0, run_norm(lib, low, None, gamma, 0.0))
    check_norm(low, None, gamma, 1e-38, run_norm(lib, low, None, gamma, 1e-38))
