"""float16 tree attention holds its weights to 22 bits, whatever kernel takes the rows: the bound of single precision beside
the output's own rounding, which weights of 11 bits would pass (test_weights_of_11_bits_would_be_seen)."""

import pytest
import torch

from tests import clear_util as U
from tests import draft_util as D
from tests.test_gpu_clear import lib, make_cache  # noqa: F401  (lib: the fixture)
from tests.test_gpu_clear_draft import ints

CASES = [  # lens, new, page, heads, group, dim: rows a cached head are new * group
    ([300, 90], 5, 16, 3, 1, 64), ([200, 700], 4, 32, 2, 4, 128), ([180], 6, 16, 2, 2, 256),            # few rows
    ([150, 400], 17, 16, 2, 1, 64), ([260, 64], 12, 32, 2, 4, 128), ([700, 333], 32, 48, 2, 2, 96),     # 17 .. 64
    ([64, 900], 64, 16, 1, 1, 128),
    ([130, 290], 65, 16, 2, 1, 64), ([500, 222], 20, 32, 2, 4, 128), ([128, 1000], 128, 64, 1, 1, 96),  # 65 .. 128
    ([400, 129], 129, 16, 1, 1, 64), ([600], 75, 32, 2, 4, 128)]                                        # more


def state(lens, new, page, heads, group, dim):
    c, s, table = make_cache(new + dim, lens, page, heads, dim)
    q = U.rand(new, len(lens), new, heads * group, dim).half()
    seen = D.ancestors(D.random_tree(new + 1, len(lens), new))
    # scores of a deviation of about 2: a row's sum is of some ten terms, whose roundings do not cancel
    return q, c, s, table, seen, 1.6 * dim ** -0.5


def bound(want, size):
    """The output's rounding (and that below 2^-14, 2^-25); of sum p |v|: weights 2^-22, scores of up to 2^5 in single precision
    2^-19, cut-off terms of the tensor cores' sums 7e-9 for each of up to 1000 positions, together below 2^-16."""
    return 1.01 * U.UNIT[torch.float16] * want.abs() + 2.0 ** -16 * size + 2.0 ** -25


@pytest.mark.gpu
@pytest.mark.parametrize("case", CASES)
def test_float16_weights(lib, case):
    q, c, s, table, seen, scale = state(*case)
    out = torch.empty_like(q, device="cuda")
    lib.tree_attention(q.cuda(), *[t.cuda() for t in (*c, *s)], table.cuda(), ints(case[0]).cuda(), D.words(seen).cuda(), out, scale)
    lib.sync_status()
    want, size = D.tree_attention(q, *c, *s, table, case[0], seen, scale)
    err = (out.cpu().double() - want).abs()
    assert torch.all(err <= bound(want, size)), float((err / bound(want, size)).max())


@pytest.mark.gpu
@pytest.mark.parametrize("new,group", [(2, 4), (8, 4), (24, 4), (40, 4)])
def test_float16_weights_of_more_blocks_than_run_at_once(lib, new, group):
    """Whole sequences a block, the longest first."""
    lens = [new + 1 + (i * 53) % 170 for i in range(100)]
    q, c, s, table, seen, scale = state(lens, new, 16, 2, group, 64)
    out = torch.empty_like(q, device="cuda")
    lib.tree_attention(q.cuda(), *[t.cuda() for t in (*c, *s)], table.cuda(), ints(lens).cuda(), D.words(seen).cuda(), out, scale)
    lib.sync_status()
    want, size = D.tree_attention(q, *c, *s, table, lens, seen, scale)
    assert torch.all((out.cpu().double() - want).abs() <= bound(want, size))


@pytest.mark.parametrize("case", CASES)
def test_weights_of_11_bits_would_be_seen(case, monkeypatch):
    """On the CPU: the same definition with each weight rounded to float16 below the row's largest breaks the bound."""
    q, c, s, table, seen, scale = state(*case)
    want, size = D.tree_attention(q, *c, *s, table, case[0], seen, scale)
    softmax = torch.softmax

    def rounded(z, dim):
        p = torch.exp(z - z.amax(dim))
        return (p * 128).half().double() / (128 * p.sum(dim))

    monkeypatch.setattr(torch, "softmax", rounded)
    off, _ = D.tree_attention(q, *c, *s, table, case[0], seen, scale)
    monkeypatch.setattr(torch, "softmax", softmax)
    off = off.half().double()
    assert torch.any((off - want).abs() > bound(want, size))
    assert torch.all((want.half().double() - want).abs() <= bound(want, size))
