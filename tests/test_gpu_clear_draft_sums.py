"""Verification of given tokens over rows that add up to 64 and more, where a part of them was rejected."""

import pytest
import torch

from tests import draft_util as D
from tests.test_gpu_clear import lib  # noqa: F401  (the fixture)
from tests.test_gpu_clear_draft import ints, reported, run_verify

pytestmark = pytest.mark.gpu


def rows_of_one_child(vocab, values, rejected):
    """A root whose row has `values` at given tokens, and one child of token `rejected` that is not accepted."""
    target = torch.zeros(1, 2, vocab)
    for at, v in values.items():
        target[0, 0, at] = v
    target[0, 1, 0] = 1
    return target, None, ints([[0, rejected]]), ints([[-1, 0]]), torch.tensor([[0.5, 0.9375]])


@pytest.mark.parametrize("vocab", [2000, 40007])
@pytest.mark.parametrize("spread", [1, 97])
@pytest.mark.parametrize("most,rejected", [(128, 0.5), (64, 0.5), (64, 0.75), (63, 0.5), (62, 0.75)])
def test_verify_given_tokens_of_rows_that_add_up_to_too_much(lib, vocab, spread, most, rejected):
    """`most` ones and the rejected token beside them, together in one run of the vocabulary or far apart: from 64 on the row, the
    rejected token in it, has no next token."""
    at = (7 + spread * torch.arange(most + 1) * (vocab // 2000 if spread > 1 else 1)) % vocab
    values = {int(x): 1.0 for x in at[1:]}
    assert len(values) == most and int(at[0]) not in values
    values[int(at[0])] = rejected
    args = rows_of_one_child(vocab, values, int(at[0]))
    total = most + rejected
    path, count, following = run_verify(lib, *args)
    assert path.tolist() == [[0, -1]] and int(count[0]) == 1
    if total >= 64:
        assert int(following[0]) == -1
        reported(lib)
    else:
        lib.sync_status()
        want = D.verify(args[0][0], None, *[x[0] for x in args[2:]])
        assert (path[0, :1].tolist(), int(count[0]), int(following[0])) == want
