"""Drafted tokens: argument checks that need no GPU, and the definitions that the GPU tests compare with,
against hand-computed values."""

import ctypes

import pytest
import torch

from tests import draft_util as D
from tests.test_clear_host import lib  # noqa: F401  (the fixture)


def test_null_handles_and_sizes_out_of_range(lib):
    three = (ctypes.c_int64 * 3)(64, 64, 64)
    cache = (None, None, three, None, None, 1, 16, None, 1)
    assert lib.rosetta_clear_tree_mask(None, None, 1, 0, 1, None, three, None) == -1
    assert lib.rosetta_clear_tree_attention(None, 0, None, three, 0, 0, 1, 1, 64, *cache, None, None, three, 1.0, None, three, None) == -1
    assert lib.rosetta_clear_verify(None, 0, None, three, None, None, None, 1, None, 1, None, 1, 0, 1, 1, None, 1, None, None, None) == -1
    assert lib.rosetta_clear_cache_keep(None, 0, 1, 1, 64, *cache, None, None, 1, None, None) == -1
    assert lib.rosetta_clear_cache_read(None, 0, 0, 1, 1, 64, *cache, None, None, None, three, None, three, None) == -1


def test_reference_mask_by_hand():
    """0 - 1 - 3 and 0 - 2, and a root of its own."""
    seen = D.ancestors(torch.tensor([[-1, 0, 0, 1, -1]]))
    assert seen[0].int().tolist() == [[1, 0, 0, 0, 0], [1, 1, 0, 0, 0], [1, 0, 1, 0, 0], [1, 1, 0, 1, 0], [0, 0, 0, 0, 1]]
    assert D.words(seen).tolist() == [[[1], [3], [5], [11], [16]]]
    chain = D.ancestors(torch.arange(-1, 33)[None])
    assert D.words(chain)[0, [0, 31, 32, 33]].tolist() == [[1, 0], [-1, 0], [-1, 1], [-1, 3]]


def test_reference_attention_by_hand():
    """A context of one position and two drafted ones that do not see each other; equal scores."""
    k, v = torch.ones(1, 1, 4, 4, dtype=torch.int8), torch.zeros(1, 1, 4, 4, dtype=torch.int8)
    v[0, 0, :3, 0] = torch.tensor([10, 20, 40], dtype=torch.int8)
    one = torch.ones(1, 1)
    out, size = D.tree_attention(torch.ones(1, 2, 1, 4), k, v, one, one, torch.tensor([[0]]), [3], torch.eye(2).bool()[None], 1.0)
    assert out[0, :, 0, 0].tolist() == [15, 25] and torch.equal(out, size)
    # the first drafted position is before the beginning, the second sees nothing
    out, _ = D.tree_attention(torch.ones(1, 2, 1, 4), k, v, one, one, torch.tensor([[0]]), [1], torch.tensor([[[1, 1], [1, 0]]]).bool(), 1.0)
    assert out[0, :, 0, 0].tolist() == [10, 0]


def rows(*values):
    return torch.tensor(values, dtype=torch.float32)


@pytest.mark.parametrize("u,path,following", [
    # q(x) = 1/2 against p(x) = 1/4: accepted below a half
    ([0.0, 0.4375, 0.0], [0, 1], 0),
    # rejected; what is left is (1/8, 0, 1/8) of p - q = (1/8, -1/4, 1/8): the second child, token 2, has q = 1/4, Z = 1/4
    # and left 1/8: always accepted
    ([0.0, 0.5, 0.9375], [0, 2], 1),
])
def test_reference_verification_of_drawn_tokens_by_hand(u, path, following):
    target = rows([0.375, 0.25, 0.375], [1, 0, 0], [0, 1, 0])
    draft = rows([0.25, 0.5, 0.25], [1, 0, 0], [1, 0, 0])
    got = D.verify(target, draft, torch.tensor([0, 1, 2]), torch.tensor([-1, 0, 0]), torch.tensor(u))
    assert got == (path, len(path), following)


def test_reference_verification_leaves_what_the_draft_did_not_cover():
    target, draft = rows([0.375, 0.25, 0.375]), rows([0.25, 0.5, 0.25])
    both = (target.expand(3, 3), draft.expand(3, 3), torch.tensor([0, 1, 1]), torch.tensor([-1, 0, 0]))
    # token 1 twice: rejected, and with nothing left of it rejected for any number; then 1/16 + 1/16 of tokens 0 and 2
    assert D.verify(*both, torch.tensor([0.4375, 0.5, 0.0])) == ([0], 1, 0)
    assert D.verify(*both, torch.tensor([0.5, 0.5, 0.0])) == ([0], 1, 2)


def test_reference_verification_of_given_tokens_by_hand():
    target = rows([0.5, 0.25, 0.25], [0, 0, 1], [1, 0, 0])
    tree = (torch.tensor([0, 0, 1]), torch.tensor([-1, 0, 0]))
    assert D.verify(target, None, *tree, torch.tensor([0.0, 0.4375, 0.0])) == ([0, 1], 2, 2)
    # token 0 rejected: token 1 has a half of what is left
    assert D.verify(target, None, *tree, torch.tensor([0.0, 0.5, 0.4375])) == ([0, 2], 2, 0)
    assert D.verify(target, None, *tree, torch.tensor([0.9375, 0.5, 0.5])) == ([0], 1, 2)


def test_reference_keep_by_hand():
    """Pages of two rows: row 3 moves before row 1's place from a page of twice the scale."""
    cache, scale = torch.zeros(2, 1, 2, 4, dtype=torch.int8), torch.tensor([[1.0], [2.0]])
    cache[0, 0, 0], cache[0, 0, 1], cache[1, 0, 0], cache[1, 0, 1] = 100, 7, 50, 61
    c, s = D.keep(cache, scale, torch.tensor([[0, 1]]), [1], torch.tensor([[2, 0]]), [1])
    assert c[:, 0, :, 0].tolist() == [[50, 61], [50, 61]] and s.tolist() == [[2.0], [2.0]]
    c, s = D.keep(cache, scale, torch.tensor([[0, 1]]), [1], torch.tensor([[0, 2]]), [2])
    # row 1 stays in page 0 at its scale, row 3 becomes row 2
    assert c[:, 0, :, 0].tolist() == [[100, 7], [61, 61]] and s.tolist() == [[1.0], [2.0]]


def test_reference_read_by_hand():
    cache, scale = torch.arange(16, dtype=torch.int8).reshape(2, 1, 2, 4), torch.tensor([[0.5], [2.0]])
    out = D.read(cache, scale, torch.tensor([[1, 0]]), [-1], [3], torch.full((1, 5, 1, 4), 9.0))
    assert out[0, :, 0, 0].tolist() == [9, 16, 24, 0, 9]


class NoCalls:
    def __getattr__(self, name):
        def call(*args):
            raise AssertionError(f"{name} was called")
        return call


@pytest.fixture
def handle():
    from paper_2609_16915_gb300 import clear
    c = clear.Clear.__new__(clear.Clear)
    c._h, c.device, c._L = None, -1, NoCalls()     # (tensors of the CPU are on device -1)
    return c


def test_binding_refuses_other_shapes_and_types(handle):
    i32 = torch.int32
    parents, mask = torch.zeros(2, 40, dtype=i32), torch.zeros(2, 40, 2, dtype=i32)
    for bad in [dict(parents=parents.long()), dict(parents=parents[0]), dict(mask=mask[..., :1]), dict(mask=mask[:1]), dict(mask=mask.long()),
                dict(parents=parents.t().contiguous().t())]:
        with pytest.raises(ValueError):
            handle.tree_mask(**{**dict(parents=parents, mask=mask), **bad})
    p = torch.zeros(2, 3, 50)
    n = torch.zeros(2, 3, dtype=i32)
    base = dict(target=p, tokens=n, parents=n, uniform=n.float(), path=n, count=n[:, 0].contiguous(), next_token=n[:, 0].contiguous(), draft=p)
    for bad in [dict(target=p.double()), dict(draft=p.half()), dict(draft=p[:, :2]), dict(tokens=n.long()), dict(parents=n[:, :2]),
                dict(uniform=n), dict(path=n[:, :2]), dict(count=n), dict(next_token=n[:, 0].long().contiguous()), dict(target=p[0]),
                dict(path=n[:1].expand(2, 3))]:
        with pytest.raises(ValueError):
            handle.verify(**{**base, **bad})
    c, s = torch.zeros(4, 2, 16, 64, dtype=torch.int8), torch.ones(4, 2)
    table, one = torch.zeros(2, 2, dtype=i32), torch.zeros(2, dtype=i32)
    base = dict(k_cache=c, v_cache=c, k_scale=s, v_scale=s, page_table=table, first=one, path=n, count=one)
    for bad in [dict(k_cache=c.float()), dict(v_cache=c[:3]), dict(k_scale=s[:3]), dict(first=one.long()), dict(path=n.long()), dict(path=n[:1]),
                dict(count=one[:1]), dict(page_table=table[:1])]:
        with pytest.raises(ValueError):
            handle.cache_keep(**{**base, **bad})
    k = torch.zeros(2, 5, 2, 64)
    base = dict(k_cache=c, v_cache=c, k_scale=s, v_scale=s, page_table=table, first=one, lengths=one, k=k, v=k)
    for bad in [dict(k=k.double()), dict(v=k.half()), dict(v=k[:, :4]), dict(k=k[:, :, :1], v=k[:, :, :1]), dict(lengths=one.long()),
                dict(first=one[:1])]:
        with pytest.raises(ValueError):
            handle.cache_read(**{**base, **bad})
    q = torch.zeros(2, 40, 4, 64)
    base = dict(q=q, k_cache=c, v_cache=c, k_scale=s, v_scale=s, page_table=table, lengths=one, mask=mask, out=q)
    for bad in [dict(mask=mask[..., :1]), dict(mask=mask.long()), dict(mask=mask[:, :39]), dict(q=q[:, :, :3]), dict(out=q.half())]:
        with pytest.raises(ValueError):
            handle.tree_attention(**{**base, **bad})
