"""Drafted tokens through the layer: what is decided before anything reaches the GPU."""

import pytest
import torch

from paper_2609_16915_gb300 import clear_layer as L

VOCAB, WIDTH = 12, 8


class OneToken:
    """A head that always gives the token 3, on the CPU."""
    class packed:
        channels = VOCAB

    def __call__(self, y, residual=None):
        return torch.eye(VOCAB)[3].expand(*y.shape[:2], VOCAB)


@pytest.mark.parametrize("rows", [VOCAB, VOCAB + 5])
def test_trees_are_drawn_from_roots_without_a_token(rows):
    """Such a root stays as it is (the step over the tree reports it), and no row outside the embedding is asked for."""
    seen = []

    class Embedding(torch.Tensor):
        @classmethod
        def __torch_function__(cls, func, types, args=(), kwargs=None):
            if func is torch.Tensor.__getitem__:
                seen.append(torch.as_tensor(args[1]))
            return super().__torch_function__(func, types, args, kwargs or {})

    roots = torch.tensor([2, -1, VOCAB, rows, 1 << 30, -(1 << 31)], dtype=torch.int32)
    tokens, draft = L.draw_tree(OneToken(), torch.rand(rows, WIDTH).as_subclass(Embedding), roots, torch.tensor([-1, 0, 0, 1]))
    assert torch.equal(tokens[:, 0], roots) and bool((tokens[:, 1:] == 3).all())
    assert draft[:, :2, 3].tolist() == [[1.0, 1.0]] * 6 and not draft[:, 2:].any()
    assert seen and all(0 <= int(s.min()) and int(s.max()) < rows for s in seen)


def test_trees_are_not_drawn_from_an_embedding_without_the_heads_tokens():
    with pytest.raises(ValueError, match="embedding"):
        L.draw_tree(OneToken(), torch.rand(VOCAB - 1, WIDTH), torch.zeros(1, dtype=torch.int32), torch.tensor([-1, 0]))


class NoCalls:
    def __getattr__(self, name):
        def call(*args):
            raise AssertionError(f"{name} was called")
        return call


@pytest.fixture
def layer():
    from paper_2609_16915_gb300 import clear
    layer = L.Layer.__new__(L.Layer)
    layer.lib = clear.Clear.__new__(clear.Clear)
    layer.lib._h, layer.lib.device, layer.lib._L = None, -1, NoCalls()      # (tensors of the CPU are on device -1)
    return layer


def test_a_drafted_step_refuses_before_anything_moves(layer):
    b, nodes = 2, 5
    cache = L.Cache(b, 64, 2, 16, device="cpu")
    n, u = torch.zeros((b, nodes), dtype=torch.int32), torch.zeros(b, nodes)
    base = dict(cache=cache, tokens=n, parents=n, uniform=u, draft=torch.zeros(b, nodes, VOCAB))
    for bad in [dict(tokens=n.long()), dict(tokens=n[0]), dict(parents=n.long()), dict(parents=n[:, :4]), dict(uniform=u.double()),
                dict(uniform=u[:1]), dict(draft=torch.zeros(b, nodes, VOCAB).half()), dict(draft=torch.zeros(b, nodes, VOCAB - 1)),
                dict(draft=torch.zeros(b, nodes - 1, VOCAB)), dict(cache=L.Cache(b + 1, 64, 2, 16, device="cpu"))]:
        with pytest.raises(ValueError):
            L.drafted_step(layer, OneToken(), torch.rand(VOCAB, WIDTH), **{**base, **bad})
    assert cache.room == 64 and cache.lengths.tolist() == [0, 0]


def test_a_step_under_a_mask_that_does_not_fit_moves_nothing(layer):
    layer.heads, layer.kv_heads, layer.dim = 2, 1, 16
    for tokens, bad in [(5, torch.zeros(2, 5, 1)), (5, torch.zeros(2, 4, 1, dtype=torch.int32)), (5, torch.zeros(2, 5, 2, dtype=torch.int32)),
                        (33, torch.zeros(2, 33, 1, dtype=torch.int32)), (5, torch.zeros(1, 5, 1, dtype=torch.int32)), (5, torch.zeros(5, 1, dtype=torch.int32)),
                        (1025, torch.zeros(2, 1025, 33, dtype=torch.int32))]:
        cache = L.Cache(2, 2048, 1, 16, device="cpu")
        x = torch.zeros(2, tokens, 32, dtype=torch.bfloat16)
        with pytest.raises(ValueError):
            layer.step(x, torch.zeros_like(x), cache, bad)
        assert cache.room == 2048 and cache.lengths.tolist() == [0, 0]
