"""Trees whose root is no token: verification keeps nothing of them and says so."""

import pytest
import torch

from tests.test_gpu_clear import FLOATS, lib  # noqa: F401  (lib: the fixture)
from tests.test_gpu_clear_draft import drafted, reported, run_verify
from tests.test_gpu_clear_draft_layer import DIM, KV, drafted_state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("batch,nodes,vocab", [(5, 1, 40), (5, 9, 300), (5, 40, 20011), (700, 3, 64)])
def test_verify_roots_without_a_token(lib, drawn, dtype, batch, nodes, vocab):
    """Such a sequence keeps nothing and has no next token; the others are as they were."""
    target, draft, tokens, parents, uniform = drafted(vocab, batch, nodes, vocab, dtype, drawn)
    tokens[:, 0] = torch.arange(batch, dtype=torch.int32) % vocab
    good = run_verify(lib, target, draft, tokens, parents, uniform)
    lib.sync_status()
    bad = tokens.clone()
    none = {0: -1, 2: vocab, 3: 1 << 30, batch - 1: -(1 << 31)}
    for b, x in none.items():
        bad[b, 0] = x
    path, count, following = run_verify(lib, target, draft, bad, parents, uniform)
    reported(lib)
    for b in range(batch):
        if b in none:
            assert bool((path[b] == -1).all()) and int(count[b]) == 0 and int(following[b]) == -1
        else:
            assert torch.equal(path[b], good[0][b]) and count[b] == good[1][b] and following[b] == good[2][b]


@pytest.mark.parametrize("root", [-1, 300, 1 << 30])
def test_a_drafted_step_from_a_root_without_a_token(root):
    """The sequence stays where it was, and its next step begins the same way; the other one goes on."""
    L, layer, embedding, head = drafted_state()
    up = torch.tensor([[-1, 0, 0, 1]] * 2, dtype=torch.int32, device="cuda")
    cache = L.Cache(2, 64, KV, DIM, page=16)
    x = embedding[torch.arange(40).reshape(2, 20).cuda()]
    layer.before_table(x, torch.zeros_like(x), cache)
    trees = torch.tensor([[7, 2, 3, 4], [root, 2, 3, 4]], dtype=torch.int32, device="cuda")
    uniform = torch.full((2, 4), 0.5, device="cuda")
    path, count, following, _ = L.drafted_step(layer, head, embedding, cache, trees, up, uniform)
    with pytest.raises(RuntimeError, match="rosetta_clear_sync_status failed"):
        layer.lib.sync_status()
    assert path[1].tolist() == [-1] * 4 and int(count[1]) == 0 and int(following[1]) == -1
    assert int(count[0]) >= 1 and 0 <= int(following[0]) < 300
    assert cache.lengths.tolist() == [20 + int(count[0]), 20]
    trees[:, 0] = following
    path, count, following, _ = L.drafted_step(layer, head, embedding, cache, trees, up, uniform)
    with pytest.raises(RuntimeError, match="rosetta_clear_sync_status failed"):
        layer.lib.sync_status()
    assert int(count[1]) == 0 and int(following[1]) == -1 and int(cache.lengths[1]) == 20
    layer.lib.sync_status()


def test_an_embedding_without_the_heads_tokens_is_refused():
    L, layer, embedding, head = drafted_state()
    up = torch.tensor([[-1, 0]], dtype=torch.int32, device="cuda")
    cache = L.Cache(1, 16, KV, DIM, page=16)
    with pytest.raises(ValueError, match="embedding"):
        L.drafted_step(layer, head, embedding[:299], cache, torch.ones_like(up), up, torch.zeros(1, 2, device="cuda"))
    assert cache.lengths.tolist() == [0] and cache.room == 16
    # one with more rows than the head has tokens is a table with padding
    more = torch.cat([embedding, embedding[:5]])
    out = [L.drafted_step(layer, head, e, L.Cache(1, 16, KV, DIM, page=16), torch.ones_like(up), up, torch.zeros(1, 2, device="cuda"))
           for e in (embedding, more)]
    layer.lib.sync_status()
    assert all(torch.equal(x, y) for x, y in zip(*out))
