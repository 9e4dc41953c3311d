"""Drafted tokens through the layer: under a tree's mask, and the whole step with verification and what the cache keeps."""

import pytest
import torch

from tests import clear_util as U
from tests import draft_util as D
from tests.test_gpu_clear_layer import DIM, HEADS, KV, WIDTH, make_layer, tokens

pytestmark = pytest.mark.gpu


def test_layer_under_a_mask_against_64_bits():
    """As for causal tokens, the 8-bit rounding aside: behind a context of 20 tokens, 25 that see their ancestors."""
    L, weights, layer, _ = make_layer(6)
    x, r = tokens(2, 45, 11)
    parents = D.random_tree(3, 2, 25)
    mask = torch.empty(2, 25, 1, dtype=torch.int32, device="cuda")
    layer.lib.tree_mask(parents.cuda(), mask)
    cache = L.Cache(2, 45, KV, DIM)
    layer.before_table(x[:, :20], r[:, :20].clone(), cache)
    q, s = layer.before_table(x[:, 20:], r[:, 20:].contiguous(), cache, mask)
    layer.lib.sync_status()
    w = {k: v.double().cpu() for k, v in weights.items()}

    def norm(v):
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + L.EPS)

    h = x.double().cpu() + r.double().cpu()
    qkv = (norm(h) @ w["qkv"].T).reshape(2, 45, HEADS + 2 * KV, DIM)
    hidden = torch.ones(2, 45, 45).triu(1).bool()
    hidden[:, 20:, 20:] = ~D.ancestors(parents)
    out = torch.zeros(2, 45, HEADS, DIM, dtype=torch.float64)
    for b in range(2):
        for i in range(HEADS):
            k, v = qkv[b, :, HEADS + i // 2], qkv[b, :, HEADS + KV + i // 2]
            out[b, :, i] = torch.softmax((qkv[b, :, i] @ k.T * DIM ** -0.5).masked_fill(hidden[b], -torch.inf), 1) @ v
    h = h + norm(out.reshape(2, 45, -1)) @ w["o"].T
    want = norm(h)[:, 20:].reshape(50, WIDTH)
    got = q.cpu().double() * s.cpu().double()[:, None]
    # 8-bit activations, weights, keys and values of 1 / 127 of their largest: a few per cent of the rms
    assert float((got - want).norm() / want.norm()) < 0.06


def drafted_state(vocab=300):
    L, _, layer, _ = make_layer(6)
    embedding = U.rand(41, vocab, WIDTH).to(torch.bfloat16).cuda()
    return L, layer, embedding, L.Head(0.3 * embedding.float(), layer.lib)


def test_drafted_step_is_its_parts():
    """Path, count and next token follow from the probabilities, and the cache from the path."""
    L, layer, embedding, head = drafted_state()
    batch, nodes, lib = 3, 40, layer.lib
    up = D.random_tree(7, 1, nodes)[0].cuda()
    trees, draft = L.draw_tree(head, embedding, torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda"), up,
                               torch.Generator(device="cuda").manual_seed(5))
    parents = up.expand(batch, nodes)
    uniform = torch.rand((batch, nodes), generator=torch.Generator().manual_seed(2)).cuda()
    caches = [L.Cache(batch, 100, KV, DIM) for _ in range(2)]
    x = embedding[torch.arange(batch * 33).reshape(batch, 33).cuda() % 300]
    for c in caches:
        layer.before_table(x, torch.zeros_like(x), c)
        c.lengths[1] = 20
    path, count, following, code = L.drafted_step(layer, head, embedding, caches[0], trees, parents, uniform, draft)
    lib.sync_status()
    c = caches[1]
    mask = torch.empty(batch, nodes, 2, dtype=torch.int32, device="cuda")
    lib.tree_mask(parents, mask)
    xs = embedding[trees.long()]
    residual = torch.zeros_like(xs)
    y, again = layer.step(xs, residual, c, mask)
    target = head(y, residual)
    lib.sync_status()
    assert torch.equal(code, again)
    for b in range(batch):
        want = D.verify(target[b].cpu(), draft[b].cpu(), trees[b].cpu(), up.cpu(), uniform[b].cpu())
        assert (path[b, :want[1]].tolist(), int(count[b]), int(following[b])) == want
    first = (c.lengths - nodes).tolist()
    assert first == [33, 20, 33] and caches[0].lengths.tolist() == [f + n for f, n in zip(first, count.tolist())]
    for i in range(2):
        held, scale = D.keep(c.tensors()[i].cpu(), c.tensors()[i + 2].cpu(), c.pages.cpu(), first, path.cpu(), count.tolist())
        assert torch.equal(caches[0].tensors()[i].cpu(), held) and torch.equal(caches[0].tensors()[i + 2].cpu(), scale)


def test_drafted_steps_and_single_tokens_agree():
    """After three drafted steps the layer sees what it would after the accepted tokens one by one, within the cache's rounding."""
    L, layer, embedding, head = drafted_state()
    nodes = 6
    up = torch.tensor([-1, 0, 0, 1, 1, 2], dtype=torch.int32, device="cuda")
    cache, last, accepted = L.Cache(1, 96, KV, DIM, page=16), torch.tensor([4], dtype=torch.int32, device="cuda"), []
    g = torch.Generator(device="cuda").manual_seed(3)
    for _ in range(3):
        trees, draft = L.draw_tree(head, embedding, last, up, g)
        uniform = torch.rand((1, nodes), device="cuda", generator=g)
        path, count, last, _ = L.drafted_step(layer, head, embedding, cache, trees, up[None], uniform, draft)
        accepted += trees[0, path[0, :int(count[0])].long()].tolist()
    assert int(cache.lengths[0]) == len(accepted) and len(accepted) >= 3
    single = L.Cache(1, 96, KV, DIM, page=16)
    for t in accepted:
        x = embedding[torch.tensor([[t]], device="cuda")]
        layer.before_table(x, torch.zeros_like(x), single)
    outs = []
    for c in (cache, single):
        x = embedding[last.long()][None]
        q, s = layer.before_table(x, torch.zeros_like(x), c)
        outs.append(q.float() * s[:, None])
    layer.lib.sync_status()
    assert float((outs[0] - outs[1]).norm() / outs[1].norm()) < 0.06


def test_nodes_without_a_token_take_no_part():
    """Padding (no parent, any token) is left out silently; a child whose token is none is left out and reported."""
    L, layer, embedding, head = drafted_state()
    up = torch.tensor([[-1, 0, 0, -1]], dtype=torch.int32, device="cuda")
    uniform = torch.full((1, 4), 0.5, device="cuda")
    for lone, bad in ((300, False), (-7, False), (1 << 30, False), (5, True)):
        cache = L.Cache(1, 16, KV, DIM, page=16)
        trees = torch.tensor([[1, -1 if bad else 2, 300 if bad else 3, lone]], dtype=torch.int32, device="cuda")
        path, count, following, _ = L.drafted_step(layer, head, embedding, cache, trees, up, uniform)
        if bad:
            with pytest.raises(RuntimeError, match="rosetta_clear_sync_status failed"):
                layer.lib.sync_status()
            assert int(count[0]) == 1
        layer.lib.sync_status()
        assert 3 not in path[0].tolist() and 0 <= int(following[0]) < 300
        assert int(cache.lengths[0]) == int(count[0])


def test_a_full_cache_stops_a_drafted_step():
    L, layer, embedding, head = drafted_state()
    cache = L.Cache(1, 16, KV, DIM, page=16)
    chain = torch.arange(-1, 16, dtype=torch.int32, device="cuda")[None]
    with pytest.raises(ValueError, match="16 positions"):
        L.drafted_step(layer, head, embedding, cache, torch.zeros_like(chain), chain, torch.zeros(1, 17, device="cuda"))
    assert cache.lengths.tolist() == [0]


def test_the_command_drafts(capsys):
    from paper_2609_16915_gb300 import clear_layer
    clear_layer.main()
    assert "drafted: 8 trees of 9 nodes" in capsys.readouterr().out
