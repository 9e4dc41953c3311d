"""Drafted tokens (tree_mask, tree_attention, verify, cache_keep, cache_read) against their definitions.

Whole numbers and bytes have to be equal; floats stay within bounds that follow from their
roundings, stated at each check."""

import math

import pytest
import torch

from tests import clear_util as U
from tests import draft_util as D
from tests.test_gpu_clear import FLOATS, lib, make_cache  # noqa: F401  (lib: the fixture)

pytestmark = pytest.mark.gpu


def ints(values):
    return torch.tensor(values, dtype=torch.int32)


def refused(call, **args):
    from paper_2609_16915_gb300 import RosettaError
    with pytest.raises(RosettaError) as e:
        call(**args)
    assert e.value.status == -1


def reported(lib):
    refused(lib.sync_status)
    lib.sync_status()       # once


# ------------------------------------------------------------------ the tree's mask


@pytest.mark.parametrize("batch,nodes", [(1, 1), (2, 2), (3, 31), (4, 32), (4, 33), (2, 64), (3, 257), (2, 1024), (300, 17)])
def test_tree_mask(lib, batch, nodes):
    parents = D.random_tree(nodes, batch, nodes)
    mask = torch.full((batch, nodes, -(-nodes // 32)), 77, dtype=torch.int32, device="cuda")
    assert lib.tree_mask(parents.cuda(), mask) is mask
    lib.sync_status()
    assert torch.equal(mask.cpu(), D.words(D.ancestors(parents)))


def test_tree_mask_of_chains_shared_trees_and_wider_rows(lib):
    chain = torch.arange(-1, 1023, dtype=torch.int32)[None]
    mask = torch.empty((1, 1024, 32), dtype=torch.int32, device="cuda")
    lib.tree_mask(chain.cuda(), mask)
    want = D.words(torch.ones(1, 1024, 1024).tril().bool())
    assert torch.equal(mask.cpu(), want)
    parents = D.random_tree(5, 1, 40).cuda().expand(3, 40)
    wide = torch.full((3, 41, 5), 77, dtype=torch.int32, device="cuda")
    lib.tree_mask(parents, wide[:, :40, 2:4])
    lib.sync_status()
    assert torch.equal(wide[:, :40, 2:4].cpu(), D.words(D.ancestors(parents[:1].cpu())).expand(3, 40, 2))
    wide[:, :40, 2:4] = 77
    assert bool((wide == 77).all())


def test_tree_mask_reports_parents_out_of_range(lib):
    bad, good = ints([[-1, 0, 2, -2, 3, 9]]), ints([[-1, 0, -1, -1, 3, -1]])
    mask = torch.empty((1, 6, 1), dtype=torch.int32, device="cuda")
    lib.tree_mask(bad.cuda(), mask)
    reported(lib)
    assert torch.equal(mask.cpu(), D.words(D.ancestors(good)))


# ------------------------------------------------------------------ attention


def check_tree(lib, dtype, lens, new, page, heads, group, dim, seen=None, seed=5, scale=None, change=None):
    c, s, table = make_cache(seed, lens, page, heads, dim)
    if change:
        change(c, s, table)
    batch = len(lens)
    wide = U.rand(seed + 9, batch, new, heads * group + 1, dim).to(dtype)
    q = wide[:, :, :heads * group]
    if seen is None:
        seen = D.ancestors(D.random_tree(seed, batch, new))
    mask = D.words(seen).cuda().expand(batch, -1, -1)
    out = torch.full((batch, new, heads * group, dim), 9.0, dtype=dtype, device="cuda")
    lib.tree_attention(wide.cuda()[:, :, :heads * group], *[t.cuda() for t in (*c, *s)], table.cuda(), ints(lens).cuda(), mask, out, scale)
    lib.sync_status()
    want, size = D.tree_attention(q, *c, *s, table, lens, seen, dim ** -0.5 if scale is None else scale)
    # as causal attention: the output's rounding, and errors of the weights, rounded to 11 bits for the product with V (22
    # in single precision), scores in single precision
    weights = 2.0 ** -16 if dtype == torch.float32 else 2.0 ** -10
    err = (out.cpu().double() - want).abs()
    bound = 1.01 * U.UNIT[dtype] * want.abs() + weights * size + 1e-9
    assert torch.all(err <= bound), float((err - bound).max())
    return out


TREES = [  # lens, new, page, heads, group, dim
    ([1], 1, 16, 1, 1, 64), ([82], 5, 16, 12, 1, 64), ([9, 10, 15, 16, 17, 33], 9, 16, 2, 4, 128), ([100, 3000, 40, 517], 16, 32, 2, 8, 128),
    ([7, 64], 7, 16, 3, 2, 96), ([200, 130], 130, 64, 2, 3, 64), ([33, 300], 33, 128, 1, 8, 128), ([40, 77], 5, 24, 2, 2, 64),
    ([19, 50], 3, 1, 1, 7, 80), ([300], 20, 16, 1, 16, 256), ([129], 2, 16, 1, 128, 128), ([260, 44], 40, 32, 5, 1, 20),
    ([2000], 64, 16, 1, 4, 128), ([700, 260], 257, 32, 1, 4, 96), ([1300], 150, 128, 1, 2, 256), ([1100], 1024, 32, 1, 1, 64),
    ([600, 100, 350], 64, 48, 2, 4, 128), ([5000], 31, 64, 1, 2, 128), ([64, 128, 192], 64, 64, 1, 4, 128)]


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("lens,new,page,heads,group,dim", TREES)
def test_tree_attention(lib, dtype, lens, new, page, heads, group, dim):
    check_tree(lib, dtype, lens, new, page, heads, group, dim)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("batch,new,group", [(100, 20, 1), (100, 33, 2), (100, 70, 4), (128, 9, 8), (129, 9, 8), (300, 18, 1)])
def test_tree_attention_of_many_uneven_sequences(lib, dtype, batch, new, group):
    """More blocks than run at once, equal lengths, sequences shorter than their trees and empty ones among them."""
    lens = [new + (i * 37) % 90 if i % 7 else i % 5 for i in range(batch)]
    check_tree(lib, dtype, lens, new, 16, 2, group, 64)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("lens,new,page,heads,group,dim", [
    ([40, 3, 0, 70], 40, 16, 2, 4, 128),        # rows before the first position among them
    ([13, 12], 13, 16, 1, 1, 64), ([65, 31], 64, 32, 2, 2, 96), ([50, 20], 33, 24, 1, 3, 20), ([300, 260], 257, 64, 1, 1, 64)])
def test_tree_attention_under_any_bits(lib, dtype, lens, new, page, heads, group, dim):
    """Masks that are no trees: rows that see no drafted position, nodes that see later ones, one mask for all."""
    g = torch.Generator().manual_seed(new)
    seen = torch.rand((len(lens), new, new), generator=g) < 0.3
    seen[:, ::3] = False
    out = check_tree(lib, dtype, lens, new, page, heads, group, dim, seen=seen)
    for b, n in enumerate(lens):
        if n <= new:        # nothing before the drafted positions
            assert not out[b, ::3].any()
    check_tree(lib, dtype, lens, new, page, heads, group, dim, seen=seen[:1])


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("new,group", [(4, 1), (20, 2), (70, 4)])
def test_tree_attention_scales(lib, dtype, new, group):
    for scale in (0.0, -0.05):
        check_tree(lib, dtype, [200, 90], new, 16, 2, group, 128, scale=scale)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("new,group", [(1, 2), (9, 2), (16, 4), (32, 4), (40, 4)])
@pytest.mark.parametrize("pages_each", [40, 5000, 70000])
def test_tree_attention_under_long_lists(lib, dtype, new, group, pages_each):
    """Lists with room for many more positions than there are: what a cache of a long context gives."""
    lens, page, heads, dim = [new + 200, new + 3, new + 1], 16, 2, 64
    c, s, table = make_cache(3, lens, page, heads, dim)
    wide = torch.full((3, pages_each), 1 << 30, dtype=torch.int32)
    wide[:, :table.shape[1]] = table
    q, seen = U.rand(4, 3, new, heads * group, dim).to(dtype), D.ancestors(D.random_tree(1, 3, new))
    out = torch.empty_like(q, device="cuda")
    lib.tree_attention(q.cuda(), *[t.cuda() for t in (*c, *s)], wide.cuda(), ints(lens).cuda(), D.words(seen).cuda(), out)
    lib.sync_status()
    want, size = D.tree_attention(q, *c, *s, table, lens, seen, dim ** -0.5)
    weights = 2.0 ** -16 if dtype == torch.float32 else 2.0 ** -10
    assert torch.all((out.cpu().double() - want).abs() <= 1.01 * U.UNIT[dtype] * want.abs() + weights * size + 1e-9)


@pytest.mark.parametrize("dtype,context", [(torch.float32, 1 << 16), (torch.float32, 1 << 18), (torch.float16, 1 << 18), (torch.bfloat16, 1 << 18)])
@pytest.mark.parametrize("new,group", [(2, 4), (8, 4), (24, 4), (48, 4)])
def test_tree_attention_of_long_contexts(lib, dtype, context, new, group):
    """Page lists that repeat 2048 positions, values of one sign: what sums lose as they grow would show.  Behind them a chain of
    drafted positions; bounds as for causal attention of such contexts."""
    batch, pages, page, dim = 40, 33, 64, 128
    kc, vc = U.int8(5, pages, 1, page, dim), U.int8(6, pages, 1, page, dim, lo=1)
    ks, vs = torch.rand(pages, 1, generator=torch.Generator().manual_seed(7)) / 60, torch.rand(pages, 1, generator=torch.Generator().manual_seed(8)) / 60
    q = U.rand(9, 1, new, group, dim).to(dtype)
    each = context // page
    table = torch.cat([(torch.arange(each) * 7 % 32), torch.tensor([32])]).to(torch.int32)     # the drafted ones in page 32
    mask = D.words(torch.ones(1, new, new).tril().bool()).cuda().expand(batch, -1, -1)
    out = torch.empty((batch, new, group, dim), dtype=dtype, device="cuda")
    lib.tree_attention(q.cuda().expand(batch, -1, -1, -1).contiguous(), kc.cuda(), vc.cuda(), ks.cuda(), vs.cuda(),
                       table.cuda().expand(batch, -1).contiguous(), torch.full((batch,), context + new, dtype=torch.int32, device="cuda"), mask, out)
    lib.sync_status()
    # the context's positions `context / 2048` times each: once, with that added to their scores' exponent
    k = (kc[:32, 0].double() * ks[:32, :, None].double()).flatten(0, 1)
    v = (vc[:32, 0].double() * vs[:32, :, None].double()).flatten(0, 1)
    kd, vd = kc[32, 0, :new].double() * ks[32].double(), vc[32, 0, :new].double() * vs[32].double()
    for t in range(new):
        for h in range(group):
            z = torch.cat([k @ q[0, t, h].double() * dim ** -0.5 + math.log(context / 2048), kd[:t + 1] @ q[0, t, h].double() * dim ** -0.5])
            p = torch.softmax(z, 0)
            want = p @ torch.cat([v, vd[:t + 1]])       # (all values positive: the sum of p |v| too)
            bound = 2.0 ** -18 * want if dtype == torch.float32 else (U.UNIT[dtype] + 2.0 ** -10) * want
            assert torch.all((out[:, t, h].cpu().double() - want).abs() <= bound)


@pytest.mark.parametrize("new,group", [(6, 2), (40, 2)])
@pytest.mark.parametrize("dim", [64, 128, 20])
def test_tree_attention_never_reads_what_is_masked(lib, new, group, dim):
    """The rows behind a sequence's end, other pages, and bits from `tokens` on change nothing."""
    lens, page, heads = [40, 57], 16, 2
    c, s, table = make_cache(3, lens, page, heads, dim, spare=3)
    q = U.rand(4, 2, new, heads * group, dim).to(torch.float16)
    mask = D.words(D.ancestors(D.random_tree(1, 2, new)))
    outs = []
    for poison in (False, True):
        if poison:
            used = {int(p) for b in range(2) for p in table[b, :-(-lens[b] // page)]}
            for p in range(c[0].shape[0]):
                if p not in used:
                    s[0][p], s[1][p] = math.nan, math.inf
                    c[0][p], c[1][p] = -128, 127
            for b in range(2):
                p = table[b, (lens[b] - 1) // page].long()
                c[0][p, :, lens[b] % page:], c[1][p, :, lens[b] % page:] = 127, -128
            table = table.clone()
            table[:, -3:] = 1 << 30
            mask = mask.clone()
            mask[..., -1] |= -(1 << new % 32)
        out = torch.empty_like(q, device="cuda")
        lib.tree_attention(q.cuda(), *[t.cuda() for t in (*c, *s)], table.cuda(), ints(lens).cuda(), mask.cuda(), out)
        lib.sync_status()
        outs.append(out.cpu())
    assert torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("dim", [64, 20])
@pytest.mark.parametrize("what", ["scale", "value scale"])
def test_pages_without_a_number_reach_the_rows_that_see_them(lib, dtype, dim, what):
    """Drafted positions 16 .. 31 of 48 lie in a page whose scale is a NaN: nodes that see none of them are untouched."""
    new, lens, page, heads, group = 48, [96], 16, 2, 2
    seen = torch.eye(new).bool()
    seen[40, 20] = seen[3, 31] = seen[20, 3] = True
    c, s, table = make_cache(7, lens, page, heads, dim)
    q = U.rand(4, 1, new, heads * group, dim).to(dtype)
    want, size = D.tree_attention(q, *c, *s, table, lens, seen[None], dim ** -0.5)
    s[1 if what == "value scale" else 0][table[0, 4].long()] = math.nan
    out = torch.empty_like(q, device="cuda")
    lib.tree_attention(q.cuda(), *[t.cuda() for t in (*c, *s)], table.cuda(), ints(lens).cuda(), D.words(seen[None]).cuda(), out)
    lib.sync_status()
    touched = seen[:, 16:32].any(1)
    out = out.cpu().double()[0]
    assert bool(out[touched].isnan().all())
    weights = 2.0 ** -16 if dtype == torch.float32 else 2.0 ** -10
    assert torch.all((out - want[0]).abs()[~touched] <= (1.01 * U.UNIT[dtype] * want.abs() + weights * size + 1e-9)[0, ~touched])


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("new,group,dim,exponent", [(6, 2, 128, 14), (6, 2, 128, 60), (40, 2, 128, 27), (40, 2, 64, 60), (10, 2, 20, 27)])
def test_tree_attention_beside_scales_far_from_1(lib, dtype, new, group, dim, exponent):
    """A drafted page of huge values that only the last node sees takes nothing from the others' precision."""
    lens, page, heads = [64 + new], 16, 2
    c, s, table = make_cache(7, lens, page, heads, dim)
    s[1][table[0, 4].long()] *= 2.0 ** exponent
    seen = torch.zeros(new, new).bool()
    seen[-1] = True
    q = U.rand(4, 1, new, heads * group, dim).to(dtype)
    out = torch.empty_like(q, device="cuda")
    lib.tree_attention(q.cuda(), *[t.cuda() for t in (*c, *s)], table.cuda(), ints(lens).cuda(), D.words(seen[None]).cuda(), out)
    lib.sync_status()
    want, size = D.tree_attention(q, *c, *s, table, lens, seen[None], dim ** -0.5)
    weights = 2.0 ** -10 if dtype == torch.bfloat16 else 2.0 ** -16
    err = (out.cpu().double() - want).abs()[:, :-1]
    assert torch.all(err <= (1.01 * U.UNIT[dtype] * want.abs() + weights * size + (2.0 ** -25 if dtype == torch.float16 else 1e-42))[:, :-1])


@pytest.mark.parametrize("new,group", [(5, 2), (30, 2)])
@pytest.mark.parametrize("dim", [64, 20])
def test_tree_attention_pages_out_of_range_are_masked_and_reported(lib, new, group, dim):
    c, s, table = make_cache(3, [90], 16, 2, dim)
    q = U.rand(4, 1, new, 2 * group, dim)
    seen = torch.ones(new, new).tril().bool()
    bad = table.clone()
    bad[0, 2], bad[0, 5] = c[0].shape[0], -7
    out = torch.empty_like(q, device="cuda")
    dev = [t.cuda() for t in (*c, *s)]
    mask = D.words(seen[None]).cuda()
    lib.tree_attention(q.cuda(), *dev, bad.cuda(), ints([90]).cuda(), mask, out)
    reported(lib)
    k, v = ((x[table[0].long()].double() * y[table[0].long()].double()[:, :, None, None]).permute(1, 0, 2, 3).flatten(1, 2) for x, y in zip(c, s))
    for t in range(new):
        for h in range(2 * group):
            at = [p for p in range(90 - new + t + 1) if p // 16 not in (2, 5)]
            p = torch.softmax(k[h // group, at] @ q[0, t, h].double() * dim ** -0.5, 0)
            want, size = p @ v[h // group, at], p @ v[h // group, at].abs()
            assert torch.all((out[0, t, h].cpu().double() - want).abs() <= 2.0 ** -16 * size + 1e-9)
    # a length past the page list counts as the list's end
    lib.tree_attention(q.cuda(), *dev, table.cuda(), ints([5000]).cuda(), mask, out)
    reported(lib)
    want, size = D.tree_attention(q, *c, *s, table, [5000], seen[None], dim ** -0.5)
    assert torch.all((out.cpu().double() - want).abs() <= 2.0 ** -16 * size + 1e-9)


def test_tree_attention_refuses(lib):
    c, s, table = make_cache(3, [40, 30], 16, 2, 64)
    q = torch.randn(2, 5, 4, 64, device="cuda")
    mask = torch.ones(2, 5, 1, dtype=torch.int32, device="cuda")
    base = dict(q=q, k_cache=c[0].cuda(), v_cache=c[1].cuda(), k_scale=s[0].cuda(), v_scale=s[1].cuda(), page_table=table.cuda(),
                lengths=ints([40, 30]).cuda(), mask=mask, out=torch.empty_like(q))
    for bad in [dict(softmax_scale=math.inf), dict(out=q), dict(mask=base["out"].view(torch.int32)[:, :, 0, :1])]:
        refused(lib.tree_attention, **{**base, **bad})
    big = torch.zeros(2, 1025, 4, 64, device="cuda")
    refused(lib.tree_attention, **{**base, **dict(q=big, out=torch.empty_like(big), mask=torch.zeros(2, 1025, 33, dtype=torch.int32, device="cuda"))})
    refused(lib.tree_mask, parents=torch.zeros(1, 1025, dtype=torch.int32, device="cuda"), mask=torch.zeros(1, 1025, 33, dtype=torch.int32, device="cuda"))
    refused(lib.tree_mask, parents=mask[:, :, 0], mask=mask)
    refused(lib.tree_mask, parents=mask[:, :, 0], mask=torch.zeros(1, 5, 1, dtype=torch.int32, device="cuda").expand(2, 5, 1))
    lib.tree_mask(mask[:0, :, 0], mask[:0])
    lib.sync_status()


# ------------------------------------------------------------------ verification


def rows_of(seed, sharp, *shape):
    return torch.softmax(sharp * U.rand(seed, *shape), -1)


def drafted(seed, batch, nodes, vocab, dtype, drawn, sharp=2.0):
    """(target, draft or None, tokens, parents, uniform): tokens of the draft's own distribution, or the likeliest ones."""
    logits = sharp * U.rand(seed, batch, nodes, vocab)
    target = torch.softmax(logits, -1).to(dtype)
    near = torch.softmax(logits + 0.7 * U.rand(seed + 1, batch, nodes, vocab), -1)
    parents = D.random_tree(seed, batch, nodes)
    tokens = torch.zeros((batch, nodes), dtype=torch.int32)
    g = torch.Generator().manual_seed(seed + 2)
    seq = torch.arange(batch)
    for c in range(1, nodes):
        q = near[seq, parents[:, c].clamp_min(0).long()]
        tokens[:, c] = (torch.multinomial(q, 1, generator=g)[:, 0] if drawn else q.topk(min(vocab, 3), 1).indices[:, c % min(vocab, 3)]).to(torch.int32)
    uniform = torch.rand((batch, nodes), generator=g)
    return target, near.to(dtype) if drawn else None, tokens, parents, uniform


def run_verify(lib, target, draft, tokens, parents, uniform):
    b, n = target.shape[:2]
    path = torch.full((b, n), 55, dtype=torch.int32, device="cuda")
    count, following = torch.full((b,), 55, dtype=torch.int32, device="cuda"), torch.full((b,), 55, dtype=torch.int32, device="cuda")

    def cuda(t):
        return t if t is None or t.is_cuda else t.cuda()

    lib.verify(cuda(target), cuda(tokens), cuda(parents), cuda(uniform), path, count, following, draft=cuda(draft))
    return path.cpu(), count.cpu(), following.cpu()


def check_verify(lib, target, draft, tokens, parents, uniform):
    path, count, following = run_verify(lib, target, draft, tokens, parents, uniform)
    lib.sync_status()
    for b in range(target.shape[0]):
        want = D.verify(target[b].cpu(), None if draft is None else draft[b].cpu(), tokens[b], parents[b], uniform[b])
        n = want[1]
        assert path[b, :n].tolist() == want[0] and bool((path[b, n:] == -1).all()) and int(count[b]) == n and int(following[b]) == want[2], b
    return count


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("batch,nodes,vocab", [(1, 1, 1), (2, 2, 2), (3, 5, 31), (5, 7, 32), (4, 33, 33), (6, 20, 128), (3, 70, 129), (3, 12, 1000),
                                               (2, 9, 5003), (9, 4, 513)])
def test_verify(lib, drawn, dtype, batch, nodes, vocab):
    check_verify(lib, *drafted(vocab + nodes, batch, nodes, vocab, dtype, drawn))


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("vocab", [50257, 128256])
def test_verify_large_vocabularies(lib, drawn, dtype, vocab):
    check_verify(lib, *drafted(vocab, 2, 4, vocab, dtype, drawn, sharp=4.0))


@pytest.mark.parametrize("drawn", [True, False])
def test_verify_many_sequences_and_children(lib, drawn):
    """Roots of 40 children: many rejections before one is accepted."""
    batch, nodes, vocab = 200, 41, 60
    args = list(drafted(3, batch, nodes, vocab, torch.float32, drawn, sharp=1.0))
    args[3] = torch.cat([ints([[-1]]), torch.zeros((1, 40), dtype=torch.int32)], 1).expand(batch, nodes)
    if drawn:       # children of the root's row, some of them tokens that it hardly gives
        g = torch.Generator().manual_seed(9)
        args[2][:, 1:] = torch.multinomial(torch.rand(batch, vocab, generator=g), 40, replacement=True, generator=g).to(torch.int32)
    else:
        args[2][:, 1:] = torch.randint(0, vocab, (batch, 40), generator=torch.Generator().manual_seed(9), dtype=torch.int32)
    args[4] = 0.3 + 0.7 * args[4]
    check_verify(lib, *args)


def test_verify_a_tree_of_1024_nodes(lib):
    target, draft, tokens, parents, uniform = drafted(8, 2, 1024, 17, torch.float32, True)
    parents[0] = torch.arange(-1, 1023)     # a chain, accepted to its end
    uniform[0] = 0.0
    uniform[0, 0] = 0.999
    count = check_verify(lib, target, draft, tokens, parents, uniform)
    assert int(count[0]) == 1024


def test_verify_numbers_at_borders(lib):
    """Halves, quarters and eighths are exact everywhere: a number at a border is rejected, or the next token's."""
    target = torch.tensor([[[0.375, 0.25, 0.375], [1, 0, 0], [0, 1, 0]]])
    draft = torch.tensor([[[0.25, 0.5, 0.25], [1, 0, 0], [1, 0, 0]]])
    below = 0.5 - 2.0 ** -25
    for u1 in (0.0, below, 0.5, 1 - 2.0 ** -24):
        for u0 in (0.0, below, 0.5, 1 - 2.0 ** -24):
            for second in (1, 2):
                tokens, parents, u = ints([[0, 1, second]]), ints([[-1, 0, 0]]), torch.tensor([[u0, u1, 0.5]])
                check_verify(lib, target, draft, tokens, parents, u)
                check_verify(lib, target, None, tokens, parents, u)


def test_verify_numbers_out_of_range(lib):
    """Below 0 and NaN count as 0, from 1 on as just below 1."""
    target, _, tokens, parents, uniform = drafted(3, 4, 6, 40, torch.float32, False)
    for value, like in ((-1.0, 0.0), (math.nan, 0.0), (1.0, 1 - 2.0 ** -24), (7.0, 1 - 2.0 ** -24), (math.inf, 1 - 2.0 ** -24)):
        a = run_verify(lib, target, None, tokens, parents, torch.full_like(uniform, value))
        b = run_verify(lib, target, None, tokens, parents, torch.full_like(uniform, like))
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    lib.sync_status()


def test_verify_equal_rows_accept_everything(lib):
    """A draft that is the target is always accepted; a target without the drafted tokens never."""
    target, _, tokens, _, uniform = drafted(5, 3, 8, 300, torch.float32, True)
    chain = torch.arange(-1, 7, dtype=torch.int32).expand(3, 8)
    for b in range(3):
        for c in range(1, 8):
            tokens[b, c] = int(target[b, c - 1].argmax())
    assert check_verify(lib, target, target, tokens, chain, uniform).tolist() == [8, 8, 8]
    none = target.clone()
    none[:, 0] = 0
    none[torch.arange(3), 0, (tokens[:, 1].long() + 1) % 300] = 1
    assert check_verify(lib, none, target, tokens, chain, uniform).tolist() == [1, 1, 1]
    # nothing is left: the target's own row
    half = torch.zeros(1, 2, 4)
    half[0, 0] = torch.tensor([0.25, 0.25, 0.25, 0.25])
    more = torch.tensor([[[0.5, 0.5, 0.5, 0.5], [1, 0, 0, 0]]])
    check_verify(lib, half, more, ints([[0, 1]]), ints([[-1, 0]]), torch.tensor([[0.6, 0.75]]))
    check_verify(lib, torch.tensor([[[0.0, 1.0], [0.5, 0.5]]]), None, ints([[0, 0]]), ints([[-1, 0]]), torch.tensor([[0.3, 0.1]]))


@pytest.mark.parametrize("drawn", [True, False])
@pytest.mark.parametrize("children", [1, 3])
def test_verified_tokens_are_distributed_as_the_target(lib, drawn, children):
    """The token after the root over 60000 sequences, within five standard deviations of the target's row."""
    batch, vocab = 60000, 12
    p, q = rows_of(1, 1.5, vocab), rows_of(2, 1.0, vocab)
    g = torch.Generator().manual_seed(4)
    tokens = torch.zeros((batch, 1 + children), dtype=torch.int32)
    tokens[:, 1:] = (torch.multinomial(q.expand(batch, vocab), children, replacement=True, generator=g) if drawn
                     else q.topk(children).indices.expand(batch, children)).to(torch.int32)
    parents = torch.cat([ints([-1]), torch.zeros(children, dtype=torch.int32)]).expand(batch, -1)
    uniform = torch.rand((batch, 1 + children), generator=g)
    path, count, following = run_verify(lib, p.cuda().expand(batch, 1 + children, vocab), q.cuda().expand(batch, 1 + children, vocab) if drawn else None,
                                        tokens, parents, uniform)
    lib.sync_status()
    first = torch.where(count > 1, tokens[torch.arange(batch), path[:, 1].clamp_min(0).long()], following)
    share = torch.bincount(first.long(), minlength=vocab).double() / batch
    assert torch.all((share - p.double()).abs() <= 5 * torch.sqrt(p.double() * (1 - p.double()) / batch))


def test_verify_nodes_and_rows_that_are_none(lib):
    target, draft, tokens, parents, uniform = drafted(6, 6, 5, 50, torch.float32, True)
    good = run_verify(lib, target, draft, tokens, parents, uniform)
    lib.sync_status()
    bad_tokens, bad_parents, bad_target = tokens.clone(), parents.clone(), target.clone()
    bad_tokens[0, 1:], bad_tokens[1, 1:] = 50, -1
    bad_parents[2, 1:] = ints([1, 7, -2, 4])
    bad_target[3] = 0
    bad_target[4, :, 7] = math.nan
    got = run_verify(lib, bad_target, draft, bad_tokens, bad_parents, uniform)
    reported(lib)
    lone = torch.full_like(parents, -1)
    alone = run_verify(lib, target, draft, tokens, lone, uniform)
    lib.sync_status()
    for i in range(3):      # no nodes but the root
        assert torch.equal(torch.stack([x[i] for x in got[1:]]), torch.stack([x[i] for x in alone[1:]]))
    assert int(got[2][3]) == -1 and int(got[1][3]) == 1
    bad_target[4, :, 7] = 0
    zero = run_verify(lib, bad_target, draft, tokens, parents, uniform)
    for x, y, z in zip(got, zero, good):
        assert torch.equal(x[4], y[4]) and torch.equal(x[5], z[5])
    reported(lib)           # (the row of zeros)
    huge = torch.full((1, 2, 200), 2.0)
    assert int(run_verify(lib, huge, None, ints([[0, 0]]), ints([[-1, -1]]), torch.zeros(1, 2))[2][0]) == -1
    reported(lib)
    run_verify(lib, 1.5 * huge, None, ints([[0, 0]]), ints([[-1, -1]]), torch.zeros(1, 2))
    reported(lib)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("drawn", [True, False])
def test_verify_rows_of_wider_buffers(lib, dtype, drawn):
    """Rows at odd places, and paths in a wider buffer."""
    target, draft, tokens, parents, uniform = drafted(12, 3, 6, 333, dtype, drawn)
    want = run_verify(lib, target, draft, tokens, parents, uniform)
    for off in (0, 1, 3, 8):
        wide = [torch.full((3, 7, 360), math.nan, dtype=dtype, device="cuda") for _ in range(2)]
        for w, x in zip(wide, (target, draft)):
            if x is not None:
                w[:, :6, off:off + 333] = x.cuda()
        got = run_verify(lib, wide[0][:, :6, off:off + 333], wide[1][:, :6, off:off + 333] if drawn else None, tokens, parents, uniform)
        lib.sync_status()
        assert all(torch.equal(x, y) for x, y in zip(got, want))
    paths = torch.full((3, 9), 55, dtype=torch.int32, device="cuda")
    count, following = (torch.empty(3, dtype=torch.int32, device="cuda") for _ in range(2))
    lib.verify(target.cuda(), tokens.cuda(), parents.cuda(), uniform.cuda(), paths[:, 2:8], count, following,
               draft=None if draft is None else draft.cuda())
    lib.sync_status()
    assert torch.equal(paths[:, 2:8].cpu(), want[0]) and bool((paths[:, :2] == 55).all()) and bool((paths[:, 8:] == 55).all())


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("vocab", [333, 9001])
def test_verify_target_and_draft_rows_that_lie_differently(lib, dtype, vocab):
    """Target rows on 16 bytes, draft rows not, and the other way round."""
    args = drafted(14, 4, 8, vocab, dtype, True, sharp=1.0)
    want = check_verify(lib, *args)
    assert int(want.max()) > 1
    pitch = (vocab + 31) // 16 * 16
    for off_p, off_q in ((0, 1), (3, 0), (2, 5)):
        wide = [torch.full((4, 8, pitch), math.nan, dtype=dtype, device="cuda") for _ in range(2)]
        for w, x, off in zip(wide, args[:2], (off_p, off_q)):
            w[:, :, off:off + vocab] = x.cuda()
        check_verify(lib, wide[0][:, :, off_p:off_p + vocab], wide[1][:, :, off_q:off_q + vocab], *args[2:])


@pytest.mark.parametrize("batch", [1, 30, 60, 90, 170, 700])
def test_verify_clusters_of_every_size(lib, batch):
    """The CTAs of a sequence go by the batch: the same results whatever their number."""
    args = drafted(15, 10, 6, 16500, torch.float32, True, sharp=1.5)
    one = run_verify(lib, *[x[:1] for x in args])
    many = run_verify(lib, *[torch.cat([x] * (-(-batch // 10)))[:batch] for x in args])
    lib.sync_status()
    for b in range(10):
        want = D.verify(*[x[b] for x in args])
        for i in range(b, batch, 10):
            assert (many[0][i, :want[1]].tolist(), int(many[1][i]), int(many[2][i])) == want
    assert all(torch.equal(x, y[:1]) for x, y in zip(one, many))


def test_verify_beyond_32_bits(lib):
    """Rows whose places pass 2^32 elements."""
    nodes, vocab = 40, 120_000_000 // 1024
    target = torch.zeros((1025, nodes, vocab), dtype=torch.float16, device="cuda")
    target[1024, :, 5] = 0.5
    target[1024, :, vocab - 1] = 0.5
    tokens = torch.full((1025, nodes), vocab - 1, dtype=torch.int32)
    chain = torch.arange(-1, nodes - 1, dtype=torch.int32).expand(1025, nodes)
    assert 1024 * nodes * vocab > 1 << 32
    path, count, following = run_verify(lib, target, None, tokens, chain, torch.full((1025, nodes), 0.25))
    reported(lib)           # (the rows of zeros)
    assert int(count[1024]) == nodes and path[1024].tolist() == list(range(nodes)) and int(following[1024]) == 5
    assert int(count[3]) == 1 and int(following[3]) == -1


def test_verify_refuses(lib):
    p = torch.full((2, 3, 8), 0.125, device="cuda")
    n, u = torch.full((2, 3), -1, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, device="cuda")
    path, count, following = torch.empty_like(n), *(torch.empty(2, dtype=torch.int32, device="cuda") for _ in range(2))
    base = dict(target=p, tokens=n, parents=n, uniform=u, path=path, count=count, next_token=following)
    for bad in [dict(path=n), dict(path=u.view(torch.int32)), dict(count=following), dict(count=path[0, :2]), dict(path=p.view(torch.int32)[0, :2, :3])]:
        refused(lib.verify, **{**base, **bad})
    big = torch.zeros(1, 1025, dtype=torch.int32, device="cuda")
    refused(lib.verify, target=torch.zeros(1, 1025, 4, device="cuda"), tokens=big, parents=big, uniform=big.float(), path=big.clone(), count=count[:1],
            next_token=following[:1])
    refused(lib.verify, **{**base, "target": p[:, :, :0]})
    lib.verify(p[:0], n[:0], n[:0], u[:0], path[:0], count[:0], following[:0])
    lib.sync_status()


# ------------------------------------------------------------------ keeping


def paths_of(seed, batch, new, counts):
    g = torch.Generator().manual_seed(seed)
    path = torch.full((batch, new), -1, dtype=torch.int32)
    for b in range(batch):
        path[b, :counts[b]] = torch.randperm(new, generator=g)[:counts[b]].sort().values.to(torch.int32)
    return path


def check_keep(lib, firsts, new, counts, page, heads, dim, seed=3, path=None, change=None):
    c, s, table = make_cache(seed, [max(f, 0) + new for f in firsts], page, heads, dim)
    if change:
        change(c, s, table)
    if path is None:
        path = paths_of(seed, len(firsts), new, counts)
    dev = [t.cuda() for t in (*c, *s)]
    lib.cache_keep(*dev, table.cuda(), ints(firsts).cuda(), path.cuda(), ints(counts).cuda())
    lib.sync_status()
    for i in range(2):
        want, scale = D.keep(c[i], s[i], table, firsts, path, counts)
        assert torch.equal(dev[i].cpu(), want) and torch.equal(dev[i + 2].cpu().nan_to_num(-1), scale.nan_to_num(-1)), i


KEEPS = [  # firsts, new, counts, page, heads, dim
    ([0], 1, [1], 16, 1, 64), ([77], 5, [3], 16, 12, 64), ([30, 0, 15, 16, 17], 9, [1, 9, 4, 8, 0], 16, 2, 128), ([100, 1000], 64, [7, 20], 32, 8, 128),
    ([5, 40], 33, [33, 30], 24, 3, 20), ([3], 40, [21], 1, 2, 4), ([60, 0], 130, [100, 64], 64, 1, 256), ([-1, 20, -5], 8, [3, 5, 8], 16, 2, 96),
    ([1000], 1024, [700], 1024, 1, 64), ([10], 1024, [1024], 128, 2, 64), ([7], 300, [299], 5, 1, 252)]


@pytest.mark.parametrize("firsts,new,counts,page,heads,dim", KEEPS)
def test_keep(lib, firsts, new, counts, page, heads, dim):
    check_keep(lib, firsts, new, counts, page, heads, dim)


def test_keep_what_stays_in_its_place(lib):
    """A chain that was accepted whole, or in part: nothing changes."""
    chain = torch.arange(40, dtype=torch.int32).expand(3, 40)
    c, s, table = make_cache(3, [60, 41, 100], 16, 2, 64)
    dev = [t.cuda() for t in (*c, *s)]
    lib.cache_keep(*dev, table.cuda(), ints([20, 1, 60]).cuda(), chain.cuda(), ints([40, 7, 0]).cuda())
    lib.sync_status()
    for x, y in zip(dev, (*c, *s)):
        # (rows before the drafts too: a page keeps its own scale)
        assert torch.equal(x.cpu(), y)


def test_keep_scales(lib):
    """Pages of zeros, of scales far apart, and without a number."""
    def change(c, s, table):
        for i in range(2):
            s[i][table[0, 1].long()] *= 2.0 ** 40
            s[i][table[1]] = 0
            s[i][table[2, 2].long()] = math.nan
            s[i][table[3, 1].long()] *= 2.0 ** -30

    check_keep(lib, [10, 10, 20, 10], 40, [12, 12, 20, 20], 16, 2, 64, change=change)
    check_keep(lib, [10, 10, 20, 10], 40, [30, 40, 1, 2], 16, 2, 64, change=change)


def test_keep_paths_that_are_none(lib):
    c, s, table = make_cache(3, [60] * 6, 16, 2, 64)
    dev = [t.cuda() for t in (*c, *s)]
    path = paths_of(1, 6, 20, [5] * 6)
    path[0, 2] = path[0, 1]         # twice the same
    path[1, 0] = -1
    path[2, 4] = 20
    path[3, :5] = ints([9, 8, 7, 6, 5])
    counts = ints([5, 5, 5, 5, 21, -1])
    lib.cache_keep(*dev, table.cuda(), ints([40] * 6).cuda(), path.cuda(), counts.cuda())
    reported(lib)
    for x, y in zip(dev, (*c, *s)):
        assert torch.equal(x.cpu(), y)


def test_keep_skips_pages_out_of_range(lib):
    """Rows from a page that is none stay away, and so do rows to one; other sequences are not touched."""
    c, s, table = make_cache(3, [64, 64], 16, 2, 64)
    bad = table.clone()
    bad[0, 3] = c[0].shape[0]
    dev = [t.cuda() for t in (*c, *s)]
    path = torch.full((2, 34), -1, dtype=torch.int32)     # (of 34 drafted tokens)
    path[:, :3] = ints([2, 20, 21])
    lib.cache_keep(*dev, bad.cuda(), ints([30, 30]).cuda(), path.cuda(), ints([3, 3]).cuda())
    reported(lib)
    for i in range(2):
        # of sequence 0 only row 32 moves to 30: under the scales of pages 1 and 2, while 50 and 51 lie in the bad page
        want, scale = D.keep(c[i], s[i], table, [30, 30], path, [1, 3])
        # (position 32, in page 2, would have been the third: nothing of it moved)
        assert torch.equal(dev[i].cpu(), want) and torch.equal(dev[i + 2].cpu(), scale)
    # past the end of the list
    dev = [t.cuda() for t in (*c, *s)]
    path = torch.full((2, 100), -1, dtype=torch.int32)
    path[:, 0] = 99
    lib.cache_keep(*dev, table.cuda(), ints([30, 30]).cuda(), path.cuda(), ints([1, 1]).cuda())
    reported(lib)
    for x, y in zip(dev, (*c, *s)):
        assert torch.equal(x.cpu(), y)


@pytest.mark.parametrize("form", ["rows first", "gaps"])
def test_keep_and_read_caches_of_other_orders(lib, form):
    lens, page, heads, dim = [50, 33], 16, 3, 64
    c, s, table = make_cache(3, lens, page, heads, dim)
    dev = []
    for x in c:
        if form == "rows first":
            dev.append(x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3))
        else:
            big = torch.zeros((x.shape[0], heads, page, dim + 4), dtype=torch.int8, device="cuda")
            big[..., :dim] = x.cuda()
            dev.append(big[..., :dim])
    sd = [t.cuda() for t in s]
    firsts, counts = [30, 13], [6, 9]
    path = paths_of(5, 2, 20, counts)
    lib.cache_keep(*dev, *sd, table.cuda(), ints(firsts).cuda(), path.cuda(), ints(counts).cuda())
    k, v = (torch.zeros((2, 50, heads, dim), dtype=torch.float16, device="cuda") for _ in range(2))
    lib.cache_read(*dev, *sd, table.cuda(), ints([0, 0]).cuda(), ints([36, 22]).cuda(), k, v)
    lib.sync_status()
    for i, out in enumerate((k, v)):
        want, scale = D.keep(c[i], s[i], table, firsts, path, counts)
        assert torch.equal(dev[i].cpu(), want) and torch.equal(sd[i].cpu(), scale)
        assert torch.equal(out.cpu(), D.read(want, scale, table, [0, 0], [36, 22], torch.zeros(2, 50, heads, dim, dtype=torch.float16)))


# ------------------------------------------------------------------ reading


READS = [  # firsts, lens, tokens, page, heads, dim
    ([0], [1], 1, 16, 1, 64), ([70], [77], 7, 16, 12, 64), ([0, 30, 100], [40, 31, 100], 40, 16, 2, 128), ([-3, 5], [20, 100], 30, 32, 3, 96),
    ([0, 17], [200, 63], 200, 24, 2, 20), ([1, 2], [70, 9], 69, 1, 2, 4), ([3], [400], 397, 64, 1, 256), ([100, -200, -10], [50, 50, 0], 60, 16, 2, 64),
    ([5], [1030], 1025, 1024, 1, 252)]


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("firsts,lens,tokens,page,heads,dim", READS)
def test_read(lib, dtype, firsts, lens, tokens, page, heads, dim):
    c, s, table = make_cache(4, lens, page, heads, dim)
    base = U.rand(5, len(lens), tokens, 2 * heads, dim).to(dtype)
    both = base.cuda()      # keys and values are slices of one buffer
    k, v = both[:, :, :heads], both[:, :, heads:]
    lib.cache_read(*[t.cuda() for t in (*c, *s)], table.cuda(), ints(firsts).cuda(), ints(lens).cuda(), k, v)
    lib.sync_status()
    for i, out in enumerate((k, v)):
        # the product in single precision, rounded once more: the same words
        assert torch.equal(out.cpu(), D.read(c[i], s[i], table, firsts, lens, base[:, :, i * heads:(i + 1) * heads]))


@pytest.mark.parametrize("dtype", FLOATS)
def test_read_into_rows_of_other_orders(lib, dtype):
    c, s, table = make_cache(4, [50, 40], 16, 3, 64)
    args = [t.cuda() for t in (*c, *s)], table.cuda(), ints([2, 0]).cuda(), ints([50, 40]).cuda()
    want = [D.read(c[i], s[i], table, [2, 0], [50, 40], torch.zeros(2, 48, 3, 64, dtype=dtype)) for i in range(2)]
    heads_first = [torch.zeros(2, 3, 48, 64, dtype=dtype, device="cuda").transpose(1, 2) for _ in range(2)]
    odd = [torch.zeros(2, 48, 3, 67, dtype=dtype, device="cuda")[..., 1:65] for _ in range(2)]
    for k, v in (heads_first, odd):
        lib.cache_read(*args[0], *args[1:], k, v)
        lib.sync_status()
        assert torch.equal(k.cpu(), want[0]) and torch.equal(v.cpu(), want[1])
    assert not odd[0]._base[..., 0].any() and not odd[0]._base[..., 65:].any()


def test_read_pages_and_lengths_out_of_range(lib):
    c, s, table = make_cache(4, [60], 16, 2, 64)
    bad = table.clone()
    bad[0, 1] = -1
    for t, n in ((bad, 60), (table, 9000)):
        k, v = (torch.full((1, 200, 2, 64), 9.0, device="cuda") for _ in range(2))
        lib.cache_read(*[x.cuda() for x in (*c, *s)], t.cuda(), ints([0]).cuda(), ints([n]).cuda(), k, v)
        reported(lib)
        for i, out in enumerate((k, v)):
            want = D.read(c[i], s[i], table, [0], [n], torch.full((1, 200, 2, 64), 9.0))
            if t is bad:
                want[0, 16:32] = 9
            assert torch.equal(out.cpu(), want)


def test_cache_calls_refuse(lib):
    c, s, table = make_cache(3, [40, 30], 16, 2, 64)
    kc, vc, ks, vs = [t.cuda() for t in (*c, *s)]
    table, n = table.cuda(), ints([0, 0]).cuda()
    path = torch.zeros(2, 5, dtype=torch.int32, device="cuda")
    base = dict(k_cache=kc, v_cache=vc, k_scale=ks, v_scale=vs, page_table=table, first=n, path=path, count=n)
    one = kc[:1].expand(kc.shape[0], -1, -1, -1)
    for bad in [dict(v_cache=kc), dict(v_scale=ks), dict(k_cache=one, v_cache=one), dict(path=kc.view(torch.int32)[0, 0, :2, :5]),
                dict(count=ks.view(torch.int32)[0]), dict(path=torch.zeros(2, 1025, dtype=torch.int32, device="cuda"))]:
        refused(lib.cache_keep, **{**base, **bad})
    k, v = torch.zeros(2, 5, 2, 64, device="cuda"), torch.zeros(2, 5, 2, 64, device="cuda")
    del base["path"], base["count"]
    base.update(lengths=n, k=k, v=v)
    for bad in [dict(v=k), dict(k=k[:, :1].expand(2, 5, 2, 64)), dict(k=v, v=v.view(2, 2, 5, 64).transpose(1, 2)),
                dict(k=kc.view(-1).view(torch.float32)[:1280].view(2, 5, 2, 64))]:
        refused(lib.cache_read, **{**base, **bad})
    lib.cache_keep(kc, vc, ks, vs, table[:0], n[:0], path[:0], n[:0])
    lib.cache_read(kc, vc, ks, vs, table[:0], n[:0], n[:0], k[:0], v[:0])
    lib.sync_status()


def test_beyond_32_bits(lib):
    """A cache of over 4 GiB, with the pages that are used at its end: attention, keep and read."""
    pages, heads, page, dim, new = 70000, 8, 64, 128, 40
    kc = torch.zeros((pages, heads, page, dim), dtype=torch.int8, device="cuda")
    vc = torch.zeros_like(kc)
    ks, vs = torch.zeros((pages, heads), device="cuda"), torch.zeros((pages, heads), device="cuda")
    table = torch.tensor([[pages - 1, 69000, 40000]], dtype=torch.int32)
    at = table[0].long()
    c, s, _ = make_cache(4, [3 * page], page, heads, dim, extra=0)
    for big, small in zip((kc, vc, ks, vs), (*c, *s)):
        big[at.cuda()] = small[:3].cuda()
    own = torch.tensor([[0, 1, 2]], dtype=torch.int32)
    small = [t[:3] for t in (*c, *s)]
    seen = D.ancestors(D.random_tree(2, 1, new))
    for group in (1, 2):
        q = U.rand(2, 1, new, heads * group, dim).half()
        out = torch.empty_like(q, device="cuda")
        lib.tree_attention(q.cuda(), kc, vc, ks, vs, table.cuda(), ints([150]).cuda(), D.words(seen).cuda(), out)
        lib.sync_status()
        ref, size = D.tree_attention(q, *small, own, [150], seen, dim ** -0.5)
        assert torch.all((out.cpu().double() - ref).abs() <= U.UNIT[q.dtype] * ref.abs() + 2.0 ** -10 * size + 1e-9)
    path = paths_of(1, 1, new, [9])
    lib.cache_keep(kc, vc, ks, vs, table.cuda(), ints([110]).cuda(), path.cuda(), ints([9]).cuda())
    k, v = (torch.zeros((1, 119, heads, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lib.cache_read(kc, vc, ks, vs, table.cuda(), ints([0]).cuda(), ints([119]).cuda(), k, v)
    lib.sync_status()
    for i, out in enumerate((k, v)):
        want, scale = D.keep(small[i], small[i + 2], own, [110], path, [9])
        assert torch.equal((kc, vc)[i][at.cuda()].cpu(), want) and torch.equal((ks, vs)[i][at.cuda()].cpu(), scale)
        assert torch.equal(out.cpu(), D.read(want, scale, own, [0], [119], torch.zeros(1, 119, heads, dim, dtype=torch.bfloat16)))


# ------------------------------------------------------------------ together: streams, graphs, two handles


def step_state(nodes, seed=1, vocab=700):
    """What one step over drafted tokens takes: the tree in the cache, its queries, the probabilities behind it."""
    lens = [90 + nodes, 41 + nodes]
    c, s, table = make_cache(seed, lens, 16, 2, 64)
    target, draft, tokens, parents, uniform = (x.cuda() for x in drafted(seed, 2, nodes, vocab, torch.float32, True))
    n = ints(lens).cuda()
    return dict(c=[t.cuda() for t in (*c, *s)], table=table.cuda(), lengths=n, first=n - nodes, q=U.rand(seed, 2, nodes, 8, 64).half().cuda(),
                target=target, draft=draft, tokens=tokens, parents=parents, uniform=uniform,
                mask=torch.empty(2, nodes, -(-nodes // 32), dtype=torch.int32, device="cuda"), out=torch.empty(2, nodes, 8, 64, dtype=torch.float16, device="cuda"),
                path=torch.empty(2, nodes, dtype=torch.int32, device="cuda"), count=torch.empty(2, dtype=torch.int32, device="cuda"),
                following=torch.empty(2, dtype=torch.int32, device="cuda"), k=torch.zeros(2, 140, 2, 64, device="cuda"), v=torch.zeros(2, 140, 2, 64, device="cuda"))


def step(lib, t, stream=None):
    lib.tree_mask(t["parents"], t["mask"], stream=stream)
    lib.tree_attention(t["q"], *t["c"], t["table"], t["lengths"], t["mask"], t["out"], stream=stream)
    lib.verify(t["target"], t["tokens"], t["parents"], t["uniform"], t["path"], t["count"], t["following"], draft=t["draft"], stream=stream)
    lib.cache_keep(*t["c"], t["table"], t["first"], t["path"], t["count"], stream=stream)
    lib.cache_read(*t["c"], t["table"], t["first"], t["lengths"], t["k"], t["v"], stream=stream)


RESULTS = ("mask", "out", "path", "count", "following", "k", "v")


@pytest.mark.parametrize("nodes,vocab", [(5, 700), (40, 700), (12, 20000)])
def test_a_step_on_other_streams_handles_and_in_graphs(lib, nodes, vocab):
    from paper_2609_16915_gb300 import clear
    a = step_state(nodes, vocab=vocab)
    step(lib, a)
    lib.sync_status()
    want = {n: a[n].clone() for n in RESULTS}
    pages, table = [t.cpu() for t in step_state(nodes, vocab=vocab)["c"]], a["table"].cpu()
    ref, size = D.tree_attention(a["q"].cpu(), *pages, table, a["lengths"].tolist(), D.ancestors(a["parents"].cpu()), 0.125)
    assert torch.all((a["out"].cpu().double() - ref).abs() <= U.UNIT[torch.float16] * ref.abs() + 2.0 ** -10 * size + 1e-9)
    for b in range(2):
        got = D.verify(*[a[n][b].cpu() for n in ("target", "draft", "tokens", "parents", "uniform")])
        assert (a["path"][b, :got[1]].tolist(), int(a["count"][b]), int(a["following"][b])) == got
    for i, name in enumerate("kv"):
        held, scale = D.keep(pages[i], pages[i + 2], table, a["first"].tolist(), a["path"].cpu(), a["count"].tolist())
        assert torch.equal(a["c"][i].cpu(), held) and torch.equal(a["c"][i + 2].cpu(), scale)
        assert torch.equal(a[name].cpu(), D.read(held, scale, table, a["first"].tolist(), a["lengths"].tolist(), torch.zeros(2, 140, 2, 64)))

    # two handles at once, on streams of their own
    others = [(clear.Clear(), step_state(nodes, vocab=vocab), torch.cuda.Stream()) for _ in range(2)]
    torch.cuda.synchronize()
    for handle, t, s in others:
        step(handle, t, stream=s)
    for handle, t, s in others:
        handle.sync_status(s)
        assert all(torch.equal(t[n], want[n]) for n in RESULTS)

    b = step_state(nodes, vocab=vocab)
    start = [x.clone() for x in b["c"]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(lib, b)
    for _ in range(2):
        for x, y in zip(b["c"], start):
            x.copy_(y)
        for n in RESULTS:
            b[n].zero_()
        graph.replay()
        lib.sync_status()
        assert all(torch.equal(b[n], want[n]) for n in RESULTS)
