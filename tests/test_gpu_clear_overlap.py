"""Outputs whose rows share memory are refused before anything is enqueued; every order of rows that lie apart is taken."""

import pytest
import torch

from tests import clear_util as U
from tests.test_gpu_clear import lib, make_cache  # noqa: F401  (lib: the fixture)

pytestmark = pytest.mark.gpu

LENS, PAGE, HEADS, DIM = [40, 33], 16, 2, 64


def refused(call):
    from paper_2609_16915_gb300 import RosettaError
    with pytest.raises(RosettaError) as e:
        call()
    assert e.value.status == -1


@pytest.mark.parametrize("new", [1, 3, 40])
def test_attention_outputs(lib, new):
    c, s, table = make_cache(3, LENS, PAGE, HEADS, DIM)
    args = [t.cuda() for t in (*c, *s, table)]
    lengths = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    q = U.rand(4, 2, new, 4, DIM).cuda()
    want = torch.empty_like(q)
    lib.attention(q, *args, lengths, want)

    def run(out):
        lib.attention(q, *args, lengths, out)
        return out

    big = torch.zeros(1 << 20, device="cuda")
    refused(lambda: run(big[:DIM].expand(2, new, 4, DIM)))
    refused(lambda: run(big[:new * 4 * DIM].view(1, new, 4, DIM).expand(2, -1, -1, -1)))
    refused(lambda: run(big[:2 * new * DIM].view(2, new, 1, DIM).expand(-1, -1, 4, -1)))
    refused(lambda: run(big.as_strided((2, new, 4, DIM), (new * 4 * DIM - 1, 4 * DIM, DIM, 1))))
    refused(lambda: run(big.as_strided((2, new, 4, DIM), (4 * new * DIM, 4 * DIM, DIM - 4, 1))))
    if new > 1:
        refused(lambda: run(big[:8 * DIM].view(2, 1, 4, DIM).expand(-1, new, -1, -1)))
    assert not big.any()
    # heads, sequences and tokens outermost; slices; a stride that no row uses
    for order in [(0, 2, 1), (1, 0, 2), (2, 1, 0), (2, 0, 1)]:
        shape = [(2, new, 4)[i] for i in order]
        back = [order.index(i) for i in range(3)]
        assert torch.equal(run(torch.empty((*shape, DIM), device="cuda").permute(*back, 3)), want)
        assert torch.equal(run(torch.empty((*shape, DIM + 8), device="cuda").permute(*back, 3)[..., :DIM]), want)
    one = torch.empty((1, new, 4, DIM), device="cuda").expand(1, -1, -1, -1)
    lib.attention(q[:1], *args[:4], args[4][:1], lengths[:1], one.as_strided((1, new, 4, DIM), (0, 4 * DIM, DIM, 1)))
    assert torch.equal(one, want[:1])
    lib.sync_status()


def test_appended_caches(lib):
    c, s, table = make_cache(3, LENS, PAGE, HEADS, DIM)
    x = U.rand(5, 2, 3, HEADS, DIM)
    first = torch.tensor([20, 30], dtype=torch.int32)
    want = [U.append(x, c[i], s[i], table, first) for i in range(2)]
    xd, td, fd = x.cuda(), table.cuda(), first.cuda()
    k, v, ks, vs = [t.cuda() for t in (*c, *s)]

    def run(k, v, ks, vs):
        lib.cache_append(xd, xd, k, v, ks, vs, td, fd)

    wide = k[:1].expand(k.shape[0], -1, -1, -1)
    before = [t.clone() for t in (k, v, ks, vs)]
    refused(lambda: run(k, k, ks, vs))
    refused(lambda: run(k, v, ks, ks))
    refused(lambda: run(wide, wide, ks, vs))
    heads = k[:, :1].expand(-1, HEADS, -1, -1)
    refused(lambda: run(heads, heads, ks, vs))
    half = torch.zeros(k.numel() + 64, dtype=torch.int8, device="cuda")
    refused(lambda: run(half[:k.numel()].view(k.shape), half[64:].view(k.shape), ks, vs))
    lib.sync_status()
    for a, b in zip(before, (k, v, ks, vs)):
        assert torch.equal(a, b)
    # keys and values of a page, of a head, of a row side by side
    for at in (1, 2, 3):
        both = torch.stack([k, v], at)
        pair = both.select(at, 0), both.select(at, 1)
        ksd, vsd = ks.clone(), vs.clone()
        run(*pair, ksd, vsd)
        lib.sync_status()
        for i in range(2):
            assert torch.equal(pair[i].cpu(), want[i][0]) and torch.equal((ksd, vsd)[i].cpu(), want[i][1])
