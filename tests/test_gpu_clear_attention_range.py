"""Attention where the value scales of pages lie far apart.  A row's weights are rounded relative to what the row
itself sees: pages it does not see, or gives no weight to, take nothing from it, whatever their scales.

Bounds: the output's rounding; the weights' for the product with V (11 bits for bfloat16, 22 otherwise), and scores in
single precision, both relative to sum p |v| of the row."""

import pytest
import torch

from tests import clear_util as U
from tests.test_gpu_clear import FLOATS, lib, make_cache  # noqa: F401  (lib: the fixture)

pytestmark = pytest.mark.gpu


def check(lib, dtype, q, c, s, table, lens, rows=None):
    """rows[b]: the tokens of sequence b that are compared (all)."""
    dim = q.shape[3]
    lengths = torch.tensor(lens, dtype=torch.int32)
    out = torch.full(q.shape, 9.0, dtype=dtype, device="cuda")
    lib.attention(q.cuda(), *[t.cuda() for t in (*c, *s)], table.cuda(), lengths.cuda(), out)
    lib.sync_status()
    want, size = U.attention(q, *c, *s, table, lengths, dim ** -0.5)
    weights = 2.0 ** -10 if dtype == torch.bfloat16 else 2.0 ** -16
    err = (out.cpu().double() - want).abs()
    bound = 1.01 * U.UNIT[dtype] * want.abs() + weights * size + (2.0 ** -25 if dtype == torch.float16 else 1e-42)
    for b in range(len(lens)):
        t = slice(None) if rows is None else rows[b]
        assert torch.all(err[b, t] <= bound[b, t]), float((err[b, t] / (size[b, t] + 1e-300)).max())


EXPONENTS = [10, 14, 20, 27, 60, 90]
DECODE = [  # new, heads, group, dim, page
    (1, 2, 4, 128, 16), (1, 12, 1, 64, 32), (2, 1, 8, 96, 16), (3, 2, 5, 256, 16), (1, 2, 2, 20, 16)]
PROMPTS = [(40, 2, 4, 128, 16), (70, 1, 1, 64, 32), (90, 2, 3, 96, 16), (40, 1, 2, 256, 16), (20, 2, 2, 20, 16)]


def without_weight(lib, dtype, exponent, new, heads, group, dim, page, lens):
    c, s, table = make_cache(3, lens, page, heads, dim)
    q = (1 + 0.3 * U.rand(4, len(lens), new, heads * group, dim)).to(dtype)
    for b in range(len(lens)):
        p = table[b, 1].long()      # scores of about -60: weights of 2^-86
        c[0][p], s[0][p] = -127, 60 / (127 * dim ** 0.5)
        s[1][p] *= 2.0 ** exponent
    # (rows that see nothing else do not exist: the first page is before it)
    check(lib, dtype, q, c, s, table, lens)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("exponent", EXPONENTS)
@pytest.mark.parametrize("new,heads,group,dim,page", DECODE)
def test_decoding_beside_a_page_without_weight(lib, dtype, exponent, new, heads, group, dim, page):
    if exponent < 90:               # (2^-86 of 2^90 is weight again)
        without_weight(lib, dtype, exponent, new, heads, group, dim, page, [150, 64])


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("exponent", [14, 27, 60])
def test_decoding_over_ranges_of_a_long_context(lib, dtype, exponent):
    without_weight(lib, dtype, exponent, 1, 2, 4, 128, 16, [3000, 1500])


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("exponent", EXPONENTS)
def test_decoding_before_a_page_of_another_token(lib, dtype, exponent):
    """Three tokens, the last alone on its page: the first two do not see it."""
    lens, page, heads, dim = [97, 33], 16, 2, 64
    c, s, table = make_cache(5, lens, page, heads, dim)
    for b, n in enumerate(lens):
        s[1][table[b, (n - 1) // page].long()] *= 2.0 ** exponent
    q = U.rand(6, 2, 3, heads * 2, dim).to(dtype)
    check(lib, dtype, q, c, s, table, lens, [slice(0, 2)] * 2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("exponent", [14, 20, 27, 60])
def test_decoding_values_that_shrink_from_page_to_page(lib, dtype, exponent):
    """The weight lies on pages of ever smaller and ever larger scales."""
    lens, page, heads, dim = [200, 90], 16, 2, 64
    for sign in (-1, 1):
        c, s, table = make_cache(7, lens, page, heads, dim)
        q = (1 + 0.3 * U.rand(8, 2, 1, heads * 4, dim)).to(dtype)
        for b, n in enumerate(lens):
            last = (n - 1) // page
            for j in range(last + 1):
                p = table[b, j].long()
                s[1][p] *= 2.0 ** (sign * exponent * j / last)
                c[0][p], s[0][p] = 127, 20 * (1 + sign * -j / last) / (127 * dim ** 0.5)      # weights that go the other way
        check(lib, dtype, q, c, s, table, lens)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("exponent,score", [(-30, 5.0), (-30, 27.0), (-90, 20.0), (30, 0.0), (30, -20.0), (None, 3.0)])
def test_decoding_scales_that_change_far_into_a_long_context(lib, dtype, exponent, score):
    """Ranges of over 4096 positions, whose first 4096 have other scales (None: zeros) and other scores than the rest."""
    batch, context, page, dim, group, half = 160, 1 << 16, 64, 64, 4, 32
    c = [U.int8(i, 2 * half, 1, page, dim) for i in (1, 2)]
    s = [(1 + U.rand(i, 2 * half, 1).abs()) / 60 for i in (3, 4)]
    c[0][:half], s[0][:half] = 127 if score >= 0 else -127, max(abs(score), 1e-3) / (127 * dim ** 0.5)
    s[1][:half] *= 0.0 if exponent is None else 2.0 ** exponent
    q = (1 + 0.3 * U.rand(5, 1, 1, group, dim)).to(dtype)
    at = torch.arange(context // page)
    table = torch.where(at < 64, at * 7 % half, half + at * 5 % half).to(torch.int32)[None]
    out = torch.empty((batch, 1, group, dim), dtype=dtype, device="cuda")
    lib.attention(q.cuda().expand(batch, -1, -1, -1).contiguous(), *[t.cuda() for t in (*c, *s)],
                  table.cuda().expand(batch, -1).contiguous(), torch.full((batch,), context, dtype=torch.int32, device="cuda"), out)
    lib.sync_status()
    want, size = U.attention(q, *c, *s, table, [context], dim ** -0.5)
    weights = 2.0 ** -10 if dtype == torch.bfloat16 else 2.0 ** -16
    assert torch.all((out.cpu().double() - want).abs() <= 1.01 * U.UNIT[dtype] * want.abs() + weights * size + 1e-42)


def at_the_ends(lib, dtype, exponent, new):
    lens, page, heads, dim = [100, 64], 16, 2, 64
    c, s, table = make_cache(13, lens, page, heads, dim)
    s[1] *= 2.0 ** exponent
    check(lib, dtype, U.rand(14, 2, new, heads * 2, dim).to(dtype), c, s, table, lens)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("exponent", [-112, -60, 60, 118])
def test_decoding_scales_at_the_ends_of_single_precision(lib, dtype, exponent):
    at_the_ends(lib, dtype, exponent, 1)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("exponent", EXPONENTS)
@pytest.mark.parametrize("new,heads,group,dim,page", PROMPTS)
def test_prompts_beside_a_page_without_weight(lib, dtype, exponent, new, heads, group, dim, page):
    if exponent < 90:
        without_weight(lib, dtype, exponent, new, heads, group, dim, page, [150, 32 + new])


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("exponent", [14, 27, 60])
def test_prompts_over_ranges_of_a_long_context(lib, dtype, exponent):
    without_weight(lib, dtype, exponent, 20, 1, 4, 128, 16, [3000, 1500])


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("exponent", EXPONENTS)
@pytest.mark.parametrize("new,heads,group,dim,page", PROMPTS)
def test_prompts_before_later_pages(lib, dtype, exponent, new, heads, group, dim, page):
    """The last page's scale: tokens before it do not see it."""
    lens = [150, new]
    c, s, table = make_cache(5, lens, page, heads, dim)
    rows = []
    for b, n in enumerate(lens):
        last = (n - 1) // page
        s[1][table[b, last].long()] *= 2.0 ** exponent
        rows.append(slice(0, max(0, last * page - (n - new))))
    q = U.rand(6, 2, new, heads * group, dim).to(dtype)
    check(lib, dtype, q, c, s, table, lens, rows)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("exponent", [14, 20, 27, 60])
def test_prompts_over_values_that_shrink_from_page_to_page(lib, dtype, exponent):
    lens, new, page, heads, dim = [200, 90], 60, 16, 2, 64
    for sign in (-1, 1):
        c, s, table = make_cache(7, lens, page, heads, dim)
        q = (1 + 0.3 * U.rand(8, 2, new, heads * 2, dim)).to(dtype)
        for b, n in enumerate(lens):
            last = (n - 1) // page
            for j in range(last + 1):
                p = table[b, j].long()
                s[1][p] *= 2.0 ** (sign * exponent * j / last)
                c[0][p], s[0][p] = 127, 20 * (1 + sign * -j / last) / (127 * dim ** 0.5)
        check(lib, dtype, q, c, s, table, lens)


@pytest.mark.parametrize("new", [1, 60])
@pytest.mark.parametrize("dtype", FLOATS)
def test_value_scales_of_either_sign_and_none(lib, dtype, new):
    """Negative scales, pages of zeros first and last, and pages that hold nothing but zeros."""
    lens, page, heads, dim = [180, 70], 16, 2, 64
    c, s, table = make_cache(9, lens, page, heads, dim)
    s[1] *= torch.where(torch.arange(s[1].numel()) % 3 == 0, -1.0, 1.0).reshape(s[1].shape)
    for b, n in enumerate(lens):
        s[1][table[b, 0].long()] = 0
        s[1][table[b, (n - 1) // page].long()] = 0
    q = U.rand(6, 2, new, heads * 2, dim).to(dtype)
    check(lib, dtype, q, c, s, table, lens)
    s[1].zero_()
    check(lib, dtype, q, c, s, table, lens)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("exponent", [-112, -60, 60, 118])
def test_prompts_scales_at_the_ends_of_single_precision(lib, dtype, exponent):
    at_the_ends(lib, dtype, exponent, 60)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("context", [1 << 15, 1 << 17, 1 << 18])
def test_sums_of_long_contexts_lose_no_more_than_said(lib, dtype, context):
    """Values of one sign, one range for a whole context: what the tensor cores cut off is one-sided, so the mean of the errors
    shows it below the outputs' own rounding (2^-9 of a bfloat16 at most: the mean of 100 outputs that have nothing in common
    is within 1e-4, and there are 25600).  An accumulator loses 2^-12 at most."""
    pages, page, dim, group, batch, own = 32, 64, 128, 50, 160, 4
    kc, vc = U.int8(5, pages, 1, page, dim), U.int8(6, pages, 1, page, dim, lo=1)
    g = torch.Generator().manual_seed(7)
    ks, vs = torch.rand((pages, 1), generator=g) / 60, (1 + torch.rand((pages, 1), generator=g)) / 60
    q = U.rand(9, own, 1, group, dim).to(dtype)
    table = (torch.arange(context // page) * 7 % pages).to(torch.int32)
    out = torch.empty((batch, 1, group, dim), dtype=dtype, device="cuda")
    lib.attention(q.cuda().repeat(batch // own, 1, 1, 1), kc.cuda(), vc.cuda(), ks.cuda(), vs.cuda(), table.cuda().expand(batch, -1).contiguous(),
                  torch.full((batch,), context, dtype=torch.int32, device="cuda"), out)
    lib.sync_status()
    one = torch.arange(pages, dtype=torch.int32)[None].expand(own, -1).contiguous()
    want, size = U.attention(q, kc, vc, ks, vs, one, [pages * page] * own, dim ** -0.5)
    err = (out[:own].cpu().double() - want) / size
    assert abs(float(err.mean())) <= 2.0 ** -12 + 1e-4, float(err.mean())


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("dim,rising", [(128, 30.0), (64, -30.0), (128, 0.0)])
def test_ranges_of_more_than_one_run(lib, dtype, dim, rising):
    """Contexts around multiples of 32768, under lists for more, whose scores rise or fall by `rising` on the way."""
    lens, page, group, capacity = [70000, 32768, 32769, 33000, 65536, 65601, 500, 0], 64, 48, 1 << 17
    pages = -(-max(lens) // page)
    c = [U.int8(i, pages, 1, page, dim) for i in (1, 2)]
    s = [(1 + U.rand(i, pages, 1).abs()) / 60 for i in (3, 4)]
    if rising:
        c[0][:] = torch.where(U.int8(5, *c[0].shape) > 0, 127, 120).to(torch.int8)
        s[0][:, 0] = rising * torch.arange(pages) / pages / (124 * dim ** 0.5) + 1e-4
    q = (1 + 0.3 * U.rand(6, len(lens), 1, group, dim)).to(dtype)
    table = torch.zeros(len(lens), capacity // page, dtype=torch.int32)
    table[:, :pages] = torch.arange(pages)
    many = 20                       # (as many blocks as fill the GPU: no splits)
    out = torch.empty((len(lens) * many, 1, group, dim), dtype=dtype, device="cuda")
    lib.attention(q.cuda().repeat(many, 1, 1, 1), *[t.cuda() for t in (*c, *s)], table.cuda().repeat(many, 1),
                  torch.tensor(lens * many, dtype=torch.int32, device="cuda"), out)
    lib.sync_status()
    got = out.cpu().reshape(many, len(lens), 1, group, dim)
    assert bool((got == got[0]).all())
    want, size = U.attention(q, *c, *s, table, lens, dim ** -0.5)
    # the weights; for 16-bit types what accumulators lose besides
    weights = {torch.float32: 2.0 ** -16, torch.float16: 2.0 ** -12 + 2.0 ** -16, torch.bfloat16: 2.0 ** -10 + 2.0 ** -12}[dtype]
    assert torch.all((got[0].double() - want).abs() <= 1.01 * U.UNIT[dtype] * want.abs() + weights * size + 2.0 ** -25)


# ------------------------------------------------------------------ what a call asks memory for


def used_by(call):
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    call()
    return before - torch.cuda.mem_get_info()[0]


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("new,heads,group,dim,capacity", [(2048, 8, 4, 128, 1 << 17), (2048, 8, 4, 128, 1 << 20), (1024, 8, 2, 256, 1 << 20),
                                                         (1, 8, 4, 128, 1 << 20)])
def test_workspace_does_not_follow_the_page_lists(dtype, new, heads, group, dim, capacity):
    """Short sequences under page lists for long ones: no more than 256 MiB, or what one cached head of one sequence takes."""
    from paper_2609_16915_gb300 import clear
    batch, page = 8, 64
    kc = torch.zeros((64, heads, page, dim), dtype=torch.int8, device="cuda")
    ks = torch.ones((64, heads), device="cuda")
    table = (torch.arange(batch * (capacity // page), device="cuda") % 64).to(torch.int32).reshape(batch, -1)
    q = torch.zeros((batch, new, heads * group, dim), dtype=dtype, device="cuda")
    out = torch.empty_like(q)
    lengths = torch.full((batch,), min(new + 100, 500), dtype=torch.int32, device="cuda")
    lib = clear.Clear()
    used = used_by(lambda: (lib.attention(q, kc, kc, ks, ks, table, lengths, out), lib.sync_status()))
    lib.close()
    assert used <= (256 << 20) + (64 << 20)


@pytest.mark.parametrize("dtype,new,heads,group,dim,length", [(torch.float32, 512, 4, 2, 256, 3000), (torch.float32, 2048, 8, 4, 128, 2500),
                                                             (torch.float32, 2048, 8, 4, 128, 33000)])
def test_heads_in_several_launches(lib, dtype, new, heads, group, dim, length):
    """More partial results than 256 MiB: the same as sequence by sequence under lists for no more than the length (each within
    2^-16 of the sums of |v|, at most 127 x 1.5 / 60)."""
    batch, page = 8, 64
    each = -(-length // page)
    c, s, _ = make_cache(3, [length], page, heads, dim, extra=0)
    c, s = [t.cuda() for t in c], [t.cuda() for t in s]
    table = (torch.arange(batch)[:, None] * 5 + torch.arange(each)) % each
    lists = torch.zeros((batch, (1 << 20) // page), dtype=torch.int32)
    lists[:, :each] = table
    q = U.rand(4, batch, new, heads * group, dim).to(dtype).cuda()
    lengths = torch.tensor([length - 3 * b for b in range(batch)], dtype=torch.int32, device="cuda")
    out, one = torch.empty_like(q), torch.empty_like(q)
    lib.attention(q, *c, *s, lists.cuda(), lengths, out)
    short = table.to(torch.int32).cuda().contiguous()
    for b in range(batch):
        lib.attention(q[b:b + 1], *c, *s, short[b:b + 1], lengths[b:b + 1], one[b:b + 1])
    lib.sync_status()
    assert float((out - one).abs().max()) <= 2 * 2.0 ** -16 * 127 * 1.5 / 60


@pytest.mark.parametrize("lens,new,page,heads,group,dim", [
    ([1], 1, 16, 1, 1, 64), ([5], 1, 16, 4, 4, 128), ([77, 30], 1, 16, 6, 2, 64), ([16, 3], 2, 16, 2, 8, 96), ([40], 20, 16, 2, 1, 256),
    ([60, 50], 48, 16, 2, 1, 128), ([33], 33, 32, 2, 4, 64), ([300], 90, 16, 1, 4, 96)])
def test_float16_weights_of_22_bits(lib, lens, new, page, heads, group, dim):
    """Values whose terms cancel, so that the weights' rounding shows beside the output's: with 11 bits every one of these shapes
    is past the bound."""
    c, s, table = make_cache(11, lens, page, heads, dim)
    check(lib, torch.float16, U.rand(12, len(lens), new, heads * group, dim).half(), c, s, table, lens)


@pytest.mark.parametrize("rest", [-112, -50, 0, 60])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_decoding_zeros_far_into_a_long_context(lib, dtype, rest):
    """The first 4096 positions of every range are zeros, and the scales behind them are far from 1."""
    batch, page, dim, group, context = 160, 64, 64, 4, 1 << 16
    c = [U.int8(i, 64, 1, page, dim) for i in (1, 2)]
    s = [(1 + U.rand(i, 64, 1).abs()) / 60 for i in (3, 4)]
    s[1][:32], s[1][32:] = 0, s[1][32:] * 2.0 ** rest
    q = U.rand(5, 1, 1, group, dim).to(dtype)
    at = torch.arange(context // page)
    table = torch.where(at % 70 < 66, at * 7 % 32, 32 + at * 5 % 32).to(torch.int32)[None]
    out = torch.empty((batch, 1, group, dim), dtype=dtype, device="cuda")
    lib.attention(q.cuda().expand(batch, -1, -1, -1).contiguous(), *[t.cuda() for t in (*c, *s)],
                  table.cuda().expand(batch, -1).contiguous(), torch.full((batch,), context, dtype=torch.int32, device="cuda"), out)
    lib.sync_status()
    want, size = U.attention(q, *c, *s, table, [context], dim ** -0.5)
    weights = 2.0 ** -10 if dtype == torch.bfloat16 else 2.0 ** -16
    assert torch.all((out.cpu().double() - want).abs() <= 1.01 * U.UNIT[dtype] * want.abs() + weights * size + 1e-42)
