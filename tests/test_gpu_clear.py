"""The decoder layer in the clear (rosetta_clear_*) against its definitions.

Whole numbers (sums, codes, cache bytes and their scales) have to be equal; floats stay
within bounds that follow from their roundings, stated at each check."""

import math

import numpy as np
import pytest
import torch

from tests import clear_util as U

pytestmark = pytest.mark.gpu

FLOATS = [torch.float32, torch.float16, torch.bfloat16]


@pytest.fixture(scope="module")
def lib():
    from paper_2609_16915_gb300 import clear
    return clear.Clear()


# ------------------------------------------------------------------ norm


def run_norm(lib, x, residual, gamma, eps, alias=False):
    t, w = x.shape
    q = torch.full((t, w), 99, dtype=torch.int8, device="cuda")
    scale = torch.full((t,), 99.0, device="cuda")
    xd, rd = x.cuda(), residual.cuda() if residual is not None else None
    out = rd if alias else torch.empty_like(xd)
    lib.norm(xd, gamma.cuda(), q, scale, residual=rd, sum_out=out, eps=eps)
    lib.sync_status()
    return q.cpu(), scale.cpu(), out.cpu()


def check_norm(x, residual, gamma, eps, got):
    q, scale, total = got
    y, want, h = U.norm(x, residual, gamma, eps)
    # the sum of squares: width / 64 additions in a row at most, then a tree, each half a unit
    rel = 2.0 ** -24 * (x.shape[1] / 64 + 40)
    assert torch.all((scale.double() - want).abs() <= rel * want + 1e-42)
    s = scale.double()[:, None]
    assert torch.all((q.double() * s - y).abs() <= s * (0.5 + 128 * rel) + 1e-42)
    assert torch.all((total.double() - h).abs() <= h.abs() * U.UNIT[x.dtype] * (1 + 2.0 ** -10) + 2.0 ** -25)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("tokens,width", [(1, 1), (1, 768), (3, 7), (5, 64), (2, 255), (4, 1021), (77, 4096), (3, 8200),
                                          (2, 16384), (2, 40961)])
def test_norm(lib, dtype, tokens, width):
    x, r = U.rand(1, tokens, width).to(dtype), (3 * U.rand(2, tokens, width)).to(dtype)
    gamma = 1 + 0.2 * U.rand(3, width)
    check_norm(x, r, gamma, 1e-5, run_norm(lib, x, r, gamma, 1e-5))
    check_norm(x, None, gamma, 0.0, run_norm(lib, x, None, gamma, 0.0))


def test_norm_in_place_and_wider_rows(lib):
    x, r = U.rand(1, 9, 520).to(torch.bfloat16), U.rand(2, 9, 520).to(torch.bfloat16)
    gamma = U.rand(3, 520)
    check_norm(x, r, gamma, 1e-6, run_norm(lib, x, r, gamma, 1e-6, alias=True))
    for off, width in [(0, 512), (1, 512), (8, 504), (3, 77)]:
        wide = U.rand(4, 9, 520 + 3).cuda()
        q = torch.full((9, 600), 99, dtype=torch.int8, device="cuda")
        scale = torch.empty(9, device="cuda")
        part = wide[:, off:off + width]
        g = U.rand(5, width)
        lib.norm(part, g.cuda(), q[:, 5:5 + width], scale)
        lib.sync_status()
        assert bool((q[:, :5] == 99).all()) and bool((q[:, 5 + width:] == 99).all())
        check_norm(part.cpu(), None, g, 1e-6, (q[:, 5:5 + width].cpu(), scale.cpu(), part.cpu()))


def test_norm_rows_of_zero_tiny_and_not_finite(lib):
    x = U.rand(1, 6, 300)
    x[0] = 0                        # scale 0
    x[1] *= 1e-30                   # eps dominates
    x[2, 17] = math.nan
    x[3, 299] = math.inf
    x[4, 0] = -math.inf
    gamma = torch.ones(300)
    q, scale, total = run_norm(lib, x, None, gamma, 1e-6)
    assert scale[0] == 0 and not q[0].any()
    assert torch.isnan(scale[2:5]).all()
    check_norm(x[[0, 1, 5]], None, gamma, 1e-6, (q[[0, 1, 5]], scale[[0, 1, 5]], total[[0, 1, 5]]))
    # eps 0 and a row of zeros: 0 * infinity has no value, and the scale says so
    assert torch.isnan(run_norm(lib, torch.zeros(1, 40), None, torch.ones(40), 0.0)[1]).all()


def test_norm_refuses(lib):
    from paper_2609_16915_gb300 import RosettaError
    x, g = torch.randn(4, 64, device="cuda"), torch.ones(64, device="cuda")
    q, s = torch.empty(4, 64, dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    for bad in [dict(x=x.cpu()), dict(gamma=g[:63]), dict(q=q.float()), dict(scale=s[:3]), dict(residual=x.half()),
                dict(x=x.t()), dict(gamma=g.double()), dict(x=x.double())]:
        with pytest.raises(ValueError):
            lib.norm(**{**dict(x=x, gamma=g, q=q, scale=s), **bad})
    for bad in [dict(eps=-1.0), dict(eps=math.nan), dict(sum_out=x[:, :64].view(4, 64), residual=None, q=x.view(torch.int8)[:, :64]),
                dict(scale=x[0, :4])]:
        with pytest.raises(RosettaError) as e:
            lib.norm(**{**dict(x=x, gamma=g, q=q, scale=s), **bad})
        assert e.value.status == -1
    lib.norm(x[:0], g, q[:0], s[:0])    # no tokens
    lib.sync_status()


# ------------------------------------------------------------------ linear


def run_linear(lib, q, scale, weight, w_scale, bias, dtype):
    w = lib.pack_weights(weight.cuda())
    out = torch.full((q.shape[0], weight.shape[0]), 7, dtype=dtype, device="cuda")
    lib.linear(q.cuda(), scale.cuda(), w, w_scale.cuda(), out, bias=None if bias is None else bias.cuda())
    lib.sync_status()
    return out.cpu()


SIZES = [(1, 1, 1), (1, 768, 130), (2, 64, 128), (3, 65, 129), (5, 1021, 37), (8, 16, 300), (9, 4096, 64), (16, 200, 257),
         (17, 1024, 128), (31, 1025, 100), (64, 2048, 384), (65, 1000, 130), (130, 3000, 515), (256, 129, 128), (300, 2100, 260)]


@pytest.mark.parametrize("tokens,inner,channels", SIZES)
def test_linear(lib, tokens, inner, channels):
    q, weight = U.int8(1, tokens, inner, lo=-128), U.int8(2, channels, inner, lo=-128)
    scale, w_scale = U.rand(3, tokens).abs() / 50, U.rand(4, channels) / 70
    bias = U.rand(5, channels)
    want = torch.from_numpy(U.linear(q, scale, weight, w_scale, bias))
    for dtype in FLOATS:
        assert torch.equal(run_linear(lib, q, scale, weight, w_scale, bias, dtype), want.to(dtype))
    plain = torch.from_numpy(U.linear(q, scale, weight, w_scale, None))
    assert torch.equal(run_linear(lib, q, scale, weight, w_scale, None, torch.float32), plain)


@pytest.mark.parametrize("tokens", [1, 8, 40, 257])
@pytest.mark.parametrize("inner", [1024, 1025, 5000, 131071])
def test_linear_sums_at_the_ends_of_their_range(lib, tokens, inner):
    """Every product at its largest, and low bits that count: sums that single precision does not hold."""
    q = torch.full((tokens, inner), -128, dtype=torch.int8)
    weight = torch.full((4, inner), -128, dtype=torch.int8)
    weight[1, 1::2] = 127
    weight[2] = 127
    weight[3, -1] = -127
    q[-1, 0] = -127
    one = torch.ones(tokens)
    # the sum minus a multiple of 2^23 fits single precision: compare the sums themselves through a bias
    acc = q.numpy().astype(np.int64) @ weight.numpy().astype(np.int64).T
    got = run_linear(lib, q, one, weight, torch.ones(4), None, torch.float32)
    assert torch.equal(got, torch.from_numpy(acc.astype(np.float32)))
    # low bits: cancelling halves leave a small exact rest
    half = inner // 2
    q2 = torch.full((tokens, inner), 127, dtype=torch.int8)
    w2 = torch.full((1, inner), 127, dtype=torch.int8)
    w2[0, half:] = -127
    w2[0, 0], w2[0, -1] = 126, -125
    got = run_linear(lib, q2, one, w2, torch.ones(1), None, torch.float32)
    want = q2.numpy().astype(np.int64) @ w2.numpy().astype(np.int64).T
    assert torch.equal(got, torch.from_numpy(want.astype(np.float32)))


@pytest.mark.parametrize("tokens,inner,channels", [(1, 768, 300), (7, 100, 33), (20, 513, 200), (140, 1100, 300)])
@pytest.mark.parametrize("bits", [1, 3, 6, 8])
def test_linear_codes(lib, tokens, inner, channels, bits):
    q, weight = U.int8(1, tokens, inner), U.int8(2, channels, inner)
    scale, w_scale = (1 + U.rand(3, tokens).abs()) / 60, 2 / (73 * math.sqrt(inner)) * (1 + U.rand(4, channels).abs())
    bias, table = U.rand(5, channels), U.int8(6, 1 << bits, lo=-128)
    want = U.codes(U.linear(q, scale, weight, w_scale, bias), bits, -4.0, 3.5)
    w = lib.pack_weights(weight.cuda())
    code = torch.empty((tokens, channels), dtype=torch.uint8, device="cuda")
    values = torch.empty((tokens, channels), dtype=torch.int8, device="cuda")
    lib.linear_codes(q.cuda(), scale.cuda(), w, w_scale.cuda(), code, bits, -4.0, 3.5, bias=bias.cuda(),
                     table=table.cuda(), values=values)
    only = torch.empty_like(code)
    lib.linear_codes(q.cuda(), scale.cuda(), w, w_scale.cuda(), only, bits, -4.0, 3.5, bias=bias.cuda())
    lib.sync_status()
    assert np.array_equal(code.cpu().numpy(), want) and torch.equal(only, code)
    assert torch.equal(values.cpu(), table[torch.from_numpy(want).long()])


TILED = [  # tiles of 64, 128 and 256 tokens, each alone, in several rounds, and in clusters of 2, 4 and 8
    (65, 129, 6000), (200, 64, 6000), (33, 2100, 6000), (100, 2100, 1300), (33, 40000, 4), (257, 1024, 4100), (65, 2100, 6000),
    (65, 2100, 2500), (100, 8192, 1300), (700, 512, 4100), (257, 2048, 4100), (200, 4096, 2500), (200, 8192, 1300), (333, 1021, 2999),
    # groups of 8, 16, 24 and 32 tokens of the kernel for few, one of them and several
    (40, 3072, 768), (64, 768, 3072), (96, 2048, 2000), (24, 1000, 6000), (30, 4096, 4100), (128, 768, 3072), (32, 14336, 300)]


@pytest.mark.parametrize("tokens,inner,channels", TILED)
def test_linear_tiles_and_groups(lib, tokens, inner, channels):
    q, weight = U.int8(1, tokens, inner, lo=-128), U.int8(2, channels, inner, lo=-128)
    scale, w_scale, bias = U.rand(3, tokens).abs() / 50, U.rand(4, channels) / 70, U.rand(5, channels)
    acc = (q.double() @ weight.double().T).numpy()          # (whole numbers below 2^31: exact)
    want = acc.astype(np.float32) * scale.numpy()[:, None] * w_scale.numpy() + bias.numpy()
    assert torch.equal(run_linear(lib, q, scale, weight, w_scale, bias, torch.float32), torch.from_numpy(want))
    code = torch.empty((tokens, channels), dtype=torch.uint8, device="cuda")
    lib.linear_codes(q.cuda(), scale.cuda(), lib.pack_weights(weight.cuda()), w_scale.cuda(), code, 8, -300.0, 250.0, bias=bias.cuda())
    lib.sync_status()
    assert np.array_equal(code.cpu().numpy(), U.codes(want, 8, -300.0, 250.0))


@pytest.mark.parametrize("tokens", [1, 13, 90])
def test_linear_codes_of_values_without_a_number(lib, tokens):
    q, weight = U.int8(1, tokens, 64), U.int8(2, 40, 64)
    scale = torch.full((tokens,), math.nan)
    code = torch.empty((tokens, 40), dtype=torch.uint8, device="cuda")
    w = lib.pack_weights(weight.cuda())
    lib.linear_codes(q.cuda(), scale.cuda(), w, torch.ones(40, device="cuda"), code, 4, -1.0, 1.0)
    lib.sync_status()
    assert not code.any()
    lib.linear_codes(q.cuda(), torch.full((tokens,), 3e38, device="cuda"), w, torch.full((40,), 3e38, device="cuda"), code, 4, -1.0, 1.0)
    lib.sync_status()
    acc = q.numpy().astype(np.int64) @ weight.numpy().astype(np.int64).T
    assert np.array_equal(code.cpu().numpy(), np.where(acc > 0, 15, np.where(acc < 0, 0, 8)).astype(np.uint8))


@pytest.mark.parametrize("tokens", [2, 33, 300])
def test_linear_wider_rows(lib, tokens):
    """Slices of wider buffers at odd offsets; what lies beside the output stays."""
    q = U.int8(1, tokens, 150)[:, 3:136]
    weight = U.int8(2, 70, 150)[:, 5:138]
    scale, w_scale = U.rand(3, tokens).abs(), U.rand(4, 70)
    qd, wd = U.int8(1, tokens, 150).cuda()[:, 3:136], U.int8(2, 70, 150).cuda()[:, 5:138]
    out = torch.full((tokens, 80), 7.0, dtype=torch.bfloat16, device="cuda")
    lib.linear(qd, scale.cuda(), lib.pack_weights(wd), w_scale.cuda(), out[:, 3:73])
    lib.sync_status()
    want = torch.from_numpy(U.linear(q, scale, weight, w_scale, None)).to(torch.bfloat16)
    assert torch.equal(out[:, 3:73].cpu(), want)
    assert bool((out[:, :3] == 7).all()) and bool((out[:, 73:] == 7).all())


def test_linear_refuses(lib):
    from paper_2609_16915_gb300 import RosettaError
    q, s = torch.ones(4, 64, dtype=torch.int8, device="cuda"), torch.ones(4, device="cuda")
    w, ws = lib.pack_weights(torch.ones(32, 64, dtype=torch.int8, device="cuda")), torch.ones(32, device="cuda")
    out, code = torch.empty(4, 32, device="cuda"), torch.empty(4, 32, dtype=torch.uint8, device="cuda")
    for bad in [dict(q=q[:, :63]), dict(scale=s[:3]), dict(weights=w.data), dict(w_scale=ws.half()), dict(out=out[:3]),
                dict(out=out.double()), dict(bias=ws[:5]), dict(q=q.cpu())]:
        with pytest.raises(ValueError):
            lib.linear(**{**dict(q=q, scale=s, weights=w, w_scale=ws, out=out), **bad})
    base = dict(q=q, scale=s, weights=w, w_scale=ws, code=code, bits=4, lo=0.0, hi=1.0)
    for bad in [dict(bits=0), dict(bits=9), dict(lo=1.0), dict(hi=math.inf), dict(lo=math.nan), dict(lo=0.0, hi=1e-45)]:
        with pytest.raises(RosettaError) as e:
            lib.linear_codes(**{**base, **bad})
        assert e.value.status == -1
    with pytest.raises(ValueError):
        lib.linear_codes(**base, table=torch.ones(16, dtype=torch.int8, device="cuda"))
    with pytest.raises(RosettaError):       # the output over the activations
        lib.linear_codes(**{**base, "q": code.view(torch.int8), "weights": lib.pack_weights(torch.ones(32, 32, dtype=torch.int8, device="cuda"))})
    with pytest.raises(ValueError):
        lib.pack_weights(torch.ones(4, 131072, dtype=torch.int8, device="cuda"))
    lib.linear(q[:0], s[:0], w, ws, out[:0])
    lib.sync_status()


# ------------------------------------------------------------------ cache


def make_cache(seed, lens, page, heads, dim, extra=2, spare=0):
    """Random caches, scales and a shuffled page table for sequences of these lengths."""
    each = max(1, -(-max(lens) // page)) + spare
    pages = len(lens) * each + extra
    g = torch.Generator().manual_seed(seed)
    table = torch.randperm(pages, generator=g)[:len(lens) * each].reshape(len(lens), each).to(torch.int32)
    c = [U.int8(seed + i, pages, heads, page, dim) for i in (1, 2)]
    s = [(0.5 + torch.rand((pages, heads), generator=g)) / 60 for _ in range(2)]
    return c, s, table


APPENDS = [  # firsts, new, page, heads, dim
    ([0, 5, 15, 16, 31], 1, 16, 2, 64), ([0, 3, -1, 40], 17, 16, 3, 128), ([7, 0], 100, 32, 1, 96), ([0, 1, 2], 5, 1, 2, 4),
    ([9, 33], 2, 24, 2, 20), ([0, 100], 200, 128, 2, 256), ([1000], 3, 1024, 1, 64)]


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("firsts,new,page,heads,dim", APPENDS)
def test_append(lib, dtype, firsts, new, page, heads, dim):
    c, s, table = make_cache(7, [max(f, 0) + new for f in firsts], page, heads, dim)
    qkv = (2 * U.rand(3, len(firsts), new, 2 * heads, dim)).to(dtype)
    qkv[0, 0, 0] *= 5       # the scale grows where rows are there already
    k, v = qkv[:, :, :heads], qkv[:, :, heads:]
    dev = [t.cuda() for t in (*c, *s)]
    first = torch.tensor(firsts, dtype=torch.int32)
    big = qkv.cuda()
    for _ in range(2):      # again over itself: the same
        lib.cache_append(big[:, :, :heads], big[:, :, heads:], *dev, table.cuda(), first.cuda())
        lib.sync_status()
        for i, x in enumerate((k, v)):
            want, scale = U.append(x, c[i], s[i], table, first)
            assert torch.equal(dev[2 + i].cpu(), scale)
            assert torch.equal(dev[i].cpu(), want)


def test_append_zeros_and_values_without_a_number(lib):
    c, s, table = make_cache(7, [20, 20, 20], 16, 1, 64)
    x = U.rand(1, 3, 20, 1, 64)
    x[0] = 0
    x[1, 2, 0, 5] = math.nan
    x[2, 18, 0, 63] = -math.inf
    dev = [t.cuda() for t in (*c, *s)]
    first = torch.zeros(3, dtype=torch.int32)
    lib.cache_append(x.cuda(), x.cuda(), *dev, table.cuda(), first.cuda())
    lib.sync_status()
    for i in range(2):
        want, scale = U.append(x, c[i], s[i], table, first)
        got, t = dev[2 + i].cpu(), table.long()
        assert got[t[0, 0]] == 0 and not dev[i].cpu()[t[0, 0]].any()
        assert torch.isnan(got[t[1, 0]]) and torch.isnan(got[t[2, 1]])
        for p in (t[0, 0], t[0, 1], t[1, 1], t[2, 0]):
            assert torch.equal(got[p], scale[p]) and torch.equal(dev[i].cpu()[p], want[p])
    # appending behind rows under a NaN scale keeps it
    lib.cache_append(x[1:2, :1].cuda(), x[1:2, :1].cuda(), *dev, table[1:2].cuda(), torch.tensor([9], dtype=torch.int32).cuda())
    lib.sync_status()
    assert torch.isnan(dev[2].cpu()[table[1, 0].long()])


def test_append_skips_pages_out_of_range(lib):
    from paper_2609_16915_gb300 import RosettaError
    c, s, table = make_cache(7, [40, 40], 16, 2, 64)
    x = U.rand(1, 2, 40, 2, 64)
    bad = table.clone()
    bad[0, 1], bad[1, 0] = c[0].shape[0], -1
    dev = [t.cuda() for t in (*c, *s)]
    lib.cache_append(x.cuda(), x.cuda(), *dev, bad.cuda(), torch.zeros(2, dtype=torch.int32).cuda())
    with pytest.raises(RosettaError) as e:
        lib.sync_status()
    assert e.value.status == -1
    lib.sync_status()       # reported once
    want, scale = U.append(x, c[0], s[0], table, [0, 0])
    for b in range(2):
        for slot in range(3):
            p = table[b, slot].long()
            skipped = (b, slot) in ((0, 1), (1, 0))
            assert torch.equal(dev[0].cpu()[p], c[0][p] if skipped else want[p])
    # past the page list
    dev = [t.cuda() for t in (*c, *s)]
    lib.cache_append(x.cuda(), x.cuda(), *dev, table.cuda(), torch.tensor([20, -1], dtype=torch.int32).cuda())
    with pytest.raises(RosettaError):
        lib.sync_status()


def check_attention(lib, dtype, lens, new, page, heads, group, dim, scale=None, seed=5, stretch=1.0):
    c, s, table = make_cache(seed, lens, page, heads, dim)
    wide = (stretch * U.rand(seed + 9, len(lens), new, heads * group + 1, dim)).to(dtype)
    q = wide[:, :, :heads * group]
    lengths = torch.tensor(lens, dtype=torch.int32)
    sc = dim ** -0.5 if scale is None else scale
    out = torch.full((len(lens), new, heads * group, dim), 9.0, dtype=dtype, device="cuda")
    lib.attention(wide.cuda()[:, :, :heads * group], *[t.cuda() for t in (*c, *s)], table.cuda(), lengths.cuda(), out, scale)
    lib.sync_status()
    want, size = U.attention(q, *c, *s, table, lengths, sc)
    # the output's rounding, and errors of the weights: rounded to 11 bits for the product with V (22 in
    # single precision), scores in single precision
    weights = 2.0 ** -16 if dtype == torch.float32 else 2.0 ** -10
    err = (out.cpu().double() - want).abs()
    bound = 1.01 * U.UNIT[dtype] * want.abs() + weights * size + 1e-9
    assert torch.all(err <= bound), float((err - bound).max())
    return out


ATTENDS = [  # lens, new, page, heads, group, dim
    ([1], 1, 16, 1, 1, 64), ([77], 1, 16, 12, 1, 64), ([0, 1, 2, 15, 16, 17, 33], 1, 16, 2, 4, 128),
    ([100, 3000, 1, 517], 1, 32, 2, 8, 128), ([5, 2, 0, 64], 7, 16, 3, 2, 96), ([200, 130], 130, 64, 2, 3, 64),
    ([31, 300], 33, 128, 1, 8, 128), ([40, 77], 5, 24, 2, 2, 64), ([19, 50], 3, 1, 1, 7, 80), ([300], 20, 16, 1, 16, 256),
    ([129], 2, 16, 1, 128, 128), ([260, 4], 40, 32, 5, 1, 20), ([2000], 64, 16, 1, 4, 128), ([70, 700], 1, 1024, 2, 4, 4),
    ([600, 9], 257, 32, 1, 4, 96), ([1300], 150, 128, 1, 2, 256)]


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("lens,new,page,heads,group,dim", ATTENDS)
def test_attention(lib, dtype, lens, new, page, heads, group, dim):
    check_attention(lib, dtype, lens, new, page, heads, group, dim)


@pytest.mark.parametrize("dtype", FLOATS)
@pytest.mark.parametrize("new", [1, 40])
def test_attention_scales(lib, dtype, new):
    check_attention(lib, dtype, [200, 90], new, 16, 2, 4, 128, scale=0.0)
    check_attention(lib, dtype, [200, 90], new, 16, 2, 4, 128, scale=-0.05)
    check_attention(lib, dtype, [200, 90], new, 16, 2, 4, 64, stretch=200.0, scale=1e-4)
    check_attention(lib, dtype, [200, 90], new, 16, 2, 4, 64, stretch=1e-6, scale=1e4)


@pytest.mark.parametrize("new", [1, 50])
def test_attention_rows_without_a_position(lib, new):
    out = check_attention(lib, torch.bfloat16, [0, 3, new], new, 16, 2, 4, 64)
    assert not out[0].any()


@pytest.mark.parametrize("new", [1, 40])
def test_attention_scales_of_pages_far_apart(lib, new):
    """Pages whose values differ by many powers of two, and pages of zeros."""
    lens, page, heads, dim = [150, 64], 16, 2, 64
    c, s, table = make_cache(3, lens, page, heads, dim)
    s[1] *= 2.0 ** (torch.arange(s[1].numel()) % 23 - 11).reshape(s[1].shape)
    s[1][table[0, 2].long()] = 0
    s[0][table[0, 4].long()] = 0
    q = U.rand(4, 2, new, 8, dim)
    out = torch.empty_like(q, device="cuda")
    lengths = torch.tensor(lens, dtype=torch.int32)
    lib.attention(q.cuda(), *[t.cuda() for t in (*c, *s)], table.cuda(), lengths.cuda(), out)
    lib.sync_status()
    want, size = U.attention(q, *c, *s, table, lengths, dim ** -0.5)
    assert torch.all((out.cpu().double() - want).abs() <= 2.0 ** -16 * size + 1e-9)


@pytest.mark.parametrize("new", [1, 24])
@pytest.mark.parametrize("dim", [64, 128, 20])
def test_attention_never_reads_what_is_masked(lib, new, dim):
    """NaN scales in pages beyond the lengths, other sequences' pages and unused table entries change nothing."""
    lens, page, heads = [40, 17], 16, 2
    c, s, table = make_cache(3, lens, page, heads, dim, spare=3)
    q = U.rand(4, 2, new, 4, dim).to(torch.float16)
    lengths = torch.tensor(lens, dtype=torch.int32)
    outs = []
    for poison in (False, True):
        if poison:
            used = {int(p) for b in range(2) for p in table[b, :-(-lens[b] // page)]}
            for p in range(c[0].shape[0]):
                if p not in used:
                    s[0][p], s[1][p] = math.nan, math.inf
                    c[0][p], c[1][p] = -128, 127
            # the rows after a sequence's end, in its last page
            for b in range(2):
                p = table[b, (lens[b] - 1) // page].long()
                c[0][p, :, lens[b] % page:], c[1][p, :, lens[b] % page:] = 127, -128
            table = table.clone()
            table[:, -3:] = 1 << 30
        out = torch.empty_like(q, device="cuda")
        lib.attention(q.cuda(), *[t.cuda() for t in (*c, *s)], table.cuda(), lengths.cuda(), out)
        lib.sync_status()
        outs.append(out.cpu())
    assert torch.equal(outs[0], outs[1])


@pytest.mark.parametrize("new", [1, 20])
@pytest.mark.parametrize("dim", [64, 20])
def test_attention_pages_out_of_range_are_masked_and_reported(lib, new, dim):
    from paper_2609_16915_gb300 import RosettaError
    c, s, table = make_cache(3, [90], 16, 2, dim)
    q = U.rand(4, 1, new, 4, dim)
    bad = table.clone()
    bad[0, 2], bad[0, 4] = c[0].shape[0], -7
    out = torch.empty_like(q, device="cuda")
    dev = [t.cuda() for t in (*c, *s)]
    lib.attention(q.cuda(), *dev, bad.cuda(), torch.tensor([90], dtype=torch.int32).cuda(), out)
    with pytest.raises(RosettaError) as e:
        lib.sync_status()
    assert e.value.status == -1
    k = (c[0][table[0].long()].double() * s[0][table[0].long()].double()[:, :, None, None]).permute(1, 0, 2, 3).flatten(1, 2)
    v = (c[1][table[0].long()].double() * s[1][table[0].long()].double()[:, :, None, None]).permute(1, 0, 2, 3).flatten(1, 2)
    for t in range(new):
        for h in range(4):
            at = [p for p in range(90 - new + t + 1) if p // 16 not in (2, 4)]
            p = torch.softmax(k[h // 2, at] @ q[0, t, h].double() * dim ** -0.5, 0)
            want, size = p @ v[h // 2, at], p @ v[h // 2, at].abs()
            assert torch.all((out[0, t, h].cpu().double() - want).abs() <= 2.0 ** -16 * size + 1e-9)
    # a length past the page list counts as the list's end
    lib.attention(q.cuda(), *dev, table.cuda(), torch.tensor([5000], dtype=torch.int32).cuda(), out)
    with pytest.raises(RosettaError):
        lib.sync_status()
    want, size = U.attention(q, *c, *s, table, [5000], dim ** -0.5)
    assert torch.all((out.cpu().double() - want).abs() <= 2.0 ** -16 * size + 1e-9)


def test_attention_and_append_beyond_32_bits(lib):
    """A cache of over 4 GiB, with the pages that are used at its end."""
    pages, heads, page, dim = 70000, 8, 64, 128
    kc = torch.zeros((pages, heads, page, dim), dtype=torch.int8, device="cuda")
    vc = torch.zeros_like(kc)
    ks, vs = torch.zeros((pages, heads), device="cuda"), torch.zeros((pages, heads), device="cuda")
    table = torch.tensor([[pages - 1, 69000, 40000]], dtype=torch.int32)
    x = U.rand(1, 1, 150, heads, dim).half()
    lib.cache_append(x.cuda(), (2 * x).cuda(), kc, vc, ks, vs, table.cuda(), torch.zeros(1, dtype=torch.int32).cuda())
    lib.sync_status()
    at = table[0].long()
    k0 = torch.zeros((3, heads, page, dim), dtype=torch.int8)
    want, scale = U.append(x, k0, torch.zeros(3, heads), torch.tensor([[0, 1, 2]]), [0])
    assert torch.equal(kc[at.cuda()].cpu(), want) and torch.equal(ks[at.cuda()].cpu(), scale)
    for new in (1, 30):
        q = U.rand(2, 1, new, 16, dim).half()
        out = torch.empty_like(q, device="cuda")
        lib.attention(q.cuda(), kc, vc, ks, vs, table.cuda(), torch.tensor([150], dtype=torch.int32).cuda(), out)
        lib.sync_status()
        ref, size = U.attention(q, want, vc[at.cuda()].cpu(), scale, vs[at.cuda()].cpu(), torch.tensor([[0, 1, 2]]), [150], dim ** -0.5)
        assert torch.all((out.cpu().double() - ref).abs() <= U.UNIT[q.dtype] * ref.abs() + 2.0 ** -10 * size + 1e-9)


@pytest.mark.parametrize("group", [4, 50])
@pytest.mark.parametrize("dtype,context", [(torch.float32, 1 << 16), (torch.float32, 1 << 19), (torch.float16, 1 << 19)])
def test_attention_of_long_contexts(lib, dtype, context, group):
    """Page lists that repeat 2048 positions, values of one sign: what sums lose as they grow would show.  Single precision within
    2^-18 of the sum (products in 22 bits, and 512 positions to an accumulator that is cut off at 24), f16 as over short contexts."""
    batch, pages, page, dim = 160, 32, 64, 128
    kc, vc = U.int8(5, pages, 1, page, dim), U.int8(6, pages, 1, page, dim, lo=1)
    ks, vs = torch.rand(pages, 1, generator=torch.Generator().manual_seed(7)) / 60, torch.rand(pages, 1, generator=torch.Generator().manual_seed(8)) / 60
    q = U.rand(9, 1, 1, group, dim).to(dtype)
    each = context // page
    table = (torch.arange(each) * 7 % pages).to(torch.int32)
    out = torch.empty((batch, 1, group, dim), dtype=dtype, device="cuda")
    lib.attention(q.cuda().expand(batch, -1, -1, -1).contiguous(), kc.cuda(), vc.cuda(), ks.cuda(), vs.cuda(),
                  table.cuda().expand(batch, -1).contiguous(), torch.full((batch,), context, dtype=torch.int32, device="cuda"), out)
    lib.sync_status()
    want, size = U.attention(q, kc, vc, ks, vs, torch.arange(pages, dtype=torch.int32)[None], [pages * page], dim ** -0.5)
    bound = 2.0 ** -18 * size if dtype == torch.float32 else U.UNIT[dtype] * want.abs() + 2.0 ** -10 * size
    assert torch.all((out.cpu().double() - want).abs() <= bound)


def test_cache_of_other_orders(lib):
    """Caches stored [page][row][head][dim], and with gaps."""
    lens, page, heads, dim = [50, 33], 16, 3, 64
    c, s, table = make_cache(3, lens, page, heads, dim)
    for form in ("rows first", "gaps"):
        dev = []
        for x in c:
            if form == "rows first":
                dev.append(x.permute(0, 2, 1, 3).contiguous().cuda().permute(0, 2, 1, 3))
            else:
                big = torch.zeros((x.shape[0], heads, page, dim + 4), dtype=torch.int8, device="cuda")
                big[..., :dim] = x.cuda()
                dev.append(big[..., :dim])
        sd = [t.cuda() for t in s]
        x = U.rand(1, 2, 3, heads, dim)
        first = torch.tensor([n - 3 for n in lens], dtype=torch.int32)
        lib.cache_append(x.cuda(), x.cuda(), *dev, *sd, table.cuda(), first.cuda())
        after = [U.append(x, c[i], s[i], table, first) for i in range(2)]
        for new in (1, 20):
            q = U.rand(4, 2, new, 2 * heads, dim)
            out = torch.empty_like(q, device="cuda")
            lengths = torch.tensor(lens, dtype=torch.int32)
            lib.attention(q.cuda(), *dev, *sd, table.cuda(), lengths.cuda(), out)
            lib.sync_status()
            for i in range(2):
                assert torch.equal(dev[i].cpu(), after[i][0]) and torch.equal(sd[i].cpu(), after[i][1])
            want, size = U.attention(q, after[0][0], after[1][0], after[0][1], after[1][1], table, lengths, dim ** -0.5)
            assert torch.all((out.cpu().double() - want).abs() <= 2.0 ** -16 * size + 1e-9)


def test_cache_refuses(lib):
    from paper_2609_16915_gb300 import RosettaError
    c, s, table = make_cache(3, [40, 30], 16, 2, 64)
    kc, vc, ks, vs = [t.cuda() for t in (*c, *s)]
    table, n = table.cuda(), torch.tensor([40, 30], dtype=torch.int32).cuda()
    q = torch.randn(2, 1, 4, 64, device="cuda")
    base = dict(q=q, k_cache=kc, v_cache=vc, k_scale=ks, v_scale=vs, page_table=table, lengths=n, out=torch.empty_like(q))
    for bad in [dict(q=q[..., :60]), dict(q=q[:, :, :3]), dict(k_cache=kc.float()), dict(v_cache=vc[:-1]), dict(k_scale=ks[:, :1]),
                dict(page_table=table.long()), dict(page_table=table[:1]), dict(lengths=n[:1]), dict(lengths=n.long()),
                dict(out=q.half()), dict(q=q.double()), dict(page_table=table.cpu()), dict(v_cache=vc.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3))]:
        with pytest.raises(ValueError):
            lib.attention(**{**base, **bad})
    for bad in [dict(softmax_scale=math.inf), dict(softmax_scale=math.nan), dict(out=q)]:
        with pytest.raises(RosettaError) as e:
            lib.attention(**{**base, **bad})
        assert e.value.status == -1
    k = torch.randn(2, 3, 2, 64, device="cuda")
    base = dict(k=k, v=k, k_cache=kc, v_cache=vc, k_scale=ks, v_scale=vs, page_table=table, first=n)
    for bad in [dict(v=k.half()), dict(k=k[:, :, :1], v=k[:, :, :1]), dict(first=n.long()), dict(v=k[:, :2])]:
        with pytest.raises(ValueError):
            lib.cache_append(**{**base, **bad})
    odd = torch.zeros(5, 2, 16, 6, dtype=torch.int8, device="cuda")     # a head of 6
    with pytest.raises(RosettaError):
        lib.cache_append(k[..., :6].contiguous(), k[..., :6].contiguous(), odd, odd.clone(), ks[:5], vs[:5], table, n)
    lib.attention(**{**base_empty(base, q), "lengths": n[:0]})
    lib.sync_status()


def base_empty(base, q):
    return dict(q=q[:0], k_cache=base["k_cache"], v_cache=base["v_cache"], k_scale=base["k_scale"], v_scale=base["v_scale"],
                page_table=base["page_table"][:0], out=torch.empty_like(q[:0]))


# ------------------------------------------------------------------ streams and graphs


def layer(lib, t, stream=None):
    """norm -> linear -> codes, append, attention on one stream, into t's buffers."""
    lib.norm(t["x"], t["gamma"], t["q"], t["scale"], stream=stream)
    lib.linear(t["q"], t["scale"], t["w"], t["w_scale"], t["qkv"], stream=stream)
    qkv = t["qkv"].view(t["batch"], -1, 4 + 2 + 2, 64)
    lib.cache_append(qkv[:, :, 4:6], qkv[:, :, 6:], *t["cache"], t["table"], t["first"], stream=stream)
    lib.attention(qkv[:, :, :4], *t["cache"], t["table"], t["lengths"], t["out"], stream=stream)


def layer_state(tokens):
    lens = [90, 41]
    c, s, table = make_cache(3, lens, 16, 2, 64)
    n = torch.tensor(lens, dtype=torch.int32).cuda()
    rows = 2 * tokens
    return dict(x=U.rand(1, rows, 256).cuda(), gamma=torch.ones(256, device="cuda"), batch=2,
                q=torch.empty(rows, 256, dtype=torch.int8, device="cuda"), scale=torch.empty(rows, device="cuda"),
                w_scale=torch.full((512,), 0.002, device="cuda"), qkv=torch.empty(rows, 512, dtype=torch.float16, device="cuda"),
                cache=[t.cuda() for t in (*c, *s)], table=table.cuda(), lengths=n, first=n - tokens,
                out=torch.empty(2, tokens, 4, 64, dtype=torch.float16, device="cuda"))


@pytest.mark.parametrize("tokens", [1, 40])
def test_other_streams_and_graphs(lib, tokens):
    weight = U.int8(2, 512, 256).cuda()
    a = layer_state(tokens)
    a["w"] = lib.pack_weights(weight)
    layer(lib, a)
    lib.sync_status()
    want = a["out"].clone()
    assert bool(want.isfinite().all()) and bool(want.any())
    side = torch.cuda.Stream()
    b = layer_state(tokens)
    b["w"] = a["w"]
    torch.cuda.synchronize()
    layer(lib, b, stream=side)
    lib.sync_status(side)
    assert torch.equal(b["out"], want)
    c = layer_state(tokens)
    c["w"] = a["w"]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(lib, c)
    graph.replay()
    graph.replay()          # appending the same tokens again changes nothing
    lib.sync_status()
    assert torch.equal(c["out"], want)
    # a larger call outgrows the workspace; the graph still holds its own
    big = torch.ones(3000, 2000, dtype=torch.int8, device="cuda")
    lib.linear(big, torch.ones(3000, device="cuda"), lib.pack_weights(big), torch.ones(3000, device="cuda"),
               torch.empty(3000, 3000, device="cuda"))
    c["out"].zero_()
    graph.replay()
    lib.sync_status()
    assert torch.equal(c["out"], want)
