"""The decoder layer in the clear, whole: its steps against the definitions, prompts against
token by token, and its table against the same table bootstrapped under encryption."""

import numpy as np
import pytest
import torch

from tests import clear_util as U

pytestmark = pytest.mark.gpu

WIDTH, INNER, HEADS, KV, DIM = 128, 192, 4, 2, 64


def make_layer(bits, lo=-3.0, hi=3.0):
    from paper_2609_16915_gb300 import clear_layer as L
    weights = L.random_weights(WIDTH, INNER, HEADS, KV, DIM, seed=3)
    codes, y_lo, y_hi = L.gelu_codes(bits, lo, hi)
    table, scale = L.value_table(codes, bits, y_lo, y_hi)
    return L, weights, L.Layer(weights, HEADS, KV, DIM, bits, lo, hi, table, scale), codes


def tokens(batch, n, seed):
    return (U.rand(seed, batch, n, WIDTH).to(torch.bfloat16).cuda(), U.rand(seed + 1, batch, n, WIDTH).to(torch.bfloat16).cuda())


def test_codes_are_those_of_the_definitions():
    """The up projection's codes and the down projection follow from the layer's 8-bit input exactly."""
    L, weights, layer, _ = make_layer(5)
    x, r = tokens(2, 40, 7)
    cache = L.Cache(2, 64, KV, DIM)
    y, code = layer.step(x, r.clone(), cache)
    again = L.Cache(2, 64, KV, DIM)
    q, s = layer.before_table(x, r.clone(), again)
    layer.lib.sync_status()
    for a, b in zip(cache.tensors(), again.tensors()):
        assert torch.equal(a, b)
    up, up_scale = (t.cpu() for t in L.quantise_channels(weights["up"]))
    want = U.codes(U.linear(q.cpu(), s.cpu(), up, up_scale, weights["up_bias"].cpu()), 5, -3.0, 3.0)
    assert np.array_equal(code.cpu().numpy(), want)
    values = layer.table.cpu()[torch.from_numpy(want).long()]
    down, down_scale = (t.cpu() for t in L.quantise_channels(weights["down"]))
    want_y = U.linear(values, torch.full((80,), layer.table_scale), down, down_scale, None)
    assert torch.equal(y.cpu().reshape(80, WIDTH), torch.from_numpy(want_y).to(torch.bfloat16))


def test_whole_layer_against_64_bits():
    """The layer's 8-bit rounding aside, its up projection follows the float layer: the mean code differs little."""
    L, weights, layer, _ = make_layer(6)
    x, r = tokens(2, 70, 11)
    q, s = layer.before_table(x, r.clone(), L.Cache(2, 70, KV, DIM))
    layer.lib.sync_status()
    w = {k: v.double().cpu() for k, v in weights.items()}

    def norm(v):
        return v / torch.sqrt((v * v).mean(-1, keepdim=True) + L.EPS)

    h = x.double().cpu() + r.double().cpu()
    qkv = (norm(h) @ w["qkv"].T).reshape(2, 70, HEADS + 2 * KV, DIM)
    out = torch.zeros(2, 70, HEADS, DIM, dtype=torch.float64)
    for b in range(2):
        for i in range(HEADS):
            k, v = qkv[b, :, HEADS + i // 2], qkv[b, :, HEADS + KV + i // 2]
            z = (qkv[b, :, i] @ k.T * DIM ** -0.5).masked_fill(torch.ones(70, 70).triu(1).bool(), -np.inf)
            out[b, :, i] = torch.softmax(z, 1) @ v
    h = h + norm(out.reshape(2, 70, -1)) @ w["o"].T
    want = norm(h).reshape(140, WIDTH)
    got = q.cpu().double() * s.cpu().double()[:, None]
    # 8-bit activations, weights, keys and values of 1 / 127 of their largest: a few per cent of the rms
    assert float((got - want).norm() / want.norm()) < 0.06


def test_prompt_and_single_tokens_agree():
    """Token by token, the cache's scales grow and its old bytes are rounded again: the same within that."""
    L, _, layer, _ = make_layer(6)
    x, r = tokens(2, 24, 5)
    r1, r2 = r.clone(), r.clone()
    q1, s1 = layer.before_table(x, r1, L.Cache(2, 32, KV, DIM, page=16))
    cache, parts = L.Cache(2, 32, KV, DIM, page=16), []
    for i in range(24):
        ri = r2[:, i:i + 1].contiguous()
        q, s = layer.before_table(x[:, i:i + 1], ri, cache)
        parts.append(q.float() * s[:, None])
    layer.lib.sync_status()
    one = (q1.float() * s1[:, None]).reshape(2, 24, WIDTH)
    many = torch.stack(parts, 1)
    assert cache.lengths.tolist() == [24, 24]
    assert float((one - many).norm() / one.norm()) < 0.06


def test_table_in_the_clear_is_the_bootstrapped_one():
    """code -> encrypt -> pbs_batch -> decrypt gives the LUT's output codes, whose values are the layer's."""
    import oracle as O
    import paper_2609_16915_gb300 as R
    import workload as W
    bits = 3
    L, _, layer, codes = make_layer(bits)
    x, r = tokens(1, 2, 21)
    y, code = layer.step(x, r, L.Cache(1, 8, KV, DIM))
    layer.lib.sync_status()
    p = W.CONFIGS["tiny"]
    assert p.msg_bits == bits
    keys = O.Keys(p, W.key_draws(p))
    flat = code.cpu().numpy().reshape(-1)[:64].astype(np.int64)
    assert len(set(flat.tolist())) > 4
    lwe = keys.encrypt(W.cipher_draws(p, flat.size, sub=9, codes=flat))

    def dev(a):
        return torch.from_numpy(np.ascontiguousarray(a).view(np.int64)).cuda()

    ctx = R.Context(p)
    ctx.upload_bsk(dev(keys.bsk))
    ctx.upload_ksk(dev(keys.ksk))
    out = torch.empty((flat.size, p.n + 1), dtype=torch.int64, device="cuda")
    ctx.pbs_batch(dev(lwe), dev(W.lut_torus(p, codes)), out)
    ctx.sync_status()
    got = keys.decrypt(out.cpu().numpy().view(np.uint64))
    assert np.array_equal(got, np.asarray(codes)[flat])
    top = (1 << bits) - 1
    _, y_lo, y_hi = L.gelu_codes(bits, -3.0, 3.0)
    values = [round((y_lo + int(c) / top * (y_hi - y_lo)) / layer.table_scale) for c in got]
    assert values == layer.table[code.reshape(-1)[:64].long()].tolist()


def test_calibration_covers_the_inputs():
    L, weights, layer, _ = make_layer(6)
    x, r = tokens(2, 64, 31)
    lo, hi = layer.calibrate(x, r.clone(), L.Cache(2, 64, KV, DIM), cut=0.0)
    _, code = layer.step(x, r.clone(), L.Cache(2, 64, KV, DIM))
    layer.lib.sync_status()
    assert lo < -1 < 1 < hi
    assert int(code.min()) == 0 and int(code.max()) == 63


def test_the_command_runs(capsys):
    from paper_2609_16915_gb300 import clear_layer
    clear_layer.main()
    text = capsys.readouterr().out
    assert "calibrated range" in text and "decode" in text
