"""A decoder layer in the clear around a bootstrapped table.

What it is for: the range [lo, hi] of the table that rosetta_pbs_batch evaluates is
calibrated, and the precision of its p-bit codes judged, by running the layer with the same
table in place, without encryption; and the codes that the layer's up projection gives are
the messages that are encrypted.  One step of the layer:

  h = x + residual;  a = attention(norm(h) W_qkv) over the 8-bit cache, the new tokens among it
  h = h + norm(a) W_o
  code = message codes of norm(h) W_up + b_up on [lo, hi];  y = table[code] W_down

It is a layer of a decoder's shape from those operators, not one of a named model: a root-mean-square
norm stands before every product (the attention's output among them), there are no position
embeddings, no gate beside the table and no biases but the table's, so a range calibrated on it is
its own, and a model's layer is put together from the same calls where they fit it.

Norms, products, cache and table values are 8-bit (clear.Clear); the residual stream is
bfloat16.  The encrypted path replaces the table alone: encrypt(code) -> pbs_batch ->
decrypt gives lut[code], and value_table() turns those output codes into the same 8-bit
values.

    python -m paper_2609_16915_gb300.clear_layer        # random weights: calibrate, prompt, decode, timings
"""

from __future__ import annotations

import math

import torch

from .clear import Clear

EPS = 1e-5


def quantise_channels(weight):
    """(int8 [channels][inner], scale [channels]) of float weights, a scale per channel."""
    scale = weight.float().abs().amax(1).clamp_min(1e-12) / 127
    return torch.round(weight.float() / scale[:, None]).to(torch.int8), scale


def value_table(out_codes, bits: int, y_lo: float, y_hi: float, device="cuda"):
    """The 8-bit values [2^bits] of a LUT's output codes (0 .. 2^bits - 1 spread over [y_lo, y_hi]), and their scale."""
    top = (1 << bits) - 1
    scale = max(abs(y_lo), abs(y_hi)) / 127
    y = [y_lo + int(c) / top * (y_hi - y_lo) for c in out_codes]
    return torch.tensor([round(v / scale) for v in y], dtype=torch.int8, device=device), scale


class Cache:
    """Pages for `batch` sequences of up to `context` positions: sequence b has pages b * each .."""

    def __init__(self, batch, context, heads, dim, page=32, device="cuda"):
        each = -(-context // page)
        shape = (batch * each, heads, page, dim)
        self.k, self.v = (torch.zeros(shape, dtype=torch.int8, device=device) for _ in range(2))
        self.k_scale, self.v_scale = (torch.zeros(shape[:2], device=device) for _ in range(2))
        self.pages = torch.arange(batch * each, dtype=torch.int32, device=device).reshape(batch, each)
        self.lengths = torch.zeros(batch, dtype=torch.int32, device=device)
        self.room = self.most = each * page     # positions; how many every sequence has left at least

    def take(self, tokens):
        """Room for `tokens` more positions of every sequence, or ValueError.  `lengths` is on the device and may be lowered there:
        it is read only where the tokens taken so far would not leave room.  (What the device alone knows to be too long, a
        length that was raised there or a graph replayed too often, Clear.sync_status reports.)"""
        if tokens > self.room:
            self.room = self.most - int(self.lengths.max())
        if tokens > self.room:
            raise ValueError(f"the cache holds {self.most} positions of a sequence: no room for {tokens} more")
        self.room -= tokens

    def tensors(self):
        return self.k, self.v, self.k_scale, self.v_scale, self.pages


class Layer:
    """weights: floats qkv [(heads + 2 kv_heads) dim][width], o [width][heads dim], up [inner][width], down [width][inner]."""

    def __init__(self, weights, heads: int, kv_heads: int, dim: int, bits: int, lo: float, hi: float, table, table_scale: float,
                 lib: Clear | None = None):
        self.lib = lib or Clear()
        self.heads, self.kv_heads, self.dim, self.bits = heads, kv_heads, dim, bits
        self.lo, self.hi, self.table = lo, hi, table
        self.packed, self.scales = {}, {}
        for name in ("qkv", "o", "up", "down"):
            q, self.scales[name] = quantise_channels(weights[name])
            self.packed[name] = self.lib.pack_weights(q)
        self.bias = weights.get("up_bias")
        width = weights["o"].shape[0]
        self.width, self.inner = width, weights["up"].shape[0]
        device = weights["o"].device
        self.gammas = {n: weights.get(n, torch.ones(w, device=device)) for n, w in
                       (("norm1", width), ("norm_a", heads * dim), ("norm2", width))}
        self.table_scale = table_scale

    def _norm(self, x, name, residual=None):
        """8-bit norm of x + residual; the sum goes back into residual."""
        q = torch.empty(x.shape, dtype=torch.int8, device=x.device)
        scale = torch.empty(x.shape[0], device=x.device)
        return self.lib.norm(x, self.gammas[name], q, scale, residual=residual, sum_out=residual, eps=EPS)

    def _linear(self, q, scale, name, bias=None):
        y = torch.empty((q.shape[0], self.packed[name].channels), dtype=torch.bfloat16, device=q.device)
        return self.lib.linear(q, scale, self.packed[name], self.scales[name], y, bias=bias)

    def before_table(self, x, residual, cache: Cache):
        """The 8-bit input of the up projection for new tokens x [batch][tokens][width]; residual and cache move on.
        ValueError, and neither moves, where the cache is full."""
        b, t, w = x.shape
        hq, hk, d = self.heads, self.kv_heads, self.dim
        cache.take(t)
        flat = residual.view(b * t, w)
        q, s = self._norm(x.reshape(b * t, w), "norm1", flat)
        qkv = self._linear(q, s, "qkv").view(b, t, hq + 2 * hk, d)
        self.lib.cache_append(qkv[:, :, hq:hq + hk], qkv[:, :, hq + hk:], *cache.tensors(), cache.lengths)
        cache.lengths += t
        a = torch.empty((b, t, hq, d), dtype=torch.bfloat16, device=x.device)
        self.lib.attention(qkv[:, :, :hq], *cache.tensors(), cache.lengths, a)
        q, s = self._norm(a.view(b * t, hq * d), "norm_a")
        return self._norm(self._linear(q, s, "o"), "norm2", flat)

    def calibrate(self, x, residual, cache: Cache, cut: float = 1e-4):
        """[lo, hi] of the table's input on these tokens, `cut` of the values off at each end."""
        q, s = self.before_table(x, residual, cache)
        y = self._linear(q, s, "up", self.bias).flatten().float().sort().values
        k = int(cut * y.numel())
        self.lo, self.hi = float(y[k]), float(y[-1 - k])
        return self.lo, self.hi

    def step(self, x, residual, cache: Cache):
        """(y [batch][tokens][width], message codes [batch * tokens][inner]) of new tokens."""
        b, t, w = x.shape
        q, s = self.before_table(x, residual, cache)
        code = torch.empty((b * t, self.inner), dtype=torch.uint8, device=x.device)
        value = torch.empty((b * t, self.inner), dtype=torch.int8, device=x.device)
        self.lib.linear_codes(q, s, self.packed["up"], self.scales["up"], code, self.bits, self.lo, self.hi, bias=self.bias,
                              table=self.table, values=value)
        scale = torch.full((b * t,), self.table_scale, device=x.device)
        return self._linear(value, scale, "down").view(b, t, w), code


def random_weights(width, inner, heads, kv_heads, dim, seed=0, device="cuda"):
    g = torch.Generator(device=device).manual_seed(seed)

    def w(n, k):
        return torch.randn((n, k), device=device, generator=g) / math.sqrt(k)

    return {"qkv": w((heads + 2 * kv_heads) * dim, width), "o": w(width, heads * dim), "up": w(inner, width),
            "down": w(width, inner), "up_bias": 0.1 * torch.randn(inner, device=device, generator=g)}


def gelu_codes(bits, lo, hi):
    """(output codes, y_lo, y_hi) of GELU on the midpoints of [lo, hi], over its own range."""
    size = 1 << bits
    ys = [x * 0.5 * (1 + math.erf(x / math.sqrt(2))) for x in (lo + (m + 0.5) * (hi - lo) / size for m in range(size))]
    y_lo, y_hi = min(ys), max(ys)
    return [min(max(math.floor((y - y_lo) / (y_hi - y_lo) * (size - 1) + 0.5), 0), size - 1) for y in ys], y_lo, y_hi


def main():
    width, inner, heads, dim, bits, batch, prompt = 768, 3072, 12, 64, 6, 8, 512    # GPT-2-small's layer
    weights = random_weights(width, inner, heads, heads, dim)
    g = torch.Generator(device="cuda").manual_seed(1)

    def tokens(n):
        return [torch.randn((batch, n, width), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2)]

    layer = Layer(weights, heads, heads, dim, bits, -4.0, 4.0, None, 1.0)
    lo, hi = layer.calibrate(*tokens(prompt), Cache(batch, prompt, heads, dim))
    codes, y_lo, y_hi = gelu_codes(bits, lo, hi)
    layer.table, layer.table_scale = value_table(codes, bits, y_lo, y_hi)
    print(f"calibrated range of the table's input: [{lo:.3f}, {hi:.3f}]")
    cache = Cache(batch, prompt + 64, heads, dim)
    events = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
    for name, n, times in (("prompt", prompt, 1), ("decode", 1, 32)):
        layer.step(*tokens(n), Cache(batch, n, heads, dim))     # warm-up
        steps = [tokens(n) for _ in range(times)]
        events[0].record()
        for x, r in steps:
            y, code = layer.step(x, r, cache)
        events[1].record()
        layer.lib.sync_status()
        print(f"{name}: {batch} x {n} tokens, {events[0].elapsed_time(events[1]) / times * 1e3:.0f} us a step;"
              f" codes 0 and {2 ** bits - 1} (clipped): {float(((code == 0) | (code == 2 ** bits - 1)).float().mean()):.2%};"
              f" messages to encrypt a token: {inner}")


if __name__ == "__main__":
    main()
