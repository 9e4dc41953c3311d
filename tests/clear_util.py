"""The decoder layer in the clear from its definitions, on the CPU: numpy in 64 bits, or in
single precision step by step where the outputs are whole numbers decided by it."""

import numpy as np
import torch

UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


def rand(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


def int8(seed, *shape, lo=-127, hi=128):
    return torch.randint(lo, hi, shape, generator=torch.Generator().manual_seed(seed), dtype=torch.int8)


def norm(x, residual, gamma, eps):
    """(y, scale, h) in 64 bits."""
    h = x.double() + (residual.double() if residual is not None else 0)
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps) * gamma.double()
    return y, y.abs().amax(1) / 127, h


def linear(q, scale, weight, w_scale, bias):
    """Exact integer sums, then the scales step by step in single precision."""
    acc = q.numpy().astype(np.int64) @ weight.numpy().astype(np.int64).T
    y = acc.astype(np.float32) * scale.numpy()[:, None]
    y = y * w_scale.numpy()
    return y + bias.numpy() if bias is not None else y


def codes(y, bits, lo, hi):
    inv = np.float32((1 << bits) / (float(np.float32(hi)) - float(np.float32(lo))))
    f = np.floor((y - np.float32(lo)) * inv)
    return np.clip(np.where(np.isnan(f), 0, f), 0, (1 << bits) - 1).astype(np.uint8)


def append(x, cache, scale, table, first):
    """cache [pages][heads][page][dim] int8 and scale [pages][heads] after appending x [batch][new][heads][dim]."""
    cache, scale = cache.numpy().copy(), scale.numpy().copy()
    x = x.float().numpy()
    page = cache.shape[2]
    for b in range(x.shape[0]):
        f, e = int(first[b]), int(first[b]) + x.shape[1]
        if f < 0:
            continue
        for slot in range(f // page, (e - 1) // page + 1):
            p, row0 = int(table[b, slot]), slot * page
            lo, hi = max(f, row0), min(e, row0 + page)
            for h in range(cache.shape[1]):
                new = x[b, lo - f:hi - f, h]
                was = scale[p, h] if lo > row0 else np.float32(0)
                with np.errstate(invalid="ignore"):
                    now = np.maximum(was, np.abs(new).max() / np.float32(127))
                if not np.isfinite(now):
                    scale[p, h] = np.nan
                    continue
                div = now if now > 0 else np.float32(1)
                if lo > row0 and now != was:
                    old = cache[p, h, :lo - row0].astype(np.float32)
                    cache[p, h, :lo - row0] = np.rint(old * (was / div)).astype(np.int8)
                cache[p, h, lo - row0:hi - row0] = np.rint(new / div).astype(np.int8)
                scale[p, h] = now
    return torch.from_numpy(cache), torch.from_numpy(scale)


def attention(q, k_cache, v_cache, k_scale, v_scale, table, lengths, softmax_scale):
    """(out, sum of p |v|: what relative errors of the weights are measured against) in 64 bits."""
    b, new, hq, d = q.shape
    heads, page = k_cache.shape[1], k_cache.shape[2]
    out, size = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for i in range(b):
        n = min(int(lengths[i]), table.shape[1] * page)
        if n <= 0:
            continue
        pages = table[i, :-(-n // page)].long()
        for h in range(heads):
            k = (k_cache[pages, h].double() * k_scale[pages, h].double()[:, None, None]).flatten(0, 1)[:n]
            v = (v_cache[pages, h].double() * v_scale[pages, h].double()[:, None, None]).flatten(0, 1)[:n]
            for t in range(new):
                seen = n - new + t + 1
                if seen <= 0:
                    continue
                for g in range(h * (hq // heads), (h + 1) * (hq // heads)):
                    p = torch.softmax(k[:seen] @ q[i, t, g].double() * softmax_scale, 0)
                    out[i, t, g], size[i, t, g] = p @ v[:seen], p @ v[:seen].abs()
    return out, size
