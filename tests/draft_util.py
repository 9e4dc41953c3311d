"""Drafted tokens from their definitions, on the CPU: attention under masks in 64 bits, verification in
whole numbers, rows of the cache in single precision step by step where bytes are decided by it."""

import numpy as np
import torch


def random_tree(seed, batch, nodes, short=True):
    """parents int32 [batch][nodes]: chains with branches; every third tree ends early (-1)."""
    g = torch.Generator().manual_seed(seed)
    at = torch.arange(nodes)
    parents = torch.where(torch.rand((batch, nodes), generator=g) < 0.4, at - 1, (torch.rand((batch, nodes), generator=g) * at).long())
    parents[:, 0] = -1
    if short:
        for b in range(2, batch, 3):
            parents[b, nodes - nodes // 3:] = -1
    return parents.to(torch.int32)


def ancestors(parents):
    """Truth values [batch][nodes][nodes]: is j node i or an ancestor of it?"""
    b, n = parents.shape
    seen = torch.zeros((b, n, n), dtype=torch.bool)
    for s in range(b):
        for i in range(n):
            j = i
            while j >= 0:
                seen[s, i, j] = True
                j = int(parents[s, j])
    return seen


def words(seen):
    """[...][n] truth values as int32 words, bit j % 32 of word j / 32."""
    bits = np.packbits(seen.numpy(), axis=-1, bitorder="little")
    pad = -bits.shape[-1] % 4
    bits = np.concatenate([bits, np.zeros((*bits.shape[:-1], pad), np.uint8)], -1)
    return torch.from_numpy(np.ascontiguousarray(bits).view("<i4").copy())


def tree_attention(q, k_cache, v_cache, k_scale, v_scale, table, lengths, seen, softmax_scale):
    """(out, sum of p |v|) in 64 bits; seen [batch or 1][tokens][tokens]."""
    b, new, hq, d = q.shape
    heads, page = k_cache.shape[1], k_cache.shape[2]
    out, size = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for i in range(b):
        n = min(int(lengths[i]), table.shape[1] * page)
        if n <= 0:
            continue
        pages = table[i, :-(-n // page)].long()
        visible = torch.ones((new, n), dtype=torch.bool)
        for j in range(max(0, new - n), new):
            visible[:, n - new + j] = seen[i % seen.shape[0], :, j]
        for h in range(heads):
            k = (k_cache[pages, h].double() * k_scale[pages, h].double()[:, None, None]).flatten(0, 1)[:n]
            v = (v_cache[pages, h].double() * v_scale[pages, h].double()[:, None, None]).flatten(0, 1)[:n]
            for t in range(new):
                at = visible[t].nonzero()[:, 0]
                if len(at) == 0:
                    continue
                kt, vt = k[at], v[at]
                for g in range(h * (hq // heads), (h + 1) * (hq // heads)):
                    p = torch.softmax(kt @ q[i, t, g].double() * softmax_scale, 0)
                    out[i, t, g], size[i, t, g] = p @ vt, p @ vt.abs()
    return out, size


ONE = 1 << 149      # floats are whole multiples of its inverse


def whole(values):
    return [int(v * 2.0 ** 149) for v in values.double().tolist()]


def verify(target, draft, tokens, parents, uniform):
    """(path, count, next) of one sequence, in whole numbers without rounding."""
    nodes, vocab = target.shape
    u = whole(uniform)
    path = [0]
    while True:
        n, chosen = path[-1], None
        first = left = whole(target[n])     # left and total: in units that become finer with each rejection
        q = whole(draft[n]) if draft is not None else None
        total = ONE
        for c in range(n + 1, nodes):
            x = int(tokens[c])
            if int(parents[c]) != n or not 0 <= x < vocab:
                continue
            if draft is None:
                if u[c] * total < left[x] * ONE:
                    chosen = c
                    break
                total = max(total - left[x], 0)
                left = [0 if i == x else w for i, w in enumerate(left)]
            else:
                if u[c] * q[x] * total < left[x] * ONE * ONE:
                    chosen = c
                    break
                left = [max(w * ONE - total * v, 0) for w, v in zip(left, q)]
                total = sum(left)
        if chosen is None:
            break
        path.append(chosen)
    if not any(left):
        left = first
    goal, run = u[0] * sum(left), 0
    for x, w in enumerate(left):
        run += w
        if run * ONE > goal:
            return path, len(path), x
    return path, len(path), -1


def keep(cache, scale, table, first, path, count):
    """cache [pages][heads][page][dim] int8 and scale [pages][heads] after rows first + path[i] became first + i."""
    old, was = cache.numpy(), scale.numpy()
    new, now = old.copy(), was.copy()
    page = old.shape[2]
    for b in range(len(first)):
        f, e = int(first[b]), int(first[b]) + int(count[b])
        if f < 0 or e == f:
            continue
        for slot in range(f // page, (e - 1) // page + 1):
            p = int(table[b, slot])
            rows = {r: (p, r) for r in range(page) if slot * page + r < f}
            for r in range(page):
                i = slot * page + r - f
                if 0 <= i < e - f:
                    at = f + int(path[b, i])
                    rows[r] = (int(table[b, at // page]), at % page)
            for h in range(old.shape[1]):
                top = np.float32(np.max([was[s, h] for s, _ in rows.values()]))     # (a NaN where there is one)
                div = top if top > 0 else np.float32(1)
                for r, (s, i) in rows.items():
                    q = old[s, h, i]
                    new[p, h, r] = q if np.isnan(top) or was[s, h] == top else np.rint(q.astype(np.float32) * (was[s, h] / div)).astype(np.int8)
                now[p, h] = top
    return torch.from_numpy(new), torch.from_numpy(now)


def read(cache, scale, table, first, lengths, out):
    """out [batch][tokens][heads][dim] with the cached rows in their places."""
    out, page = out.clone(), cache.shape[2]
    for b in range(out.shape[0]):
        n = min(int(lengths[b]), table.shape[1] * page)
        for i in range(out.shape[1]):
            at = int(first[b]) + i
            if 0 <= at < n:
                p = int(table[b, at // page])
                out[b, i] = (cache[p, :, at % page].float() * scale[p][:, None]).to(out.dtype)
    return out
