"""The operators of a decoder layer in the clear with 8-bit activations, weights
and cache, as timed cases: the layer around a bootstrapped nonlinearity, whose
linear products give the message codes that are encrypted, and on which a
table's range and precision are judged without encryption.

  norm     residual addition, root-mean-square norm, 8-bit output with a scale per token
  linear   8-bit integer product with a scale per token and channel: a float, or a message
           code of the table's range and that table's 8-bit entry
  append   new keys and values into the paged 8-bit cache, a scale per page and head
  attend   causal attention over that cache

Widths and head layouts are those of the named workloads (GPT-2-small: 768 = 12 x 64,
inner 3072; LLaMA-3-8B: 4096 = 32 x 128 over 8 cached heads, inner 14336) and odd ones.
A case is a dict: ``kind``, its sizes, the floating type, and where they apply a row
pitch wider than the row (``pitch``) and uneven lengths (``ragged``).
"""

from __future__ import annotations

import math

import torch

own = False

_TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}
EPS = 1e-5


def listed():
    return [
        # one decode token between two layers of GPT-2-small's width: latency
        {"name": "norm_one", "kind": "norm", "tokens": 1, "width": 768, "type": "bfloat16", "residual": True, "pitch": 0},
        # an odd width, single precision, rows of a wider buffer, no residual (the first norm)
        {"name": "norm_odd", "kind": "norm", "tokens": 1333, "width": 1021, "type": "float32", "residual": False, "pitch": 3},
        # a calibration batch of LLaMA-3-8B's width
        {"name": "norm_batch", "kind": "norm", "tokens": 16384, "width": 4096, "type": "bfloat16", "residual": True, "pitch": 0},
        # one decode token, GPT-2-small's inner layer up to the codes of its 6-bit GELU and the table's values
        {"name": "linear_one_codes", "kind": "linear", "tokens": 1, "inner": 768, "channels": 3072, "type": "codes",
         "bits": 6, "bias": True, "pitch": 0},
        # 24 sequences decoding at LLaMA-3-8B's inner layer
        {"name": "linear_decode", "kind": "linear", "tokens": 24, "inner": 4096, "channels": 14336, "type": "bfloat16",
         "bits": 0, "bias": False, "pitch": 0},
        # odd sizes, single precision, a short prompt
        {"name": "linear_odd", "kind": "linear", "tokens": 333, "inner": 1021, "channels": 2999, "type": "float32",
         "bits": 0, "bias": True, "pitch": 5},
        # a calibration batch through LLaMA-3-8B's inner layer
        {"name": "linear_batch", "kind": "linear", "tokens": 4096, "inner": 4096, "channels": 14336, "type": "bfloat16",
         "bits": 0, "bias": False, "pitch": 0},
        # a decode step of 256 sequences, one token each
        {"name": "append_decode", "kind": "append", "batch": 256, "new": 1, "heads": 8, "dim": 128, "page": 16,
         "context": 2048, "type": "bfloat16", "ragged": True},
        # prompts entering the cache, starting inside a page
        {"name": "append_prompt", "kind": "append", "batch": 8, "new": 2043, "heads": 8, "dim": 128, "page": 32,
         "context": 2101, "type": "float16", "ragged": True},
        # one decode token of GPT-2-small over a short context
        {"name": "attend_one", "kind": "attend", "batch": 1, "new": 1, "heads": 12, "group": 1, "dim": 64, "page": 16,
         "context": 77, "type": "float16", "ragged": False},
        # a decode step of 64 uneven sequences, LLaMA-3-8B's heads
        {"name": "attend_decode", "kind": "attend", "batch": 64, "new": 1, "heads": 8, "group": 4, "dim": 128, "page": 32,
         "context": 8192, "type": "bfloat16", "ragged": True},
        # the second half of prompts, causal, over what the cache holds
        {"name": "attend_prompt", "kind": "attend", "batch": 4, "new": 1024, "heads": 8, "group": 4, "dim": 128, "page": 32,
         "context": 2048, "type": "bfloat16", "ragged": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        b, f = most.get(c["kind"], (0, 0))
        most[c["kind"]] = max(b, w["bytes"]), max(f, w["flops"])
    kind = rng.choice(("norm", "linear", "linear", "append", "attend", "attend"))
    while True:
        if kind == "norm":
            c = {"kind": kind, "tokens": _log_int(rng, 1, 32768), "width": _log_int(rng, 64, 16384),
                 "type": rng.choice(sorted(_TYPES)), "residual": rng.random() < 0.7, "pitch": rng.choice((0, 0, 1, 64))}
        elif kind == "linear":
            c = {"kind": kind, "tokens": _log_int(rng, 1, 8192), "inner": _log_int(rng, 64, 16384),
                 "channels": _log_int(rng, 64, 16384), "type": rng.choice(sorted(_TYPES) + ["codes"]), "bits": 0,
                 "bias": rng.random() < 0.5, "pitch": rng.choice((0, 0, 3, 64))}
            if rng.random() < 0.5:
                c["inner"] = -(-c["inner"] // 64) * 64
            if c["type"] == "codes":
                c["bits"] = rng.randint(3, 8)
        else:
            c = {"kind": kind, "batch": _log_int(rng, 1, 256), "new": 1 if rng.random() < 0.5 else _log_int(rng, 1, 2048),
                 "heads": rng.choice((1, 2, 5, 8, 12)), "group": rng.choice((1, 1, 2, 4, 7, 8)),
                 "dim": rng.choice((64, 64, 96, 128, 128, 256)), "page": rng.choice((16, 32, 64, 128)),
                 "context": _log_int(rng, 1, 65536), "type": rng.choice(sorted(_TYPES)), "ragged": rng.random() < 0.6}
            c["context"] = max(c["context"], c["new"])
            if kind == "append":
                del c["group"]
            # the cache, and the plain form's scores
            if c["batch"] * c["context"] * c["heads"] * c["dim"] > 600e6:
                continue
            if kind == "attend" and c["batch"] * c["new"] * c["heads"] * c["group"] * c["context"] > 500e6:
                continue
        w = work(c)
        if w["bytes"] <= most[kind][0] and w["flops"] <= most[kind][1]:
            return c


# ------------------------------------------------------------------ sizes that depend on a case's lengths


def _lengths(case):
    """Context of each sequence after this call's tokens: all `context`, or spread below it (the first keeps it).
    An appended token has to fit; an attending one may have no position (a prompt padded on the left)."""
    b, full = case["batch"], case["context"]
    if not case["ragged"]:
        return [full] * b
    least = case["new"] if case["kind"] == "append" else 1
    return [full - (i * 7919) % (full - least + 1) for i in range(b)]


def _touched(case):
    """(sequence, page of the sequence) of every page that an append writes to."""
    page, new = case["page"], case["new"]
    return [(b, j) for b, n in enumerate(_lengths(case)) for j in range((n - new) // page, (n - 1) // page + 1)]


def work(case):
    kind = case["kind"]
    size = 4 if case["type"] == "float32" else 1 if case["type"] == "codes" else 2
    if kind == "norm":
        t, w = case["tokens"], case["width"]
        return {"bytes": t * w * ((3 if case["residual"] else 1) * size + 1) + 4 * t + 4 * w, "flops": 8 * t * w}
    if kind == "linear":
        t, k, n = case["tokens"], case["inner"], case["channels"]
        return {"bytes": t * k + n * k + t * n * size + 4 * t + (8 if case["bias"] else 4) * n, "flops": 2 * t * n * k}
    h, d = case["heads"], case["dim"]
    if kind == "append":
        rows = case["batch"] * case["new"] * h
        return {"bytes": 2 * rows * d * (size + 1) + 2 * 8 * len(_touched(case)) * h, "flops": 8 * rows * d}
    new, hq, lens = case["new"], h * case["group"], _lengths(case)
    pairs = sum(sum(max(0, n - new + 1 + t) for t in range(new)) for n in lens)
    pages = sum(-(-n // case["page"]) for n in lens)
    return {"bytes": 2 * sum(lens) * h * d + 8 * pages * h + 4 * pages + 2 * case["batch"] * new * hq * d * size,
            "flops": 4 * pairs * hq * d}


# ------------------------------------------------------------------ inputs


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 29)
    s = dict(case)

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=g)

    def small(*shape):      # 8-bit values of a normal distribution
        return (torch.randn(shape, device="cuda", generator=g, dtype=torch.float16) * 36).round_().clamp_(-127, 127).to(torch.int8)

    if case["kind"] == "norm":
        t, w, p, dt = case["tokens"], case["width"], case["pitch"], _TYPES[case["type"]]
        # activations: a few channels far larger than the rest
        big = torch.where(torch.rand(w, device="cuda", generator=g) < 0.01, 20.0, 1.0)
        s["x"] = (normal(t, w + p) * torch.nn.functional.pad(big, (0, p))).to(dt)[:, :w]
        s["residual"] = (normal(t, w + p) * 2).to(dt)[:, :w] if case["residual"] else None
        s["gamma"] = 1 + 0.1 * normal(w)
    elif case["kind"] == "linear":
        t, k, n, p = case["tokens"], case["inner"], case["channels"], case["pitch"]
        s["q"] = small(t, k + p)[:, :k]
        s["scale"] = (1 + torch.rand(t, device="cuda", generator=g)) / 60
        s["weight"] = small(n, k)
        s["w_scale"] = (1 + torch.rand(n, device="cuda", generator=g)) / (36 * math.sqrt(k))
        s["bias"] = normal(n) * 0.1 if case["bias"] else None
        s["table"] = None
        if case["bits"]:    # GELU on the midpoints of [-4, 4], in 127ths of 4
            size = 1 << case["bits"]
            x = -4 + 8 * (torch.arange(size, device="cuda", dtype=torch.float64) + 0.5) / size
            s["table"] = (0.5 * x * (1 + torch.erf(x / math.sqrt(2))) * 127 / 4).round().to(torch.int8)
    else:
        b, h, d, page, new = (case[x] for x in ("batch", "heads", "dim", "page", "new"))
        dt, lens = _TYPES[case["type"]], _lengths(case)
        each = -(-max(lens) // page)
        pages = sum(-(-n // page) for n in lens)
        order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
        slot, rows = 0, []
        for n in lens:
            rows.append((slot, -(-n // page)))
            slot += rows[-1][1]
        start = torch.tensor([r[0] for r in rows], device="cuda")[:, None]
        count = torch.tensor([r[1] for r in rows], device="cuda")[:, None]
        at = torch.arange(each, device="cuda")[None, :]
        s["pages"] = torch.where(at < count, order[(start + at).clamp_(max=pages - 1)], 0).to(torch.int32).contiguous()
        s["k_cache"], s["v_cache"] = small(pages, h, page, d), small(pages, h, page, d)
        s["k_scale"] = (1 + torch.rand(pages, h, device="cuda", generator=g)) / 72
        s["v_scale"] = (1 + torch.rand(pages, h, device="cuda", generator=g)) / 72
        lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        if case["kind"] == "append":
            qkv = normal(b, new, 2 * h, d).to(dt)      # slices of one projection's output
            s["k"], s["v"] = qkv[:, :, :h], qkv[:, :, h:]
            s["first"] = lens - new
            which = torch.tensor(_touched(case), device="cuda")
            s["seq"], s["slot"] = which[:, 0], which[:, 1]
            s["page_of"] = s["pages"][s["seq"], s["slot"]].long()
        else:
            hq = h * case["group"]
            s["q"] = (normal(b, new, hq + h, d) * 1.5).to(dt)[:, :, :hq]
            s["lengths"] = lens
            s["softmax_scale"] = 1 / math.sqrt(d)
    if own:
        from paper_2609_16915_gb300 import clear
        s["lib"] = clear.Clear()
        if case["kind"] == "linear":
            s["packed"] = s["lib"].pack_weights(s["weight"])
    return s


# ------------------------------------------------------------------ one pass


def _norm(s):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["gamma"]
    scale = y.abs().amax(1) / 127
    q = torch.where(scale[:, None] > 0, torch.round(y / scale[:, None]), 0.0)
    return q, scale, h.to(s["x"].dtype)


def _linear(s):
    # whole numbers below 2^24 in single precision: the sums are exact
    acc = s["q"].float() @ s["weight"].float().T
    y = acc * s["scale"][:, None] * s["w_scale"]
    if s["bias"] is not None:
        y = y + s["bias"]
    if not s["bits"]:
        return y.to(_TYPES[s["type"]])
    size = 1 << s["bits"]
    code = torch.floor((y + 4.0) * (size / 8.0)).clamp(0, size - 1)
    return code.to(torch.uint8), s["table"][code.long()]


def _append(x, cache, scale, s):
    page, first, new = s["page"], s["first"][s["seq"]].long()[:, None], s["new"]
    at = s["slot"][:, None] * page + torch.arange(page, device="cuda")      # positions of the touched pages
    fresh = ((at >= first) & (at < first + new))[:, None, :, None]
    kept = (at < first)[:, None, :, None]
    x = x[s["seq"][:, None], (at - first).clamp(0, new - 1)].permute(0, 2, 1, 3).float()
    was = torch.where(s["slot"][:, None] * page < first, scale[s["page_of"]], 0.0)
    now = torch.maximum(was, torch.where(fresh, x.abs(), 0.0).amax((2, 3)) / 127)
    div = torch.where(now > 0, now, 1.0)[:, :, None, None]
    old = cache[s["page_of"]]
    keep = torch.round(old.float() * (was[:, :, None, None] / div))
    cache[s["page_of"]] = torch.where(fresh, torch.round(x / div), torch.where(kept, keep, old.float())).to(torch.int8)
    scale[s["page_of"]] = now


def _attend(s):
    b, new, hq, d = s["q"].shape
    h, g, n = s["heads"], s["group"], s["pages"].shape[1] * s["page"]

    def whole(cache, scale):
        pages = s["pages"].long()
        x = cache[pages].float() * scale[pages][..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(b, h, n, d)

    q = s["q"].float().reshape(b, new, h, g, d).permute(0, 2, 3, 1, 4).reshape(b, h, g * new, d)
    score = (q @ whole(s["k_cache"], s["k_scale"]).transpose(2, 3)).mul_(s["softmax_scale"]).reshape(b, h, g, new, n)
    last = (s["lengths"].long()[:, None] - new + torch.arange(new, device="cuda"))[:, None, None, :, None]
    seen = torch.arange(n, device="cuda") <= last
    score = torch.where(seen, score, -math.inf)
    top = score.amax(4, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(4, keepdim=True)
    out = p.reshape(b, h, g * new, n) @ whole(s["v_cache"], s["v_scale"])
    out = out.reshape(b, h, g, new, d) / torch.where(total > 0, total, 1.0)
    return out.permute(0, 3, 1, 2, 4).reshape(b, new, hq, d).to(s["q"].dtype)


def _pages_values(cache, scale, pages):
    """What the 8-bit values of the pages stand for."""
    x = cache[pages]
    return torch.mul(x, scale[pages][:, :, None, None], out=torch.empty(x.shape, dtype=torch.bfloat16, device="cuda"))


def run(s):
    kind = s["kind"]
    if kind == "norm":
        if own:
            q = torch.empty(s["x"].shape, dtype=torch.int8, device="cuda")
            scale = torch.empty(s["x"].shape[0], device="cuda")
            total = torch.empty(s["x"].shape, dtype=s["x"].dtype, device="cuda") if s["residual"] is not None else None
            s["lib"].norm(s["x"], s["gamma"], q, scale, residual=s["residual"], sum_out=total, eps=EPS)
        else:
            q, scale, total = _norm(s)
        out = {"values": torch.mul(q, scale[:, None], out=torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")),
               "scale": scale}
        if s["residual"] is not None:
            out["sum"] = total
        return out
    if kind == "linear":
        if not own:
            return _linear(s)
        t, n, lib = s["tokens"], s["channels"], s["lib"]
        if not s["bits"]:
            y = torch.empty((t, n), dtype=_TYPES[s["type"]], device="cuda")
            return lib.linear(s["q"], s["scale"], s["packed"], s["w_scale"], y, bias=s["bias"])
        code = torch.empty((t, n), dtype=torch.uint8, device="cuda")
        value = torch.empty((t, n), dtype=torch.int8, device="cuda")
        lib.linear_codes(s["q"], s["scale"], s["packed"], s["w_scale"], code, s["bits"], -4.0, 4.0, bias=s["bias"],
                         table=s["table"], values=value)
        return code, value
    if kind == "append":
        if own:
            s["lib"].cache_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["pages"], s["first"])
        else:
            _append(s["k"], s["k_cache"], s["k_scale"], s)
            _append(s["v"], s["v_cache"], s["v_scale"], s)
        p = s["page_of"]
        return {"k": _pages_values(s["k_cache"], s["k_scale"], p), "k_scale": s["k_scale"][p],
                "v": _pages_values(s["v_cache"], s["v_scale"], p), "v_scale": s["v_scale"][p]}
    if not own:
        return _attend(s)
    out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    return s["lib"].attention(s["q"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["pages"], s["lengths"], out,
                              softmax_scale=s["softmax_scale"])


# ------------------------------------------------------------------ the same from the definitions, in 64 bits


def _inputs(case, seed):
    """prepare()'s tensors, without the library's handle."""
    global own
    was, own = own, False
    try:
        return prepare(case, seed)
    finally:
        own = was


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind == "norm":
        h = s["x"].double() + (s["residual"].double() if s["residual"] is not None else 0)
        rms = torch.sqrt((h ** 2).sum(1) / case["width"] + EPS)
        y = h / rms[:, None] * s["gamma"].double()
        scale = y.abs().max(1).values / 127
        out = {"values": torch.round(y / scale[:, None]) * scale[:, None], "scale": scale}
        if s["residual"] is not None:
            out["sum"] = h
        return out
    if kind == "linear":
        if case["bits"]:
            return None         # whole numbers
        y = (s["q"].double() @ s["weight"].double().T) * torch.outer(s["scale"].double(), s["w_scale"].double())
        return y + s["bias"].double() if s["bias"] is not None else y
    if kind == "append":
        out = {}
        for name in ("k", "v"):
            x, cache, scale = s[name].double().cpu(), s[name + "_cache"].cpu(), s[name + "_scale"].double().cpu()
            page, lens, new = case["page"], _lengths(case), case["new"]
            values, scales = [], []
            for (b, j), p in zip(_touched(case), s["page_of"].tolist()):
                lo, first = j * page, lens[b] - new
                a, e = max(first - lo, 0), min(lens[b] - lo, page)      # the page's rows a..e-1 are new
                fresh = x[b, lo + a - first:lo + e - first].permute(1, 0, 2)
                now = fresh.abs().amax((1, 2)) / 127
                was = scale[p]
                if a > 0:
                    now = torch.maximum(now, was)
                q = cache[p].double()
                q[:, :a] = torch.round(q[:, :a] * (was / now)[:, None, None])
                q[:, a:e] = torch.round(fresh / now[:, None, None])
                values.append(q * now[:, None, None])
                scales.append(now)
            out[name], out[name + "_scale"] = torch.stack(values), torch.stack(scales)
        return out
    lens, new, g = _lengths(case), case["new"], case["group"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        pages = s["pages"][b, :-(-n // case["page"])].long()
        hidden = (torch.arange(n, device="cuda")[None, :] - torch.arange(n - new, n, device="cuda")[:, None]) > 0
        rows = max(0, new - n)          # the first rows have no position
        for h in range(case["heads"]):
            k = (s["k_cache"][pages, h].double() * s["k_scale"][pages, h].double()[:, None, None]).flatten(0, 1)[:n]
            v = (s["v_cache"][pages, h].double() * s["v_scale"][pages, h].double()[:, None, None]).flatten(0, 1)[:n]
            for i in range(h * g, h * g + g):
                z = (s["q"][b, rows:, i].double() @ k.T * s["softmax_scale"]).masked_fill(hidden[rows:], -math.inf)
                out[b, rows:, i] = torch.softmax(z, 1) @ v
    return out
