"""Drafted tokens over the paged 8-bit cache of a decoder layer in the clear, as timed
cases: a tree of drafted tokens goes through the layer in one step, the target's
probabilities say which of them stand, and the cache keeps those.

  tree     the tree's mask from its parents, and attention of the drafted tokens over the
           cache, each seeing the context, its ancestors and itself
  verify   drafted tokens against the target's probabilities, from given random numbers
  keep     the accepted tokens' rows brought together behind the context
  read     cached rows as floats

Widths and head layouts are GPT-2-small's (12 heads of 64) and LLaMA-3-8B's (32 heads of 128
over 8 cached), as in the other operators' cases, and odd ones; vocabularies are generic sizes.
A case is a dict: ``kind``, its sizes, the floating type, and where they apply uneven
lengths and trees (``ragged``) and whether drafts were drawn from probabilities (``draft``).
``context`` counts the drafted tokens in (``new`` of them) but for ``keep``, whose drafts come behind it.
"""

from __future__ import annotations

import math

import torch

own = False

_TYPES = {"float32": torch.float32, "float16": torch.float16, "bfloat16": torch.bfloat16}


def listed():
    return [
        # one sequence of GPT-2-small, five drafted tokens: latency
        {"name": "tree_one", "kind": "tree", "batch": 1, "new": 5, "heads": 12, "group": 1, "dim": 64, "page": 16,
         "context": 82, "type": "float16", "ragged": False},
        # 16 uneven sequences with 16 drafted tokens each, LLaMA-3-8B's heads: a serving step
        {"name": "tree_decode", "kind": "tree", "batch": 16, "new": 16, "heads": 8, "group": 4, "dim": 128, "page": 32,
         "context": 4096, "type": "bfloat16", "ragged": True},
        # an odd head layout, odd sizes, single precision
        {"name": "tree_odd", "kind": "tree", "batch": 3, "new": 37, "heads": 5, "group": 7, "dim": 96, "page": 48,
         "context": 1501, "type": "float32", "ragged": True},
        # large trees over long contexts
        {"name": "tree_long", "kind": "tree", "batch": 32, "new": 64, "heads": 8, "group": 4, "dim": 128, "page": 32,
         "context": 8192, "type": "bfloat16", "ragged": True},
        # one sequence, five tokens that were given rather than drawn (the draft's likeliest): latency
        {"name": "verify_one", "kind": "verify", "batch": 1, "new": 5, "vocab": 50257, "type": "float32", "draft": False,
         "ragged": False},
        # an odd vocabulary and tree in 16 bits
        {"name": "verify_odd", "kind": "verify", "batch": 7, "new": 33, "vocab": 32003, "type": "bfloat16", "draft": True,
         "ragged": True},
        # a serving step: 64 sequences, trees drawn from the draft's probabilities
        {"name": "verify_batch", "kind": "verify", "batch": 64, "new": 64, "vocab": 128256, "type": "float32", "draft": True,
         "ragged": True},
        # what one sequence accepted
        {"name": "keep_one", "kind": "keep", "batch": 1, "new": 5, "heads": 12, "dim": 64, "page": 16, "context": 77,
         "ragged": False},
        # what 256 uneven sequences accepted of 64 drafted tokens
        {"name": "keep_batch", "kind": "keep", "batch": 256, "new": 64, "heads": 8, "dim": 128, "page": 32, "context": 1024,
         "ragged": True},
        # a short piece of two sequences in single precision, odd sizes
        {"name": "read_odd", "kind": "read", "batch": 2, "new": 131, "heads": 5, "dim": 96, "page": 48, "context": 301,
         "type": "float32", "ragged": True},
        # whole contexts of a batch, to be compared with what was written or written to other pages
        {"name": "read_batch", "kind": "read", "batch": 32, "new": 4096, "heads": 8, "dim": 128, "page": 32, "context": 4096,
         "type": "bfloat16", "ragged": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        b, f = most.get(c["kind"], (0, 0))
        most[c["kind"]] = max(b, w["bytes"]), max(f, w["flops"])
    kind = rng.choice(("tree", "tree", "tree", "verify", "verify", "keep", "read"))
    while True:
        if kind == "verify":
            c = {"kind": kind, "batch": _log_int(rng, 1, 128), "new": _log_int(rng, 1, 128), "vocab": _log_int(rng, 1000, 160000),
                 "type": rng.choice(sorted(_TYPES)), "draft": rng.random() < 0.6, "ragged": rng.random() < 0.6}
            # the probabilities, which a model has computed before
            if c["batch"] * c["new"] * c["vocab"] > 500e6:
                continue
        else:
            c = {"kind": kind, "batch": _log_int(rng, 1, 256), "new": _log_int(rng, 1, 4096 if kind == "read" else 128),
                 "heads": rng.choice((1, 2, 5, 8, 12)), "dim": rng.choice((64, 64, 96, 128, 128, 256)),
                 "page": rng.choice((16, 32, 48, 64, 128)), "context": _log_int(rng, 1, 32768), "ragged": rng.random() < 0.6}
            if kind != "keep":
                c["type"] = rng.choice(sorted(_TYPES))
                c["context"] = max(c["context"], c["new"])
            if kind == "tree":
                c["group"] = rng.choice((1, 1, 2, 4, 7, 8))
            # the cache, and the plain form's scores
            if c["batch"] * (c["context"] + c["new"]) * c["heads"] * c["dim"] > 400e6:
                continue
            if kind == "tree" and c["batch"] * c["new"] * c["heads"] * c["group"] * c["context"] > 500e6:
                continue
        w = work(c)
        if w["bytes"] <= most[kind][0] and w["flops"] <= most[kind][1]:
            return c


# ------------------------------------------------------------------ sizes that depend on a case's lengths


def _lengths(case):
    """Positions of each sequence: all `context`, or spread below it (the first keeps it); the drafted tokens fit."""
    b, full = case["batch"], case["context"]
    if not case["ragged"]:
        return [full] * b
    least = case["new"] if case["kind"] == "tree" else 1
    return [full - (i * 7919) % (full - least + 1) for i in range(b)]


def _held(case):
    """Positions that each sequence has pages for."""
    return [n + (case["new"] if case["kind"] == "keep" else 0) for n in _lengths(case)]


def _drafted_pages(case):
    """(sequence, page of the sequence) of every page that holds drafted rows, where accepted ones are kept."""
    page, new = case["page"], case["new"]
    return [(b, j) for b, n in enumerate(_lengths(case)) for j in range(n // page, (n + new - 1) // page + 1)]


def _read_first(case):
    """The last `new` positions of the longest sequence; the others end before, or begin at 0."""
    return [max(n - case["new"], 0) for n in _lengths(case)]


def work(case):
    kind, b, new = case["kind"], case["batch"], case["new"]
    size = 4 if case.get("type") == "float32" else 2
    if kind == "verify":
        # the last row of each sequence: the target's, and the draft's where its tokens were drawn; a word of the others
        rows = 2 if case["draft"] else 1
        return {"bytes": b * (case["vocab"] * size * rows + new * (rows * size + 12) + 8), "flops": b * case["vocab"] * (1 + 2 * (rows - 1))}
    h, d, lens = case["heads"], case["dim"], _lengths(case)
    pages = sum(-(-n // case["page"]) for n in lens)
    if kind == "keep":      # the path's rows, read and written
        rows = sum(_accepted(new, i) for i in range(b)) * h
        return {"bytes": 2 * 2 * rows * d + 16 * b * h + 4 * b * (new + 2), "flops": 4 * rows * d}
    if kind == "read":
        rows = sum(min(n - f, new) for n, f in zip(lens, _read_first(case)))
        return {"bytes": 2 * rows * h * d * (1 + size) + 8 * rows // case["page"] * h + 8 * b, "flops": 2 * rows * h * d}
    hq = h * case["group"]
    pairs = sum(new * (n - new + 1) for n in lens)
    return {"bytes": 2 * sum(lens) * h * d + 8 * pages * h + 4 * pages + 2 * b * new * hq * d * size + 4 * b * new,
            "flops": 4 * pairs * hq * d}


def _accepted(new, i):
    """Tokens of the path that sequence i accepted."""
    return min(new, 1 + (i * 5 + 2) % 8)


# ------------------------------------------------------------------ inputs


def _parents(case, g):
    """A tree for each sequence, its root first: chains with branches; shorter ones (of -1 behind) where ragged."""
    b, new = case["batch"], case["new"]
    r, chain = torch.rand((b, new), generator=g), torch.rand((b, new), generator=g) < 0.5
    at = torch.arange(new)
    parents = torch.where(chain, at - 1, (r * at).long())
    parents[:, 0] = -1
    if case["ragged"]:
        short = torch.tensor([new - new // 4 if i % 4 == 3 else new for i in range(b)])
        parents = torch.where(at[None, :] < short[:, None], parents, -1)
    return parents.to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1000003 * seed + 31)
    host = torch.Generator()
    host.manual_seed(1000003 * seed + 37)
    s = dict(case)
    b, new = case["batch"], case["new"]
    if case["kind"] in ("tree", "verify"):
        s["parents"] = _parents(case, host).cuda()
    if case["kind"] == "verify":
        _prepare_verify(case, s, g)
    else:
        _prepare_cache(case, s, g)
    if case["kind"] == "tree":
        hq, h, d = case["heads"] * case["group"], case["heads"], case["dim"]
        # queries are a slice of one projection's output
        s["q"] = (torch.randn((b, new, hq + 2 * h, d), device="cuda", generator=g) * 1.5).to(_TYPES[case["type"]])[:, :, :hq]
        s["softmax_scale"] = 1 / math.sqrt(d)
    elif case["kind"] == "keep":
        path = torch.full((b, new), -1, dtype=torch.int32)
        count = [_accepted(new, i) for i in range(b)]
        for i in range(b):      # the root and the nodes of a path, in order
            nodes = torch.randperm(new - 1, generator=host)[:count[i] - 1].sort().values + 1 if new > 1 else torch.zeros(0)
            path[i, 0], path[i, 1:count[i]] = 0, nodes.to(torch.int32)
        s["path"], s["count"] = path.cuda(), torch.tensor(count, dtype=torch.int32, device="cuda")
        which = torch.tensor(_drafted_pages(case), device="cuda")
        s["seq"], s["slot"] = which[:, 0], which[:, 1]
        s["page_of"] = s["pages"][s["seq"], s["slot"]].long()
    elif case["kind"] == "read":
        s["first"] = torch.tensor(_read_first(case), dtype=torch.int32, device="cuda")
        s["k"], s["v"] = (torch.zeros((b, new, case["heads"], case["dim"]), dtype=_TYPES[case["type"]], device="cuda") for _ in range(2))
    if own:
        from paper_2609_16915_gb300 import clear
        s["lib"] = clear.Clear()
    return s


def _prepare_verify(case, s, g):
    b, new, vocab, dt = case["batch"], case["new"], case["vocab"], _TYPES[case["type"]]
    s["target"] = torch.empty((b, new, vocab), dtype=dt, device="cuda")
    s["draft"] = torch.empty((b, new, vocab), dtype=dt, device="cuda") if case["draft"] else None
    likeliest = torch.empty((b, new, 16), dtype=torch.long, device="cuda")
    for n in range(new):        # peaked rows; the draft's are near the target's
        logits = 4 * torch.randn((b, vocab), device="cuda", generator=g)
        near = logits + torch.randn((b, vocab), device="cuda", generator=g)
        s["target"][:, n] = torch.softmax(logits, 1).to(dt)
        if case["draft"]:
            s["draft"][:, n] = torch.softmax(near, 1).to(dt)
        else:
            likeliest[:, n] = near.topk(16, 1).indices
    s["tokens"] = torch.zeros((b, new), dtype=torch.int32, device="cuda")
    seq, parents = torch.arange(b, device="cuda"), s["parents"].long()
    for c in range(1, new):
        up = parents[:, c].clamp_min(0)
        if case["draft"]:       # drawn from the parent's row, each anew
            q = s["draft"][seq, up].float()
            x = (q / torch.empty_like(q).exponential_(generator=g)).argmax(1)
        else:                   # the parent's likeliest that is not drafted yet
            rank = (parents[:, 1:c] == parents[:, c:c + 1]).sum(1).clamp_max(15)
            x = likeliest[seq, up, rank]
        s["tokens"][:, c] = x.to(torch.int32)
    s["uniform"] = torch.rand((b, new), device="cuda", generator=g)


def _prepare_cache(case, s, g):
    h, d, page, held = case["heads"], case["dim"], case["page"], _held(case)
    pages, each = sum(-(-n // page) for n in held), -(-max(held) // page)

    def small():            # 8-bit values of a normal distribution
        return (torch.randn((pages, h, page, d), device="cuda", generator=g, dtype=torch.float16) * 36).round_().clamp_(-127, 127).to(torch.int8)

    order = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    count = torch.tensor([-(-n // page) for n in held], device="cuda")
    start = count.cumsum(0) - count
    at = torch.arange(each, device="cuda")[None, :]
    s["pages"] = torch.where(at < count[:, None], order[(start[:, None] + at).clamp_(max=pages - 1)], 0).to(torch.int32).contiguous()
    s["k_cache"], s["v_cache"] = small(), small()
    s["k_scale"] = (1 + torch.rand(pages, h, device="cuda", generator=g)) / 72
    s["v_scale"] = (1 + torch.rand(pages, h, device="cuda", generator=g)) / 72
    s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ one pass


def _words(seen):
    """Truth values [...][n] as words of 32 bits, the lowest first."""
    n = seen.shape[-1]
    seen = torch.nn.functional.pad(seen.long(), (0, -n % 32)).reshape(*seen.shape[:-1], -1, 32)
    words = (seen << torch.arange(32, device="cuda")).sum(-1)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)


def _tree(s):
    b, new, hq, d = s["q"].shape
    h, g, page = s["heads"], s["group"], s["page"]
    n = s["pages"].shape[1] * page
    # ancestors: paths of up to 1, 2, 4 .. steps
    at = torch.arange(new, device="cuda")
    seen = ((s["parents"][:, :, None] == at) | (at[:, None] == at)).float()
    for _ in range(max(1, (new - 1).bit_length())):
        seen = ((seen @ seen) > 0).float()
    seen = seen > 0

    def whole(cache, scale):
        pages = s["pages"].long()
        x = cache[pages].float() * scale[pages][..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(b, h, n, d)

    q = s["q"].float().reshape(b, new, h, g, d).permute(0, 2, 3, 1, 4).reshape(b, h, g * new, d)
    score = (q @ whole(s["k_cache"], s["k_scale"]).transpose(2, 3)).mul_(s["softmax_scale"]).reshape(b, h, g, new, n)
    node = torch.arange(n, device="cuda") - (s["lengths"].long()[:, None] - new)     # of each position; the context below 0
    drafted = torch.gather(seen, 2, node.clamp(0, new - 1)[:, None, :].expand(b, new, n)) & (node < new)[:, None, :]
    visible = ((node < 0)[:, None, :] | drafted)[:, None, None]
    score = torch.where(visible, score, -math.inf)
    top = score.amax(4, keepdim=True)
    p = torch.exp(score - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(4, keepdim=True)
    out = p.reshape(b, h, g * new, n) @ whole(s["v_cache"], s["v_scale"])
    out = out.reshape(b, h, g, new, d) / torch.where(total > 0, total, 1.0)
    return out.permute(0, 3, 1, 2, 4).reshape(b, new, hq, d).to(s["q"].dtype), _words(seen)


def _verify(s):
    b, new, vocab = s["target"].shape
    seq = torch.arange(b, device="cuda")
    node, count = torch.zeros(b, dtype=torch.long, device="cuda"), torch.ones(b, dtype=torch.long, device="cuda")
    path = torch.full((b, new), -1, dtype=torch.long, device="cuda")
    path[:, 0] = 0
    uniform = s["uniform"].double()
    taken = torch.zeros(b, dtype=torch.float64, device="cuda")      # of the draft's row, off the target's
    left = torch.ones(b, dtype=torch.float64, device="cuda")        # the sum of what remains
    gone = torch.zeros((b, vocab), dtype=torch.bool, device="cuda")
    for c in range(1, new):
        child = s["parents"][:, c] == node
        x = s["tokens"][:, c].long()
        p, u = s["target"][seq, node, x].double(), uniform[:, c]
        if s["draft"] is not None:
            q = s["draft"][seq, node, x].double()
            yes = u * q * left < (p - taken * q).clamp_min(0)
            no = child & ~yes
            taken = torch.where(no, taken + left, taken)
            rest = (s["target"][seq, node].double() - taken[:, None] * s["draft"][seq, node].double()).clamp_min(0).sum(1)
            left = torch.where(no, rest, left)
        else:
            p = torch.where(gone[seq, x], 0.0, p)
            yes = u * left < p
            no = child & ~yes
            left = torch.where(no, (left - p).clamp_min(0), left)
            gone[seq, x] |= no
        yes = child & yes
        node = torch.where(yes, c, node)
        path[seq, count.clamp_max(new - 1)] = torch.where(yes, c, path[seq, count.clamp_max(new - 1)])
        count = count + yes
        taken, left = torch.where(yes, 0.0, taken), torch.where(yes, 1.0, left)
        gone &= ~yes[:, None]
    weight = s["target"][seq, node].double()
    if s["draft"] is not None:
        rest = (weight - taken[:, None] * s["draft"][seq, node].double()).clamp_min(0)
    else:
        rest = torch.where(gone, 0.0, weight)
    weight = torch.where(rest.sum(1, keepdim=True) > 0, rest, weight)
    total = weight.cumsum(1)
    token = (total <= uniform[:, :1] * total[:, -1:]).sum(1)
    return path.to(torch.int32), count.to(torch.int32), token.to(torch.int32)


def _keep(cache, scale, s):
    page, first, count = s["page"], s["lengths"][s["seq"]].long()[:, None], s["count"][s["seq"]].long()[:, None]
    at = s["slot"][:, None] * page + torch.arange(page, device="cuda")      # positions of the drafted rows' pages
    moved, before = (at >= first) & (at < first + count), at < first
    node = s["path"][s["seq"][:, None], (at - first).clamp(0, s["new"] - 1)].long()
    source = torch.where(moved, first + node, at)
    from_page = s["pages"][s["seq"][:, None], (source // page).clamp_max(s["pages"].shape[1] - 1)].long()
    was = scale[from_page]                                                  # [page][row][head]
    now = torch.where((moved | before)[:, :, None], was, -math.inf).amax(1)
    some = (moved | before).any(1)
    now = torch.where(some[:, None], now, scale[s["page_of"]])
    heads = torch.arange(s["heads"], device="cuda")[None, :, None]
    x = cache[from_page[:, None, :], heads, (source % page)[:, None, :]].float()
    x = torch.round(x * (was.transpose(1, 2) / torch.where(now > 0, now, 1.0)[:, :, None])[..., None])
    held = cache[s["page_of"]]
    cache[s["page_of"]] = torch.where((moved | before)[:, None, :, None], x, held.float()).to(torch.int8)
    scale[s["page_of"]] = now


def _read(cache, scale, s, out):
    at = s["first"][:, None].long() + torch.arange(s["new"], device="cuda")
    inside = (at < s["lengths"][:, None])
    slot = (at // s["page"]).clamp_max(s["pages"].shape[1] - 1)
    pages = torch.gather(s["pages"].long(), 1, slot)
    x = cache[pages[:, :, None], torch.arange(s["heads"], device="cuda"), (at % s["page"])[:, :, None]].float() * scale[pages][..., None]
    out.copy_(torch.where(inside[:, :, None, None], x, out.float()))


def _pages_values(cache, scale, pages):
    """What the 8-bit values of the pages stand for."""
    x = cache[pages]
    return torch.mul(x, scale[pages][:, :, None, None], out=torch.empty(x.shape, dtype=torch.bfloat16, device="cuda"))


def run(s):
    kind, b, new = s["kind"], s["batch"], s["new"]
    cache = [s[n] for n in ("k_cache", "v_cache", "k_scale", "v_scale", "pages")] if kind != "verify" else None
    if kind == "tree":
        if not own:
            return _tree(s)
        mask = torch.empty((b, new, -(-new // 32)), dtype=torch.int32, device="cuda")
        s["lib"].tree_mask(s["parents"], mask)
        out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
        s["lib"].tree_attention(s["q"], *cache, s["lengths"], mask, out, softmax_scale=s["softmax_scale"])
        return out, mask
    if kind == "verify":
        if not own:
            return _verify(s)
        path = torch.empty((b, new), dtype=torch.int32, device="cuda")
        count, token = (torch.empty(b, dtype=torch.int32, device="cuda") for _ in range(2))
        s["lib"].verify(s["target"], s["tokens"], s["parents"], s["uniform"], path, count, token, draft=s["draft"])
        return path, count, token
    if kind == "keep":
        if own:
            s["lib"].cache_keep(*cache, s["lengths"], s["path"], s["count"])
        else:
            _keep(s["k_cache"], s["k_scale"], s)
            _keep(s["v_cache"], s["v_scale"], s)
        p = s["page_of"]
        return {"k": _pages_values(s["k_cache"], s["k_scale"], p), "k_scale": s["k_scale"][p],
                "v": _pages_values(s["v_cache"], s["v_scale"], p), "v_scale": s["v_scale"][p]}
    if own:
        s["lib"].cache_read(*cache, s["first"], s["lengths"], s["k"], s["v"])
    else:
        _read(s["k_cache"], s["k_scale"], s, s["k"])
        _read(s["v_cache"], s["v_scale"], s, s["v"])
    return s["k"], s["v"]


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
    return {"tree": _exact_tree, "verify": _exact_verify, "keep": _exact_keep, "read": _exact_read}[case["kind"]](case, s)


def _exact_tree(case, s):
    new, g, lens = case["new"], case["group"], _lengths(case)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        pages = s["pages"][b, :-(-n // case["page"])].long()
        up = s["parents"][b].tolist()
        hidden = torch.ones((new, n), dtype=torch.bool)
        hidden[:, :n - new] = False
        for t in range(new):
            j = t
            while j >= 0:
                hidden[t, n - new + j] = False
                j = up[j]
        hidden = hidden.cuda()
        for h in range(case["heads"]):
            k = (s["k_cache"][pages, h].double() * s["k_scale"][pages, h].double()[:, None, None]).flatten(0, 1)[:n]
            v = (s["v_cache"][pages, h].double() * s["v_scale"][pages, h].double()[:, None, None]).flatten(0, 1)[:n]
            for i in range(h * g, h * g + g):
                z = (s["q"][b, :, i].double() @ k.T * s["softmax_scale"]).masked_fill(hidden, -math.inf)
                out[b, :, i] = torch.softmax(z, 1) @ v
    return out, None


def _exact_verify(case, s):
    new = case["new"]
    paths, counts, after = [], [], []
    for b in range(case["batch"]):
        up, x = s["parents"][b].tolist(), s["tokens"][b].tolist()
        u = [float(v) for v in s["uniform"][b].tolist()]
        path = [0]
        while True:
            n = path[-1]
            p = s["target"][b, n].double().cpu()
            q = s["draft"][b, n].double().cpu() if case["draft"] else None
            rest, total, found = p.clone(), 1.0, None
            for c in range(n + 1, new):
                if up[c] != n:
                    continue
                if u[c] * (float(q[x[c]]) if case["draft"] else 1.0) * total < float(rest[x[c]]):
                    found = c
                    break
                if case["draft"]:
                    rest = torch.clamp(rest - total * q, min=0)
                    total = float(rest.sum())
                else:
                    total -= float(rest[x[c]])
                    rest[x[c]] = 0
            if found is None:
                break
            path.append(found)
        if float(rest.sum()) <= 0:
            rest = p
        sums = rest.cumsum(0)
        after.append(int(torch.searchsorted(sums, u[0] * float(sums[-1]), right=True)))
        counts.append(len(path))
        paths.append(path + [-1] * (new - len(path)))
    return tuple(torch.tensor(v, dtype=torch.int32, device="cuda") for v in (paths, counts, after))


def _exact_keep(case, s):
    page, out = case["page"], {}
    for name in ("k", "v"):
        cache, scale = s[name + "_cache"].cpu(), s[name + "_scale"].cpu().double()
        table, path, count, lens = s["pages"].tolist(), s["path"].tolist(), s["count"].tolist(), _lengths(case)
        values, scales = [], []
        for (b, j), p in zip(_drafted_pages(case), s["page_of"].tolist()):
            rows, from_ = cache[p].double(), {}
            for r in range(page):
                at = j * page + r
                if at < lens[b]:
                    from_[r] = (p, r)
                elif at < lens[b] + count[b]:
                    to = lens[b] + path[b][at - lens[b]]
                    from_[r] = (table[b][to // page], to % page)
            now = scale[p]
            if from_:
                now = torch.stack([scale[k] for k in {v[0] for v in from_.values()}]).amax(0)
            for r, (k, i) in from_.items():
                rows[:, r] = torch.round(cache[k, :, i].double() * (scale[k] / now)[:, None])
            values.append(rows * now[:, None, None])
            scales.append(now)
        out[name], out[name + "_scale"] = torch.stack(values).cuda(), torch.stack(scales).cuda()
    return out


def _exact_read(case, s):
    out = []
    for name in ("k", "v"):
        x = torch.zeros(s[name].shape, dtype=torch.float64, device="cuda")
        for b, (n, first) in enumerate(zip(_lengths(case), _read_first(case))):
            pages = s["pages"][b, :-(-n // case["page"])].long()
            rows = s[name + "_cache"][pages].transpose(1, 2).double() * s[name + "_scale"][pages].double()[:, None, :, None]
            rows = rows.flatten(0, 1)[first:min(n, first + case["new"])]
            x[b, :rows.shape[0]] = rows
        out.append(x)
    return tuple(out)
