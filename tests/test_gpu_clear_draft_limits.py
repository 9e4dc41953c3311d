"""Limits of the C entry points for drafted tokens: a call that works, then the same with one argument out of range at a time,
each refused before anything is launched."""

import ctypes

import pytest
import torch

import paper_2609_16915_gb300 as R

pytestmark = pytest.mark.gpu

B, T, V, H, G, DIM, PAGES, PAGE, EACH = 2, 5, 50, 2, 3, 64, 6, 16, 3
PITCH = (1 << 40) + 1


def strides(*s):
    return (ctypes.c_int64 * 3)(*s)


class At:
    """An address, kept with the tensor that it belongs to."""

    def __init__(self, t, more=0):
        self.t, self.at = t, t.data_ptr() + more


def values(args):
    return [a.at if isinstance(a, At) else a for a in args.values()]


def refuses(call, base, changes):
    h = ctypes.c_void_p()
    assert R.load().rosetta_clear_init(ctypes.byref(h), 0, 1 << 20) == 0
    f = getattr(R.load(), call)
    try:
        assert f(h, *values(base)) == 0
        assert R.load().rosetta_clear_sync_status(h, None) == 0
        for name, value in changes:
            assert name in base
            assert f(h, *values({**base, name: value})) == -1, (name, value)
        assert f(None, *values(base)) == -1
        assert f(h, *values(base)) == 0
        assert R.load().rosetta_clear_sync_status(h, None) == 0
    finally:
        R.load().rosetta_clear_destroy(h)


def zeros(*shape, dtype=torch.int32):
    return At(torch.zeros(shape, dtype=dtype, device="cuda"))


def cache_args():
    return dict(k_cache=zeros(PAGES, H, PAGE, DIM, dtype=torch.int8), v_cache=zeros(PAGES, H, PAGE, DIM, dtype=torch.int8),
                cache_strides=strides(H * PAGE * DIM, PAGE * DIM, DIM), k_scale=zeros(PAGES, H, dtype=torch.float32),
                v_scale=zeros(PAGES, H, dtype=torch.float32), pages=PAGES, page_tokens=PAGE,
                page_table=At(torch.arange(PAGES, dtype=torch.int32, device="cuda")), table_pitch=EACH)


def off(a, by):
    return At(a.t, by)


def cache_changes(c):
    out = [(n, None) for n in ("k_cache", "v_cache", "cache_strides", "k_scale", "v_scale", "page_table")]
    out += [(n, off(c[n], 2)) for n in ("k_cache", "v_cache", "k_scale", "v_scale", "page_table")]
    out += [("cache_strides", strides(*s)) for s in ((-H * PAGE * DIM, PAGE * DIM, DIM), (H * PAGE * DIM, PAGE * DIM, DIM - 4),
                                                     (H * PAGE * DIM, PAGE * DIM + 2, DIM), (PITCH + 3, PAGE * DIM, DIM))]
    return out + [("page_tokens", 0), ("page_tokens", 1025), ("table_pitch", (1 << 26) + 1), ("pages", 1 << 31), ("heads", 0), ("heads", 4097), ("dim", 0),
                  ("dim", 260), ("dim", 62)]


BATCHES = [("batch", 65536)]


def test_tree_mask():
    base = dict(parents=At(torch.full((B, T), -1, dtype=torch.int32, device="cuda")), parents_pitch=T, batch=B, tokens=T,
                mask=zeros(B, T, 1), mask_strides=strides(T, 1, 1), stream=None)
    refuses("rosetta_clear_tree_mask", base, BATCHES + [
        ("parents", None), ("parents", off(base["parents"], 2)), ("mask", None), ("mask", off(base["mask"], 2)), ("mask_strides", None),
        ("mask_strides", strides(-T, 1, 1)), ("mask_strides", strides(T, -1, 1)), ("mask_strides", strides(0, 1, 1)), ("mask_strides", strides(T, 0, 1)),
        ("mask_strides", strides(PITCH, 1, 1)), ("mask_strides", strides(T, PITCH, 1)), ("parents_pitch", -1), ("parents_pitch", PITCH),
        ("tokens", 1025), ("mask", base["parents"])])


def test_tree_attention():
    c = cache_args()
    qs = strides(T * H * G * DIM, H * G * DIM, DIM)
    base = dict(type=0, q=zeros(B, T, H * G, DIM, dtype=torch.float32), q_strides=qs, batch=B, tokens=T, heads=H, group=G, dim=DIM, **c,
                lengths=At(torch.tensor([20, 9], dtype=torch.int32, device="cuda")), mask=zeros(B, T, 1), mask_strides=strides(T, 1, 1),
                softmax_scale=0.125, out=zeros(B, T, H * G, DIM, dtype=torch.float32), out_strides=qs, stream=None)
    refuses("rosetta_clear_tree_attention", base, BATCHES + cache_changes(c) + [
        ("type", 3), ("type", -1), ("q", None), ("q", off(base["q"], 2)), ("out", None), ("out", off(base["out"], 2)), ("out", base["q"]),
        ("q_strides", None), ("q_strides", strides(-1, H * G * DIM, DIM)), ("q_strides", strides(1, PITCH, DIM)), ("out_strides", None),
        ("out_strides", strides(0, H * G * DIM, DIM)), ("out_strides", strides(T * H * G * DIM, -1, DIM)), ("group", 0), ("group", 129),
        ("tokens", 1025), ("lengths", None), ("lengths", off(base["lengths"], 2)), ("mask", None), ("mask", off(base["mask"], 2)),
        ("mask", off(base["out"], 0)), ("mask_strides", None), ("mask_strides", strides(-1, 1, 1)), ("mask_strides", strides(T, PITCH, 1)),
        ("softmax_scale", float("inf")), ("softmax_scale", float("nan"))])


@pytest.mark.parametrize("drawn", [True, False])
def test_verify(drawn):
    p = torch.full((B, T, V), 1 / V, device="cuda")
    base = dict(type=0, target=At(p), target_strides=strides(T * V, V, 1), draft=At(p.clone()) if drawn else None,
                draft_strides=strides(T * V, V, 1) if drawn else None, tokens=zeros(B, T), tokens_pitch=T,
                parents=At(torch.full((B, T), -1, dtype=torch.int32, device="cuda")), parents_pitch=T, uniform=zeros(B, T, dtype=torch.float32),
                uniform_pitch=T, batch=B, nodes=T, vocab=V, path=zeros(B, T), path_pitch=T, count=zeros(B), next=zeros(B), stream=None)
    changes = BATCHES + [("type", 3), ("target_strides", None), ("nodes", 1025), ("vocab", 0), ("vocab", (1 << 24) + 1), ("path_pitch", T - 1),
                         ("path_pitch", PITCH), ("path_pitch", -1), ("target_strides", strides(-1, V, 1)), ("target_strides", strides(T * V, PITCH, 1)),
                         ("path", base["tokens"]), ("count", base["next"]), ("next", base["uniform"]), ("path", base["parents"])]
    for n in ("target", "tokens", "parents", "uniform", "path", "count", "next"):
        changes += [(n, None), (n, off(base[n], 2))]
    for n in ("tokens_pitch", "parents_pitch", "uniform_pitch"):
        changes += [(n, -1), (n, PITCH)]
    if drawn:
        changes += [("draft", off(base["draft"], 2)), ("draft_strides", None), ("draft_strides", strides(T * V, -1, 1)), ("draft_strides", strides(PITCH, V, 1)),
                    ("path", base["draft"])]
    refuses("rosetta_clear_verify", base, changes)


def test_cache_keep():
    c = cache_args()
    base = dict(batch=B, tokens=T, heads=H, dim=DIM, **c, first=zeros(B), path=At(torch.arange(T, dtype=torch.int32, device="cuda").repeat(B, 1)), path_pitch=T,
                count=At(torch.full((B,), 2, dtype=torch.int32, device="cuda")), stream=None)
    changes = BATCHES + cache_changes(c) + [("tokens", 1025), ("path_pitch", -1), ("path_pitch", PITCH), ("v_cache", c["k_cache"]), ("v_scale", c["k_scale"]),
                                            ("cache_strides", strides(0, PAGE * DIM, DIM)), ("first", c["k_scale"]), ("count", c["v_cache"])]
    for n in ("first", "path", "count"):
        changes += [(n, None), (n, off(base[n], 2))]
    refuses("rosetta_clear_cache_keep", base, changes)


def test_cache_read():
    c = cache_args()
    ks = strides(T * H * DIM, H * DIM, DIM)
    base = dict(type=1, batch=B, tokens=T, heads=H, dim=DIM, **c, first=zeros(B), lengths=At(torch.tensor([5, 3], dtype=torch.int32, device="cuda")),
                k=zeros(B, T, H, DIM, dtype=torch.float16), k_strides=ks, v=zeros(B, T, H, DIM, dtype=torch.float16), v_strides=ks, stream=None)
    changes = BATCHES + cache_changes(c) + [("type", 3), ("tokens", (1 << 24) + 1), ("k", base["v"]), ("k", c["k_cache"]), ("v", off(c["k_cache"], 1024)),
                                            ("k_strides", strides(T * H * DIM, 0, DIM)), ("v_strides", strides(0, H * DIM, DIM))]
    for n in ("k", "v"):
        changes += [(n + "_strides", None), (n + "_strides", strides(-1, H * DIM, DIM)), (n + "_strides", strides(T * H * DIM, PITCH, DIM)), (n, None),
                    (n, off(base[n], 1))]
    for n in ("first", "lengths"):
        changes += [(n, None), (n, off(base[n], 2))]
    refuses("rosetta_clear_cache_read", base, changes)
