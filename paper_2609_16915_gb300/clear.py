"""The decoder layer around a bootstrapped table, in the clear (rosetta_clear_*).

8-bit activations, weights and cache: the operators that a table's range and precision
are judged with, and that give the message codes which are encrypted.  Argument checks
and marshalling only; formulas, types and sizes stand in include/rosetta.h.  Buffers are
CUDA tensors that the caller allocates; rows may be slices of wider buffers, with the last
dimension contiguous.  Outputs are passed in and returned.
"""

from __future__ import annotations

import ctypes
import functools

import torch

from . import _check, load

_FLOATS = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_Strides = ctypes.c_int64 * 3


# (the second creates a Stream object each time)
_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda d: torch.cuda.current_stream(d).cuda_stream)


@functools.lru_cache(maxsize=256)
def _strides(stride):
    """The first three strides as a C array (of which only the values matter)."""
    return _Strides(*stride[:3])


def packed_size(channels: int, inner: int) -> int:
    """Bytes of packed weights: tiles of 128 channels x 64 inputs."""
    return -(-channels // 128) * -(-inner // 64) * 8192


class PackedWeights:
    """int8 weights [channels][inner] laid out for Clear.linear.  `data` comes from torch's allocator on the stream that
    packed them; the streams that have used it since are recorded with it, so that its memory is not given away under them."""

    def __init__(self, data, channels: int, inner: int, stream: int | None = None):
        self.data, self.channels, self.inner = data, channels, inner
        self.streams = {stream}

    def used_on(self, stream: int):
        if stream not in self.streams:
            self.data.record_stream(torch.cuda.ExternalStream(stream, self.data.device))
            self.streams.add(stream)


def _need(ok, what: str):
    if not ok:
        raise ValueError(what)


def _float_type(name, t, dims):
    """Number of the tensor's float type."""
    kind = _FLOATS.get(t.dtype)
    if kind is None or t.dim() != dims:
        raise ValueError(f"{name} must be a tensor of floats with {dims} dimensions")
    return kind


class Clear:
    """One workspace on one device; its calls are ordered on one stream (see the header)."""

    def __init__(self, device: int = 0, workspace_bytes: int = 0):
        h = ctypes.c_void_p()
        self._L = load()
        _check("rosetta_clear_init", self._L.rosetta_clear_init(ctypes.byref(h), device, workspace_bytes))
        self._h, self.device = h, device

    def close(self):
        if getattr(self, "_h", None):
            self._L.rosetta_clear_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- checks shared by the calls ----
    def _at(self, name, t, dtype, shape, contiguous=False):
        """Address of tensor `t`: on this device, of the type and shape, last dimension contiguous."""
        if (t.get_device() == self.device and t.dtype == dtype and t.shape == shape
                and (t.is_contiguous() or (not contiguous and t.stride(-1) == 1))):
            return t.data_ptr()
        _need(t.get_device() == self.device, f"{name} must be a tensor on CUDA device {self.device}")
        _need(t.dtype == dtype, f"{name} must be {dtype}, not {t.dtype}")
        _need(t.shape == shape, f"{name} must have shape {shape}, not {tuple(t.shape)}")
        _need(not contiguous, f"{name} must be contiguous")
        _need(shape[-1] <= 1, f"the last dimension of {name} must be contiguous")
        return t.data_ptr()

    def _rows(self, name, t, dtype, rows, width):
        """(address, pitch) of a matrix."""
        at = self._at(name, t, dtype, (rows, width))
        pitch = t.stride(0) if rows > 1 else width
        if pitch < width:
            raise ValueError(f"the rows of {name} must not overlap")
        return at, pitch

    def _stream(self, stream):
        if stream is None:
            return _current_stream(self.device)
        return getattr(stream, "cuda_stream", stream)

    # ---- the C entry points ----
    def rosetta_clear_norm(self, x, gamma, q, scale, residual=None, sum_out=None, eps=1e-6, stream=None):
        """q, scale of the root-mean-square norm of x (+ residual) [tokens][width]; sum_out receives the sum."""
        kind, dt = _float_type("x", x, 2), x.dtype
        t, w = x.shape
        xp, xs = self._rows("x", x, dt, t, w)
        rp, rs = self._rows("residual", residual, dt, t, w) if residual is not None else (None, 0)
        sp, ss = self._rows("sum_out", sum_out, dt, t, w) if sum_out is not None else (None, 0)
        qp, qs = self._rows("q", q, torch.int8, t, w)
        _check("rosetta_clear_norm", self._L.rosetta_clear_norm(
            self._h, kind, xp, xs, rp, rs, self._at("gamma", gamma, torch.float32, (w,)), eps, t, w, sp, ss, qp, qs,
            self._at("scale", scale, torch.float32, (t,)), self._stream(stream)))
        return q, scale

    def rosetta_clear_packed_bytes(self, channels, inner):
        return self._L.rosetta_clear_packed_bytes(channels, inner)

    def rosetta_clear_pack_weights(self, weight, stream=None):
        """int8 weights [channels][inner] in the linear products' layout."""
        _need(weight.dim() == 2, "weight must be a matrix")
        n, k = weight.shape
        wp, ws = self._rows("weight", weight, torch.int8, n, k)
        size = self._L.rosetta_clear_packed_bytes(n, k)
        _need(size, f"weights of {n} x {k} are out of range")
        stream = self._stream(stream)
        # (from the pool of the stream that writes it: a block of another stream's may still be in use there)
        other = stream != _current_stream(self.device)
        with torch.cuda.stream(torch.cuda.ExternalStream(stream, weight.device) if other else None):
            data = torch.empty(size, dtype=torch.int8, device=weight.device)
        _check("rosetta_clear_pack_weights", self._L.rosetta_clear_pack_weights(self._h, wp, ws, n, k, data.data_ptr(), stream))
        return PackedWeights(data, n, k, stream)

    def _linear(self, q, scale, weights, w_scale, bias, stream):
        _need(isinstance(weights, PackedWeights), "weights must come from pack_weights")
        _need(q.dim() == 2, "q must be a matrix")
        t, n, k = q.shape[0], weights.channels, weights.inner
        qp, qs = self._rows("q", q, torch.int8, t, k)
        data = self._at("weights", weights.data, torch.int8, tuple(weights.data.shape), True)
        _need(weights.data.numel() >= packed_size(n, k), f"weights must hold {packed_size(n, k)} bytes for {n} x {k}")
        args = (self._h, qp, qs, self._at("scale", scale, torch.float32, (t,)), t, data,
                self._at("w_scale", w_scale, torch.float32, (n,)),
                None if bias is None else self._at("bias", bias, torch.float32, (n,)), n, k)
        stream = self._stream(stream)
        weights.used_on(stream)
        return t, n, args, stream

    def rosetta_clear_linear(self, q, scale, weights, w_scale, out, bias=None, stream=None):
        """out [tokens][channels] = (q weights^T) scale w_scale + bias."""
        t, n, args, stream = self._linear(q, scale, weights, w_scale, bias, stream)
        kind = _float_type("out", out, 2)
        op, os = self._rows("out", out, out.dtype, t, n)
        _check("rosetta_clear_linear", self._L.rosetta_clear_linear(*args, kind, op, os, stream))
        return out

    def rosetta_clear_linear_codes(self, q, scale, weights, w_scale, code, bits, lo, hi, bias=None, table=None,
                                   values=None, stream=None):
        """The product's message codes (uint8) of a 2^bits-entry table on [lo, hi], and that table's int8 values."""
        t, n, args, stream = self._linear(q, scale, weights, w_scale, bias, stream)
        _need((table is None) == (values is None), "table and values go together")
        cp, cs = self._rows("code", code, torch.uint8, t, n)
        tp = self._at("table", table, torch.int8, (1 << bits,)) if table is not None else None
        vp, vs = self._rows("values", values, torch.int8, t, n) if values is not None else (None, 0)
        _check("rosetta_clear_linear_codes", self._L.rosetta_clear_linear_codes(
            *args, bits, lo, hi, cp, cs, tp, vp, vs, stream))
        return code, values

    def _strided(self, name, t, dtype, shape):
        """(address, strides) of a tensor [.][.][.][dim]."""
        return self._at(name, t, dtype, shape), _strides(t.stride())

    def _cache(self, k_cache, v_cache, k_scale, v_scale, page_table, batch, heads, dim):
        _need(k_cache.dim() == 4, "k_cache must be [pages][heads][page tokens][dim]")
        pages, page = k_cache.shape[0], k_cache.shape[2]
        shape = (pages, heads, page, dim)
        kp, strides = self._strided("k_cache", k_cache, torch.int8, shape)
        vp = self._at("v_cache", v_cache, torch.int8, shape)
        _need(k_cache.stride() == v_cache.stride(), "k_cache and v_cache must have the same strides")
        _need(page_table.dim() == 2, "page_table must be [batch][pages of a sequence]")
        each = page_table.shape[1]
        tp, pitch = self._rows("page_table", page_table, torch.int32, batch, each)
        _need(pitch == each, "page_table must be contiguous")
        return (kp, vp, strides, self._at("k_scale", k_scale, torch.float32, (pages, heads), True),
                self._at("v_scale", v_scale, torch.float32, (pages, heads), True), pages, page, tp, each)

    def rosetta_clear_cache_append(self, k, v, k_cache, v_cache, k_scale, v_scale, page_table, first, stream=None):
        """Append k, v [batch][tokens][heads][dim] at positions first[b] .. to the caches [pages][heads][page][dim]."""
        kind = _float_type("k", k, 4)
        shape = b, t, h, d = tuple(k.shape)
        kp, ks = self._strided("k", k, k.dtype, shape)
        vp, vs = self._strided("v", v, k.dtype, shape)
        cache = self._cache(k_cache, v_cache, k_scale, v_scale, page_table, b, h, d)
        _check("rosetta_clear_cache_append", self._L.rosetta_clear_cache_append(
            self._h, kind, kp, ks, vp, vs, b, t, h, d, *cache, self._at("first", first, torch.int32, (b,)),
            self._stream(stream)))

    def rosetta_clear_attention(self, q, k_cache, v_cache, k_scale, v_scale, page_table, lengths, out,
                                softmax_scale=None, stream=None):
        """Causal attention of q [batch][tokens][query heads][dim] over the cache; softmax_scale: dim^-1/2 unless given."""
        kind = _float_type("q", q, 4)
        shape = b, t, hq, d = tuple(q.shape)
        heads = k_cache.shape[1]
        _need(hq and heads and hq % heads == 0, "the query heads must be a multiple of the cached heads")
        qp, qs = self._strided("q", q, q.dtype, shape)
        op, os = self._strided("out", out, q.dtype, shape)
        cache = self._cache(k_cache, v_cache, k_scale, v_scale, page_table, b, heads, d)
        _check("rosetta_clear_attention", self._L.rosetta_clear_attention(
            self._h, kind, qp, qs, b, t, heads, hq // heads, d, *cache,
            self._at("lengths", lengths, torch.int32, (b,)), d ** -0.5 if softmax_scale is None else softmax_scale, op, os,
            self._stream(stream)))
        return out

    def rosetta_clear_sync_status(self, stream=None):
        _check("rosetta_clear_sync_status", self._L.rosetta_clear_sync_status(self._h, self._stream(stream)))

    # short aliases
    norm = rosetta_clear_norm
    packed_bytes = rosetta_clear_packed_bytes
    pack_weights = rosetta_clear_pack_weights
    linear = rosetta_clear_linear
    linear_codes = rosetta_clear_linear_codes
    cache_append = rosetta_clear_cache_append
    attention = rosetta_clear_attention
    sync_status = rosetta_clear_sync_status
