// Appending keys and values to the paged 8-bit cache, a scale per page and head.
//
// A unit of work is one page of one sequence, one cached head, keys or values:
//   s' = max(s of the rows before the new ones, max|new| / 127)
//   old rows q' = rint(q (s / s')) where s' grew, new rows q = rint(x / s').
// The new rows are read once (what a thread cannot keep in registers, twice), the old rows only where the scale
// grew.  Bound by the latency of a unit's chain (the first position, the values, their maximum, the bytes out): 8 sequences of
// 2043 tokens, 8 heads of 128, pages of 32, float16 23.4 us, 4.3 TB/s; a decode step of 256 sequences 3.9 us.
#include <stdint.h>

#include "clear.h"
#include "pairs.cuh"

namespace rosetta {

namespace {

// The low byte of rint(v), |v| < 2^22: v + 1.5 * 2^23 has it in its last bits (ties to even).
constexpr float kMagic = 12582912.0f;

__device__ __forceinline__ uint32_t rint_bits(float v) { return __float_as_uint(v + kMagic); }

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack {
  T v[VEC];
};

// rint(x / div) in [-127, 127], in the low byte.  Past 127 where x is so small that div = max / 127 has been rounded to few bits
// or none (below 2^-142; the quotient by multiplication is no number there).
__device__ __forceinline__ uint32_t divided(float x, float div) {
  const float v = x / div;
  return rint_bits(v > 127.0f ? 127.0f : v < -127.0f ? -127.0f : v);  // (a NaN stays one)
}

// rint(x / div) of a pack, bytes in order.  The quotient by multiplication is off by less than 1e-4 (|x / div| <= 127 and
// 2^-22 of it): only where it lies that close to a half, or is no number, the division decides.
template <int VEC>
__device__ __forceinline__ Pack<int8_t, VEC> quotients(const float (&x)[VEC], float div, float inv) {
  Pack<int8_t, VEC> out;
  uint32_t bits[VEC];
  if constexpr (VEC == 1) {
    bits[0] = divided(x[0], div);
    out.v[0] = static_cast<int8_t>(bits[0]);
  } else {
    const uint64_t inv2 = pair_of(inv, inv), minus2 = pair_of(-inv, -inv), magic2 = pair_of(kMagic, kMagic), back2 = pair_of(-kMagic, -kMagic);
    float far = 0.0f;  // the furthest from a whole number
#pragma unroll
    for (int e = 0; e < VEC; e += 2) {
      const uint64_t v = pair_of(x[e], x[e + 1]), t = fma2(v, inv2, magic2);
      const float2 off = floats_of(fma2(v, minus2, add2(t, back2))), whole = floats_of(t);
      far = max3_magnitude(far, off.x, off.y);
      bits[e] = __float_as_uint(whole.x);
      bits[e + 1] = __float_as_uint(whole.y);
    }
    if (!(far < 0.4999f)) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) bits[e] = divided(x[e], div);
    }
    uint32_t *words = reinterpret_cast<uint32_t *>(&out);
#pragma unroll
    for (int e = 0; e < VEC; e += 4)
      words[e / 4] = __byte_perm(__byte_perm(bits[e], bits[e + 1], 0x0040), __byte_perm(bits[e + 2], bits[e + 3], 0x0040), 0x5410);
  }
  return out;
}

// The largest magnitude of packs, as bits: of a 16-bit type two at a time.  A NaN or an infinity is larger than every number.
template <typename T, int VEC>
__device__ __forceinline__ void largest(const Pack<T, VEC> &x, uint32_t &m) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) m = max(m, __float_as_uint(x.v[e]) & 0x7fffffffu);
  } else if constexpr (VEC == 1) {
    m = max(m, static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(&x) & 0x7fffu));
  } else {
    const uint32_t *words = reinterpret_cast<const uint32_t *>(&x);
#pragma unroll
    for (int e = 0; e < VEC / 2; ++e) m = __vmaxu2(m, words[e] & 0x7fff7fffu);
  }
}
template <typename T, int VEC>
__device__ __forceinline__ float largest_value(uint32_t m) {
  if constexpr (sizeof(T) == 4) {
    return m < 0x7f800000u ? __uint_as_float(m) : __int_as_float(0x7f800000);
  } else {
    const uint16_t bits = static_cast<uint16_t>(VEC == 1 ? m : max(m & 0xffffu, m >> 16));
    const float v = to_float(*reinterpret_cast<const T *>(&bits));
    return v < __int_as_float(0x7f800000) ? v : __int_as_float(0x7f800000);
  }
}

// A thread's walk over the packs of consecutive rows: every `threads`-th, with its places in the source and in the cache.
struct Walk {
  uint32_t row, col, packs, rows_on, cols_on;
  int64_t src, dst, src_step, dst_step;
  uint32_t vec;
  __device__ Walk(uint32_t at, uint32_t packs_, uint32_t threads, uint32_t vec_, int64_t src_step_, int64_t dst_step_)
      : row(at / packs_), col(at % packs_), packs(packs_), rows_on(threads / packs_), cols_on(threads % packs_),
        src(row * src_step_ + col * vec_), dst(row * dst_step_ + col * vec_), src_step(src_step_), dst_step(dst_step_), vec(vec_) {}
  __device__ void on() {
    row += rows_on;
    src += rows_on * src_step;
    dst += rows_on * dst_step;
    if (cols_on == 0) return;
    col += cols_on;
    src += cols_on * vec;
    dst += cols_on * vec;
    if (col >= packs) {
      col -= packs;
      ++row;
      src += src_step - packs * vec;
      dst += dst_step - packs * vec;
    }
  }
};

// WARPS of a unit: one (four units a block), four, or sixteen for large pages.  VEC consecutive dimensions an access.
// KEPT packs of new values stay in a thread's registers between the two passes.
template <typename T, int VEC, int WARPS, int KEPT>
__global__ void __launch_bounds__(WARPS == 16 ? 512 : 128) append_kernel(const ClearAppendArgs a) {
  __shared__ float parts[16];
  constexpr uint32_t THREADS = 32 * WARPS;
  const uint32_t tid = threadIdx.x % THREADS;
  // heads and keys / values, four of them a block where a warp takes a unit
  const uint32_t unit = blockIdx.y * (WARPS == 1 ? 4 : 1) + threadIdx.x / THREADS;
  const uint32_t kv = unit & 1u, head = unit >> 1;
  if (head >= a.heads) return;  // (whole warps; there is no barrier where a block has several units)
  const uint32_t b = blockIdx.z;
  const int64_t first = a.first[b];
  if (first < 0) return;
  const int64_t slot = static_cast<uint32_t>(first) / a.page_tokens + static_cast<int64_t>(blockIdx.x), row0 = slot * a.page_tokens, end = first + a.tokens;
  if (row0 >= end) return;
  int32_t page = -1;
  if (slot < a.table_pitch) page = a.page_table[static_cast<size_t>(b) * a.table_pitch + slot];
  const int64_t lo = first > row0 ? first : row0, hi = end < row0 + a.page_tokens ? end : row0 + a.page_tokens;
  const int64_t step = a.src_strides[kv][1], line = a.cache_strides[2];
  const T *src = static_cast<const T *>(a.src[kv]) + static_cast<int64_t>(b) * a.src_strides[kv][0] + (lo - first) * step +
                 static_cast<int64_t>(head) * a.src_strides[kv][2];
  const uint32_t packs = a.dim / VEC, old_rows = static_cast<uint32_t>(lo - row0), new_rows = static_cast<uint32_t>(hi - lo);
  using P = Pack<T, VEC>;
  const auto load = [&](const Walk &w) { return *reinterpret_cast<const P *>(src + w.src); };
  uint32_t bits = 0;
  const auto take = [&](const P &x) { largest<T, VEC>(x, bits); };
  const Walk begin(tid, packs, THREADS, VEC, step, line);
  P kept[KEPT];
  Walk w = begin;
#pragma unroll
  for (int i = 0; i < KEPT; ++i, w.on())
    if (w.row < new_rows) kept[i] = load(w);
  Walk rest = w;
  // (the values do not wait for the page)
  if (page < 0 || static_cast<uint32_t>(page) >= a.pages) {
    if (tid == 0) atomicMax(a.err_flag, 1u);
    return;
  }
  int8_t *dst = a.cache[kv] + static_cast<int64_t>(page) * a.cache_strides[0] + static_cast<int64_t>(head) * a.cache_strides[1];
  float *scale = a.scale[kv] + static_cast<size_t>(page) * a.heads + head;
  const float was = old_rows ? *scale : 0.0f;
  w = begin;
#pragma unroll
  for (int i = 0; i < KEPT; ++i, w.on())
    if (w.row < new_rows) take(kept[i]);
  for (w = rest; w.row < new_rows; w.on()) take(load(w));
  float m = largest_value<T, VEC>(bits);  // (infinite where a value is not a number)
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if constexpr (WARPS > 1) {
    if (threadIdx.x % 32 == 0) parts[threadIdx.x / 32] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WARPS; ++i) m = fmaxf(m, parts[i]);
  } else {
    __syncwarp();  // (the old scale is read before it is written)
  }
  // a non-finite maximum, or an old scale that is NaN, gives NaN
  const float now = m < __int_as_float(0x7f800000) && was == was ? fmaxf(was, m / 127.0f) : __int_as_float(0x7fc00000);
  const float div = now > 0.0f ? now : 1.0f, inv = 1.0f / div;
  if (old_rows && now != was) {
    const float ratio = was / div;
    for (w = begin; w.row < old_rows; w.on()) {
      Pack<int8_t, VEC> *p = reinterpret_cast<Pack<int8_t, VEC> *>(dst + w.dst);
      Pack<int8_t, VEC> v = *p;
#pragma unroll
      for (int e = 0; e < VEC; ++e) v.v[e] = static_cast<int8_t>(rint_bits(static_cast<float>(v.v[e]) * ratio));
      *p = v;
    }
  }
  int8_t *fresh = dst + static_cast<int64_t>(old_rows) * line;
  const auto put = [&](const Walk &w, const P &x) {
    float v[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = to_float(x.v[e]);
    *reinterpret_cast<Pack<int8_t, VEC> *>(fresh + w.dst) = quotients<VEC>(v, div, inv);
  };
  w = begin;
#pragma unroll
  for (int i = 0; i < KEPT; ++i, w.on())
    if (w.row < new_rows) put(w, kept[i]);
  for (w = rest; w.row < new_rows; w.on()) put(w, load(w));
  if (tid == 0) *scale = now;
}

template <typename T, int VEC>
cudaError_t launch_vec(const ClearAppendArgs &a, cudaStream_t s) {
  const uint32_t most = (a.page_tokens - 1 + a.tokens - 1) / a.page_tokens + 1;  // pages a sequence's tokens can touch
  // as few threads as keep a unit in registers (each pack kept costs its index work, used or not): single tokens a warp
  // with two packs a lane; 16 rows of 128 two a thread, 32 rows four (8 x 2043 tokens 23 us, a third more with eight)
  const uint64_t packs = static_cast<uint64_t>(a.tokens < a.page_tokens ? a.tokens : a.page_tokens) * a.dim / VEC;
  const dim3 units(most, 2 * a.heads, a.batch);
  if (packs <= 64)
    append_kernel<T, VEC, 1, 2><<<dim3(most, (2 * a.heads + 3) / 4, a.batch), 128, 0, s>>>(a);
  else if (packs <= 256)
    append_kernel<T, VEC, 4, 2><<<units, 128, 0, s>>>(a);
  else if (packs <= 512)
    append_kernel<T, VEC, 4, 4><<<units, 128, 0, s>>>(a);
  else
    append_kernel<T, VEC, 16, 4><<<units, 512, 0, s>>>(a);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_type(const ClearAppendArgs &a, cudaStream_t s) {
  uintptr_t src = 0, dst = static_cast<uintptr_t>(a.cache_strides[0] | a.cache_strides[1] | a.cache_strides[2] | a.dim);
  int64_t strides = 0;
  for (int kv = 0; kv < 2; ++kv) {
    src |= reinterpret_cast<uintptr_t>(a.src[kv]);
    dst |= reinterpret_cast<uintptr_t>(a.cache[kv]);
    for (int i = 0; i < 3; ++i) strides |= a.src_strides[kv][i];
  }
  constexpr int WIDE = 16 / sizeof(T);
  if (src % 16 == 0 && strides % WIDE == 0 && dst % WIDE == 0) return launch_vec<T, WIDE>(a, s);
  // (dimensions and cache strides are multiples of 4, the caches 4-byte aligned)
  return src % (4 * sizeof(T)) == 0 && strides % 4 == 0 ? launch_vec<T, 4>(a, s) : launch_vec<T, 1>(a, s);
}

}  // namespace

cudaError_t launch_clear_append(const ClearAppendArgs &a, int type, cudaStream_t s) {
  if (type == kOutF32) return launch_type<float>(a, s);
  if (type == kOutF16) return launch_type<__half>(a, s);
  return launch_type<__nv_bfloat16>(a, s);
}

}  // namespace rosetta
