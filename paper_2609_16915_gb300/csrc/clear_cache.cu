// Appending keys and values to the paged 8-bit cache, a scale per page and head.
//
// A unit of work is one page of one sequence, one cached head, keys or values:
//   s' = max(s of the rows before the new ones, max|new| / 127)
//   old rows q' = rint(q (s / s')) where s' grew, new rows q = rint(x / s').
// The new rows are read twice (the second time from the cache), the old rows only where the scale
// grew.  Bound by reading the new values and writing their bytes; a decode step by its latency.
#include <stdint.h>

#include "clear.h"

namespace rosetta {

namespace {

__device__ __forceinline__ int8_t to_int8(float v) {
  return static_cast<int8_t>(__float2int_rn(fminf(fmaxf(v, -127.0f), 127.0f)));  // (a NaN gives -127, under a NaN scale)
}

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack {
  T v[VEC];
};

// WARPS of a unit: a block's four, or one for units of few values.  VEC: 4 consecutive dimensions an access
// where the strides keep them aligned, else 1.
template <typename T, int VEC, int WARPS>
__global__ void __launch_bounds__(128) append_kernel(const ClearAppendArgs a) {
  __shared__ float parts[4];
  constexpr uint32_t THREADS = 32 * WARPS;
  const uint32_t tid = threadIdx.x % THREADS;
  // heads and keys / values, four of them a block where a warp takes a unit
  const uint32_t unit = blockIdx.y * (4 / WARPS) + threadIdx.x / THREADS;
  const uint32_t kv = unit & 1u, head = unit >> 1;
  if (head >= a.heads) return;  // (whole warps; there is no barrier where a block has several units)
  const uint32_t b = blockIdx.z;
  const int64_t first = a.first[b];
  if (first < 0) return;
  const int64_t slot = first / a.page_tokens + blockIdx.x, row0 = slot * a.page_tokens, end = first + a.tokens;
  if (row0 >= end) return;
  int32_t page = -1;
  if (slot < a.table_pitch) page = a.page_table[static_cast<size_t>(b) * a.table_pitch + slot];
  if (page < 0 || static_cast<uint32_t>(page) >= a.pages) {
    if (tid == 0) atomicMax(a.err_flag, 1u);
    return;
  }
  const int64_t lo = first > row0 ? first : row0, hi = end < row0 + a.page_tokens ? end : row0 + a.page_tokens;
  const int64_t step = a.src_strides[kv][1], row = a.cache_strides[2];
  const T *src = static_cast<const T *>(a.src[kv]) + static_cast<int64_t>(b) * a.src_strides[kv][0] + (lo - first) * step +
                 static_cast<int64_t>(head) * a.src_strides[kv][2];
  int8_t *dst = a.cache[kv] + static_cast<int64_t>(page) * a.cache_strides[0] + static_cast<int64_t>(head) * a.cache_strides[1];
  const uint32_t packs = a.dim / VEC, old_rows = static_cast<uint32_t>(lo - row0);
  const uint32_t fresh = static_cast<uint32_t>(hi - lo) * packs;
  using P = Pack<T, VEC>;
  const auto load = [&](uint32_t i) { return *reinterpret_cast<const P *>(src + static_cast<int64_t>(i / packs) * step + i % packs * VEC); };
  float m = 0.0f;
  bool bad = false;  // a NaN or an infinity
  P kept;            // a thread's first pack, not read again
#pragma unroll 4
  for (uint32_t i = tid; i < fresh; i += THREADS) {
    const P x = load(i);
    if (i == tid) kept = x;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float v = fabsf(to_float(x.v[e]));
      bad |= !(v < __int_as_float(0x7f800000));
      m = fmaxf(m, v);
    }
  }
  if (bad) m = __int_as_float(0x7f800000);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  float *scale = a.scale[kv] + static_cast<size_t>(page) * a.heads + head;
  const float was = old_rows ? *scale : 0.0f;
  if constexpr (WARPS == 4) {
    if (threadIdx.x % 32 == 0) parts[threadIdx.x / 32] = m;
    __syncthreads();
    m = fmaxf(fmaxf(parts[0], parts[1]), fmaxf(parts[2], parts[3]));
  } else {
    __syncwarp();  // (the old scale is read before it is written)
  }
  // a non-finite maximum, or an old scale that is NaN, gives NaN
  const float now = m < __int_as_float(0x7f800000) && was == was ? fmaxf(was, m / 127.0f) : __int_as_float(0x7fc00000);
  const float div = now > 0.0f ? now : 1.0f;
  if (old_rows && now != was) {
    const float ratio = was / div;
    for (uint32_t i = tid; i < old_rows * packs; i += THREADS) {
      Pack<int8_t, VEC> *p = reinterpret_cast<Pack<int8_t, VEC> *>(dst + static_cast<int64_t>(i / packs) * row + i % packs * VEC);
      Pack<int8_t, VEC> v = *p;
#pragma unroll
      for (int e = 0; e < VEC; ++e) v.v[e] = to_int8(static_cast<float>(v.v[e]) * ratio);
      *p = v;
    }
  }
#pragma unroll 4
  for (uint32_t i = tid; i < fresh; i += THREADS) {
    const P x = i == tid ? kept : load(i);
    Pack<int8_t, VEC> v;
#pragma unroll
    for (int e = 0; e < VEC; ++e) v.v[e] = to_int8(to_float(x.v[e]) / div);
    *reinterpret_cast<Pack<int8_t, VEC> *>(dst + static_cast<int64_t>(old_rows + i / packs) * row + i % packs * VEC) = v;
  }
  if (tid == 0) *scale = now;
}

template <typename T, int VEC>
cudaError_t launch_vec(const ClearAppendArgs &a, cudaStream_t s) {
  const uint32_t most = (a.page_tokens - 1 + a.tokens - 1) / a.page_tokens + 1;  // pages a sequence's tokens can touch
  // a warp a unit while it has a pack or two a lane: a step of 256 sequences, 8 heads of 128
  if (a.tokens * a.dim <= 64u * VEC)
    append_kernel<T, VEC, 1><<<dim3(most, (2 * a.heads + 3) / 4, a.batch), 128, 0, s>>>(a);
  else
    append_kernel<T, VEC, 4><<<dim3(most, 2 * a.heads, a.batch), 128, 0, s>>>(a);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_type(const ClearAppendArgs &a, cudaStream_t s) {
  // (dimensions and cache strides are multiples of 4, the caches 4-byte aligned)
  uintptr_t src = 0;
  int64_t strides = 0;
  for (int kv = 0; kv < 2; ++kv) {
    src |= reinterpret_cast<uintptr_t>(a.src[kv]);
    for (int i = 0; i < 3; ++i) strides |= a.src_strides[kv][i];
  }
  return src % (4 * sizeof(T)) == 0 && strides % 4 == 0 ? launch_vec<T, 4>(a, s) : launch_vec<T, 1>(a, s);
}

}  // namespace

cudaError_t launch_clear_append(const ClearAppendArgs &a, int type, cudaStream_t s) {
  if (type == kOutF32) return launch_type<float>(a, s);
  if (type == kOutF16) return launch_type<__half>(a, s);
  return launch_type<__nv_bfloat16>(a, s);
}

}  // namespace rosetta
