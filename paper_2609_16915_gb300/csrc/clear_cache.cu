// Appending keys and values to the paged 8-bit cache, a scale per page and head.
//
// A unit of work is one page of one sequence, one cached head, keys or values:
//   s' = max(s of the rows before the new ones, max|new| / 127)
//   old rows q' = rint(q (s / s')) where s' grew, new rows q = rint(x / s').
// One block per unit: the new rows are read twice (the second time from the
// cache), the old rows only where the scale grew.
#include <stdint.h>

#include "clear.h"

namespace rosetta {

namespace {

__device__ __forceinline__ int8_t to_int8(float v) {
  return static_cast<int8_t>(__float2int_rn(fminf(fmaxf(v, -127.0f), 127.0f)));  // (a NaN gives -127, under a NaN scale)
}

template <typename T>
__global__ void __launch_bounds__(128) append_kernel(const ClearAppendArgs a) {
  __shared__ float parts[4];
  const uint32_t kv = blockIdx.y & 1u, head = blockIdx.y >> 1;
  const uint32_t b = blockIdx.z;
  const int64_t first = a.first[b];
  if (first < 0) return;
  const int64_t slot = first / a.page_tokens + blockIdx.x, row0 = slot * a.page_tokens, end = first + a.tokens;
  if (row0 >= end) return;
  if (slot >= a.table_pitch) {
    if (threadIdx.x == 0) atomicMax(a.err_flag, 1u);
    return;
  }
  const int32_t page = a.page_table[static_cast<size_t>(b) * a.table_pitch + slot];
  if (page < 0 || static_cast<uint32_t>(page) >= a.pages) {
    if (threadIdx.x == 0) atomicMax(a.err_flag, 1u);
    return;
  }
  const int64_t lo = first > row0 ? first : row0, hi = end < row0 + a.page_tokens ? end : row0 + a.page_tokens;
  const T *src = static_cast<const T *>(a.src[kv]) + static_cast<int64_t>(b) * a.src_strides[kv][0] +
                 (lo - first) * a.src_strides[kv][1] + static_cast<int64_t>(head) * a.src_strides[kv][2];
  int8_t *dst = a.cache[kv] + static_cast<int64_t>(page) * a.cache_strides[0] + static_cast<int64_t>(head) * a.cache_strides[1];
  const uint32_t fresh = static_cast<uint32_t>(hi - lo) * a.dim, old_rows = static_cast<uint32_t>(lo - row0);
  float m = 0.0f;
  bool bad = false;  // a NaN or an infinity
  for (uint32_t i = threadIdx.x; i < fresh; i += blockDim.x) {
    const float v = fabsf(to_float(src[static_cast<int64_t>(i / a.dim) * a.src_strides[kv][1] + i % a.dim]));
    bad |= !(v < __int_as_float(0x7f800000));
    m = fmaxf(m, v);
  }
  if (bad) m = __int_as_float(0x7f800000);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (threadIdx.x % 32 == 0) parts[threadIdx.x / 32] = m;
  float *scale = a.scale[kv] + static_cast<size_t>(page) * a.heads + head;
  const float was = old_rows ? *scale : 0.0f;
  __syncthreads();
  m = fmaxf(fmaxf(parts[0], parts[1]), fmaxf(parts[2], parts[3]));
  // a non-finite maximum, or an old scale that is NaN, gives NaN
  const float now = m < __int_as_float(0x7f800000) && was == was ? fmaxf(was, m / 127.0f) : __int_as_float(0x7fc00000);
  const float div = now > 0.0f ? now : 1.0f;
  if (old_rows && now != was) {
    const float ratio = was / div;
    for (uint32_t i = threadIdx.x; i < old_rows * a.dim; i += blockDim.x) {
      int8_t *p = dst + static_cast<int64_t>(i / a.dim) * a.cache_strides[2] + i % a.dim;
      *p = to_int8(static_cast<float>(*p) * ratio);
    }
  }
  for (uint32_t i = threadIdx.x; i < fresh; i += blockDim.x) {
    const float v = to_float(src[static_cast<int64_t>(i / a.dim) * a.src_strides[kv][1] + i % a.dim]);
    dst[static_cast<int64_t>(old_rows + i / a.dim) * a.cache_strides[2] + i % a.dim] = to_int8(v / div);
  }
  if (threadIdx.x == 0) *scale = now;
}

}  // namespace

cudaError_t launch_clear_append(const ClearAppendArgs &a, int type, cudaStream_t s) {
  const uint32_t most = (a.page_tokens - 1 + a.tokens - 1) / a.page_tokens + 1;  // pages a sequence's tokens can touch
  const dim3 grid(most, 2 * a.heads, a.batch);
  if (type == kOutF32)
    append_kernel<float><<<grid, 128, 0, s>>>(a);
  else if (type == kOutF16)
    append_kernel<__half><<<grid, 128, 0, s>>>(a);
  else
    append_kernel<__nv_bfloat16><<<grid, 128, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace rosetta
