// Rows of the paged 8-bit cache moved and read back.
//
// Keeping: rows first + path[i] become rows first + i, under a page's scale
//   s' = max of the scales of the pages that its rows come from,  q' = rint(q (s / s')).
// A block takes one cached head of one sequence, keys or values, page after page: path[i] >= i and increasing, so what is
// written never lies before what is still to be read but for the rows in the block's registers.  Latency bound: a
// handful of rows each.
//
// Reading: out = q s[page][head].  Bound by its bytes, one read and two or four written for each value.
#include <stdint.h>

#include "clear.h"

namespace rosetta {

namespace {

// The low byte of rint(v), |v| < 2^22: v + 1.5 * 2^23 has it in its last bits (ties to even).
__device__ __forceinline__ int8_t rint_byte(float v) { return static_cast<int8_t>(__float_as_uint(v + 12582912.0f)); }

__device__ __forceinline__ char4 rescaled(char4 q, float ratio) {
  const auto one = [&](int8_t v) { return rint_byte(fminf(fmaxf(v * ratio, -128.0f), 127.0f)); };
  return make_char4(one(q.x), one(q.y), one(q.z), one(q.w));
}

constexpr uint32_t kKeepThreads = 128, kKept = 4;

__global__ void __launch_bounds__(kKeepThreads) keep_kernel(const ClearKeepArgs a) {
  extern __shared__ int32_t s_path[];  // then, of each row of the present page: where it comes from and under which scale
  const uint32_t kv = blockIdx.x & 1u, head = blockIdx.x >> 1, b = blockIdx.y, tid = threadIdx.x;
  const int64_t first = a.first[b];
  const int32_t given = a.count[b];
  if (first < 0 || given == 0) return;
  const uint32_t count = given > 0 ? static_cast<uint32_t>(given) : 0u;
  const int32_t *path = a.path + static_cast<int64_t>(b) * a.path_pitch;
  bool bad = given < 0 || count > a.tokens;
  for (uint32_t i = tid; i < min(count, a.tokens); i += kKeepThreads) {
    const int32_t v = path[i];
    s_path[i] = v;
    bad |= v < 0 || static_cast<uint32_t>(v) >= a.tokens;
  }
  __syncthreads();
  for (uint32_t i = tid + 1; i < min(count, a.tokens); i += kKeepThreads) bad |= s_path[i] <= s_path[i - 1];
  // (a path that is none moves nothing)
  if (__syncthreads_or(bad)) {
    if (tid == 0) atomicMax(a.err_flag, 1u);
    return;
  }
  const uint32_t page_rows = a.page_tokens, words = a.dim / 4;
  int64_t *s_from = reinterpret_cast<int64_t *>(s_path + (a.tokens + 1) / 2 * 2);
  float *s_scale = reinterpret_cast<float *>(s_from + page_rows);
  __shared__ float s_most[kKeepThreads / 32];
  const int32_t *table = a.page_table + static_cast<size_t>(b) * a.table_pitch;
  int8_t *cache = a.cache[kv] + static_cast<int64_t>(head) * a.cache_strides[1];
  const int64_t line = a.cache_strides[2], end = first + count;
  const auto page_of = [&](int64_t slot) {
    const int32_t page = slot < a.table_pitch ? table[slot] : -1;
    if (page >= 0 && static_cast<uint32_t>(page) < a.pages) return page;
    atomicMax(a.err_flag, 1u);
    return -1;
  };
  for (int64_t slot = first / page_rows; slot * page_rows < end; ++slot) {
    const int64_t row0 = slot * page_rows, lo = first > row0 ? first : row0, hi = end < row0 + page_rows ? end : row0 + page_rows;
    const int32_t page = page_of(slot);
    if (page < 0) continue;  // (the same for the block)
    int8_t *dst = cache + page * a.cache_strides[0];
    float *scale = a.scale[kv] + static_cast<size_t>(page) * a.heads + head;
    const uint32_t old_rows = static_cast<uint32_t>(lo - row0), rows = static_cast<uint32_t>(hi - lo);
    const float was = *scale;
    // the largest scale, a NaN where there is one
    float most = old_rows ? was : -__int_as_float(0x7f800000);
    const auto take = [&](float v) { most = v != v || most != most ? __int_as_float(0x7fc00000) : fmaxf(most, v); };
    for (uint32_t i = tid; i < rows; i += kKeepThreads) {
      const int64_t from = first + s_path[lo - first + i];
      const int32_t of = from / page_rows == slot ? page : page_of(from / page_rows);
      s_from[i] = of < 0 ? -1 : of * a.cache_strides[0] + from % page_rows * line;
      s_scale[i] = of < 0 ? 0.0f : of == page ? was : a.scale[kv][static_cast<size_t>(of) * a.heads + head];
      if (of >= 0) take(s_scale[i]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) take(__shfl_xor_sync(0xffffffffu, most, o));
    if (tid % 32 == 0) s_most[tid / 32] = most;
    __syncthreads();
#pragma unroll
    for (uint32_t w = 0; w < kKeepThreads / 32; ++w) take(s_most[w]);
    const float now = most, div = now > 0.0f ? now : 1.0f;
    const bool number = now == now;  // (a NaN: bytes as they are)
    if (old_rows && now != was && number) {
      const float ratio = was / div;
      for (uint32_t i = tid; i < old_rows * words; i += kKeepThreads) {
        char4 *p = reinterpret_cast<char4 *>(dst + i / words * line + i % words * 4);
        *p = rescaled(*p, ratio);
      }
    }
    // a few words a thread at a time, all read before any is written
    for (uint32_t i0 = 0; i0 < rows * words; i0 += kKeepThreads * kKept) {
      char4 kept[kKept];
      bool real[kKept];
#pragma unroll
      for (uint32_t k = 0; k < kKept; ++k) {
        const uint32_t i = i0 + k * kKeepThreads + tid;
        real[k] = i < rows * words && s_from[min(i / words, rows - 1)] >= 0;
        if (!real[k]) continue;
        kept[k] = *reinterpret_cast<const char4 *>(cache + s_from[i / words] + i % words * 4);
        const float s = s_scale[i / words];
        if (number && s != now) kept[k] = rescaled(kept[k], s / div);
      }
      __syncthreads();
#pragma unroll
      for (uint32_t k = 0; k < kKept; ++k) {
        const uint32_t i = i0 + k * kKeepThreads + tid;
        if (real[k]) *reinterpret_cast<char4 *>(dst + (old_rows + i / words) * line + i % words * 4) = kept[k];
      }
      __syncthreads();
    }
    if (tid == 0 && most != -__int_as_float(0x7f800000)) *scale = now;
    __syncthreads();  // (the rows' list is free again)
  }
}

template <typename T>
__global__ void __launch_bounds__(256) read_kernel(const ClearReadArgs a) {
  const uint32_t b = blockIdx.z, head = blockIdx.y >> 1, kv = blockIdx.y & 1u, words = a.dim / 4;
  const uint32_t id = blockIdx.x * blockDim.x + threadIdx.x, i = id / words, d = id % words * 4;
  if (i >= a.tokens) return;
  int64_t len = a.lengths[b];
  const int64_t most = static_cast<int64_t>(a.table_pitch) * a.page_tokens;
  if (len > most) {
    atomicMax(a.err_flag, 1u);
    len = most;
  }
  const int64_t at = static_cast<int64_t>(a.first[b]) + i;
  if (at < 0 || at >= len) return;
  const int32_t page = a.page_table[static_cast<size_t>(b) * a.table_pitch + at / a.page_tokens];
  if (page < 0 || static_cast<uint32_t>(page) >= a.pages) {
    atomicMax(a.err_flag, 1u);
    return;
  }
  const char4 q = *reinterpret_cast<const char4 *>(a.cache[kv] + page * a.cache_strides[0] + static_cast<int64_t>(head) * a.cache_strides[1] +
                                                   at % a.page_tokens * a.cache_strides[2] + d);
  const float s = a.scale[kv][static_cast<size_t>(page) * a.heads + head];
  T *out = static_cast<T *>(a.out[kv]) + static_cast<int64_t>(b) * a.out_strides[kv][0] + static_cast<int64_t>(i) * a.out_strides[kv][1] +
           static_cast<int64_t>(head) * a.out_strides[kv][2] + d;
  out[0] = from_float<T>(q.x * s);
  out[1] = from_float<T>(q.y * s);
  out[2] = from_float<T>(q.z * s);
  out[3] = from_float<T>(q.w * s);
}

template <typename T>
cudaError_t launch_read(const ClearReadArgs &a, cudaStream_t s) {
  const uint64_t threads = static_cast<uint64_t>(a.tokens) * (a.dim / 4);
  read_kernel<T><<<dim3(static_cast<uint32_t>((threads + 255) / 256), 2 * a.heads, a.batch), 256, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_clear_keep(const ClearKeepArgs &a, cudaStream_t s) {
  const size_t smem = (a.tokens + 1) / 2 * 8 + a.page_tokens * 12ull;
  keep_kernel<<<dim3(2 * a.heads, a.batch), kKeepThreads, smem, s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_clear_read(const ClearReadArgs &a, int type, cudaStream_t s) {
  if (type == kOutF32) return launch_read<float>(a, s);
  if (type == kOutF16) return launch_read<__half>(a, s);
  return launch_read<__nv_bfloat16>(a, s);
}

}  // namespace rosetta
