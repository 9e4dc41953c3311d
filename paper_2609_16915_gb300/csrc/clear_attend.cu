// Causal attention over the paged 8-bit cache.
//
//   out = sum_p softmax(c q . K_p) V_p,  K_p = kq ks[page][head],  V_p = vq vs[page][head]
// with the running maximum m and sum l of the softmax, one pass over the positions:
//   m' = max(m, s),  l' = l 2^(m - m') + 2^(s - m'),  o' = o 2^(m - m') + 2^(s - m') V
// (scores s in units of log 2).
//
// This kernel takes every head size: a warp per query row, 32 positions at a time, a
// lane computing one position's score, then each lane summing its share of the
// head's dimensions over the 32 positions.  Every row reads all its keys and values again, and multiplies outside the
// tensor cores: 64 sequences of 2048 positions, 32 heads over 8 of 128, pages of 8, 1.8 ms (62 us with pages of 16, which the
// kernel for few rows takes); 4 x 256 queries at 1024 positions 5.1 ms (29 us).
#include <stdint.h>

#include "clear.h"

namespace rosetta {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kRowWarps = 4;

template <typename T>
__global__ void __launch_bounds__(32 * kRowWarps) attend_row_kernel(const ClearAttentionArgs a, uint32_t row_blocks) {
  __shared__ float qs[kRowWarps][256];
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t hq = a.heads * a.group;
  const uint32_t b = blockIdx.x / row_blocks;
  const uint64_t row = static_cast<uint64_t>(blockIdx.x % row_blocks) * kRowWarps + warp;  // token, query head
  if (row >= static_cast<uint64_t>(a.tokens) * hq) return;  // (no block-wide barrier below)
  const uint32_t t = static_cast<uint32_t>(row / hq), head = static_cast<uint32_t>(row % hq), kh = head / a.group;
  int64_t len = a.lengths[b];
  const int64_t most = static_cast<int64_t>(a.table_pitch) * a.page_tokens;
  if (len > most) {
    if (lane == 0) atomicMax(a.err_flag, 1u);
    len = most;
  }
  const int64_t last = len - a.tokens + t;  // the last position this row sees
  const T *q = static_cast<const T *>(a.q) + static_cast<int64_t>(b) * a.q_strides[0] + static_cast<int64_t>(t) * a.q_strides[1] +
               static_cast<int64_t>(head) * a.q_strides[2];
  for (uint32_t d = lane; d < a.dim; d += 32) qs[warp][d] = to_float(q[d]) * (a.softmax_scale * kLog2e);
  __syncwarp();
  const int32_t *table = a.page_table + static_cast<size_t>(b) * a.table_pitch;
  float m = -__int_as_float(0x7f800000), l = 0.0f, o[8] = {};
  for (int64_t p0 = 0; p0 <= last; p0 += 32) {
    const int64_t p = p0 + lane;
    float s = -__int_as_float(0x7f800000), vs = 0.0f;
    int64_t at = -1;
    if (p <= last) {
      const int32_t page = table[p / a.page_tokens];
      if (page < 0 || static_cast<uint32_t>(page) >= a.pages) {
        atomicMax(a.err_flag, 1u);
      } else {
        at = page * a.cache_strides[0] + static_cast<int64_t>(kh) * a.cache_strides[1] + p % a.page_tokens * a.cache_strides[2];
        const float ks = a.k_scale[static_cast<size_t>(page) * a.heads + kh];
        vs = a.v_scale[static_cast<size_t>(page) * a.heads + kh];
        float dot = 0.0f;
        for (uint32_t d = 0; d < a.dim; d += 4) {
          const char4 k = *reinterpret_cast<const char4 *>(a.k_cache + at + d);
          dot += qs[warp][d] * k.x + qs[warp][d + 1] * k.y + qs[warp][d + 2] * k.z + qs[warp][d + 3] * k.w;
        }
        s = dot * ks;
      }
    }
    float top = s;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    const float m2 = fmaxf(m, top);
    const float base = m2 == -__int_as_float(0x7f800000) ? 0.0f : m2;  // nothing seen yet
    const float keep = exp2f(m - base), e = at >= 0 ? exp2f(s - base) : 0.0f;
    l = l * keep + e;  // (each lane its own positions; summed at the end)
    m = m2;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] *= keep;
    const float ev = at >= 0 ? e * vs : 0.0f;
    for (int j = 0; j < 32; ++j) {
      const int64_t from = __shfl_sync(0xffffffffu, at, j);
      const float w = __shfl_sync(0xffffffffu, ev, j);
      if (from < 0) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (lane + 32 * i < a.dim) o[i] += w * static_cast<float>(a.v_cache[from + lane + 32 * i]);
    }
  }
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
  T *out = static_cast<T *>(a.out) + static_cast<int64_t>(b) * a.out_strides[0] + static_cast<int64_t>(t) * a.out_strides[1] +
           static_cast<int64_t>(head) * a.out_strides[2];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (lane + 32 * i < a.dim) out[lane + 32 * i] = from_float<T>(l == 0.0f ? 0.0f : o[i] / l);
}

template <typename T>
cudaError_t launch_rows(const ClearAttentionArgs &a, cudaStream_t s) {
  const uint64_t rows = static_cast<uint64_t>(a.tokens) * a.heads * a.group;
  const uint32_t row_blocks = static_cast<uint32_t>((rows + kRowWarps - 1) / kRowWarps);
  attend_row_kernel<T><<<static_cast<uint32_t>(a.batch * static_cast<uint64_t>(row_blocks)), 32 * kRowWarps, 0, s>>>(a, row_blocks);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_clear_attention(const ClearAttentionArgs &a, int type, cudaStream_t s) {
  if (type == kOutF32) return launch_rows<float>(a, s);
  if (type == kOutF16) return launch_rows<__half>(a, s);
  return launch_rows<__nv_bfloat16>(a, s);
}

}  // namespace rosetta
