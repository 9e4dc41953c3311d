// Residual addition, root-mean-square norm and 8-bit output with a scale per token.
//
//   h = x + r,  y = h g / sqrt(mean h^2 + eps),  s = max|y| / 127,  q = rint(y / s)
//
// The factor 1/sqrt(..) is the same for a whole row, so with M = max |h g|
//   s = M / sqrt(mean h^2 + eps) / 127  and  q = rint(h g 127 / M):
// one reduction (a sum and a maximum together) serves the norm and the scale.
// A block per token.
#include <stdint.h>

#include "clear.h"

namespace rosetta {

namespace {

// Sum of `s` and maximum of `m` over the block, in every thread.
__device__ __forceinline__ void block_sum_max(float &s, float &m, float2 *parts) {
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, o);
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  }
  if (lane == 0) parts[warp] = make_float2(s, m);
  __syncthreads();
  float2 v = lane < warps ? parts[lane] : make_float2(0.0f, 0.0f);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y = fmaxf(v.y, __shfl_xor_sync(0xffffffffu, v.y, o));
  }
  s = v.x;
  m = v.y;
}

// What the row's sum of squares and maximum of |h g| give: the stored scale, and
// q = rint((h g) up inv).  `up` lifts maxima so small that 127 / M would overflow.
struct RowScale {
  float scale, up, inv;
};

__device__ __forceinline__ RowScale row_scale(float sumsq, float top, uint32_t width, float eps) {
  RowScale r;
  const float rms = rsqrtf(sumsq / static_cast<float>(width) + eps);
  r.scale = top * rms / 127.0f;  // NaN where sumsq is NaN, or infinite by an infinity (0 * inf)
  r.up = top < 1e-30f ? 1.2676506e30f : 1.0f;  // 2^100
  r.inv = r.scale == 0.0f ? 0.0f : 127.0f / (top * r.up);
  return r;
}

__device__ __forceinline__ int8_t quantised(float hg, const RowScale &r) {
  return static_cast<int8_t>(__float2int_rn((hg * r.up) * r.inv));  // (a NaN converts to 0)
}

template <typename T>
__global__ void __launch_bounds__(256) norm_kernel(const ClearNormArgs a) {
  __shared__ float2 parts[32];
  const size_t t = blockIdx.x;
  const T *x = static_cast<const T *>(a.x) + t * a.x_pitch;
  const T *res = a.residual ? static_cast<const T *>(a.residual) + t * a.residual_pitch : nullptr;
  T *sum = a.sum_out ? static_cast<T *>(a.sum_out) + t * a.sum_pitch : nullptr;
  float s = 0.0f, m = 0.0f;
  for (uint32_t i = threadIdx.x; i < a.width; i += blockDim.x) {
    const float h = to_float(x[i]) + (res ? to_float(res[i]) : 0.0f);
    s += h * h;
    m = fmaxf(m, fabsf(h * a.gamma[i]));
  }
  block_sum_max(s, m, parts);
  const RowScale r = row_scale(s, m, a.width, a.eps);
  int8_t *q = a.q + t * a.q_pitch;
  for (uint32_t i = threadIdx.x; i < a.width; i += blockDim.x) {
    const float h = to_float(x[i]) + (res ? to_float(res[i]) : 0.0f);
    q[i] = quantised(h * a.gamma[i], r);
    if (sum) sum[i] = from_float<T>(h);
  }
  if (threadIdx.x == 0) a.scale[t] = r.scale;
}

}  // namespace

cudaError_t launch_clear_norm(const ClearNormArgs &a, int type, cudaStream_t s) {
  if (type == kOutF32)
    norm_kernel<float><<<a.tokens, 256, 0, s>>>(a);
  else if (type == kOutF16)
    norm_kernel<__half><<<a.tokens, 256, 0, s>>>(a);
  else
    norm_kernel<__nv_bfloat16><<<a.tokens, 256, 0, s>>>(a);
  return cudaGetLastError();
}

}  // namespace rosetta
