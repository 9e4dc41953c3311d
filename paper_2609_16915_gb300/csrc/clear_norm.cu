// Residual addition, root-mean-square norm and 8-bit output with a scale per token.
//
//   h = x + r,  y = h g / sqrt(mean h^2 + eps),  s = max|y| / 127,  q = rint(y / s)
//
// The factor 1/sqrt(..) is the same for a whole row, so with M = max |h g|
//   s = M / sqrt(mean h^2 + eps) / 127  and  q = rint(h g 127 / M):
// one reduction (a sum and a maximum together) serves the norm and the scale.
// Bound by reading x and r and writing h and q once: a row stays in registers between the two.  16384 x 4096 bfloat16 with
// residual 72 us, 6.5 TB/s; rows that are not aligned to 16 bytes are read element by element, 16384 x 4095 163 us.
#include <stdint.h>

#include <type_traits>

#include "clear.h"
#include "pairs.cuh"

namespace rosetta {

namespace {

// The larger, a NaN where there is one: a value that is no number reaches the row's scale.
__device__ __forceinline__ float max_nan(float x, float y) {
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(x), "f"(y));
  return m;
}

// Sum of `s` and maximum of `m` over the block, in every thread.
__device__ __forceinline__ void block_sum_max(float &s, float &m, float2 *parts) {
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, warps = blockDim.x / 32;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    s += __shfl_xor_sync(0xffffffffu, s, o);
    m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  }
  if (lane == 0) parts[warp] = make_float2(s, m);
  __syncthreads();
  float2 v = lane < warps ? parts[lane] : make_float2(0.0f, 0.0f);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    v.x += __shfl_xor_sync(0xffffffffu, v.x, o);
    v.y = max_nan(v.y, __shfl_xor_sync(0xffffffffu, v.y, o));
  }
  s = v.x;
  m = v.y;
}

// Squares leave single precision from 2^64 on, and below 2^-63, which counts where no eps hides it.  So a second sum takes the
// values times 2^-80, and where eps is tiny a third one times 2^100; a row whose plain sum is near an end of the range uses them.
// (Values of float16 do not come that far.)
constexpr float kDown = 0x1p-80f, kUp = 0x1p100f, kTinyEps = 0x1p-76f;

__device__ __forceinline__ float factor_of(float sumsq, bool tiny_eps) {  // (a NaN: kDown)
  return sumsq < 0x1p120f ? (tiny_eps && sumsq < 0x1p-100f ? kUp : 1.0f) : kDown;
}

// The sum of the squares of h times `factor`.
template <int VEC>
__device__ __forceinline__ float squares(const float (&h)[VEC], float factor) {
  if constexpr (VEC == 1) {
    return (h[0] * factor) * (h[0] * factor);
  } else {
    const uint64_t f2 = pair_of(factor, factor);
    uint64_t both = 0;
#pragma unroll
    for (int e = 0; e < VEC; e += 2) {
      const uint64_t v = mul2(pair_of(h[e], h[e + 1]), f2);
      both = e == 0 ? mul2(v, v) : fma2(v, v, both);
    }
    const float2 two = floats_of(both);
    return two.x + two.y;
  }
}

// What the row's sum of squares (of h times `factor`) and maximum of |h g| give: the stored scale, and
// q = rint((h g) up inv).  `up` lifts maxima so small that 127 / M would overflow.
struct RowScale {
  float scale, up, inv;
};

__device__ __forceinline__ RowScale row_scale(float sumsq, float top, uint32_t width, float eps, float factor) {
  RowScale r;
  const float rms = rsqrtf(sumsq / static_cast<float>(width) + eps * factor * factor);
  // an infinity leaves no trace in the rest of the row: 1 / sqrt of it is 0, and a gamma of 0 hides it from `top`
  const float infinite = __int_as_float(0x7f800000);
  r.scale = sumsq < infinite && top < infinite ? top * factor * rms / 127.0f : __int_as_float(0x7fc00000);
  r.up = top < 1e-30f ? 1.2676506e30f : 1.0f;  // 2^100
  r.inv = r.scale == 0.0f ? 0.0f : 127.0f / (top * r.up);
  return r;
}

__device__ __forceinline__ int8_t quantised(float hg, const RowScale &r) {
  return static_cast<int8_t>(__float2int_rn((hg * r.up) * r.inv));  // (a NaN converts to 0)
}

// VEC consecutive elements of a row, as one access
template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack {
  T v[VEC];
};

// The row in registers, NV packs a thread, read once.  LANES of a warp (8 or 32) per token, 256 / LANES tokens a block;
// 0: a block per token.  TINY: eps may be as small as the squares.
template <typename T, int VEC, int NV, int LANES, bool TINY>
__global__ void __launch_bounds__(LANES ? 256 : 1024) norm_kernel(const ClearNormArgs a) {
  __shared__ float2 parts[32];
  constexpr uint32_t GROUP = LANES ? LANES : 32;
  const uint32_t tid = LANES ? threadIdx.x % GROUP : threadIdx.x, threads = LANES ? GROUP : blockDim.x;
  const size_t t = LANES ? static_cast<size_t>(blockIdx.x) * (256 / GROUP) + threadIdx.x / GROUP : blockIdx.x;
  if (LANES && t >= a.tokens) return;
  const uint32_t mask = LANES == 8 ? 0xffu << (threadIdx.x % 32 / 8 * 8) : 0xffffffffu;  // the token's lanes
  const T *x = static_cast<const T *>(a.x) + t * a.x_pitch;
  const T *res = a.residual ? static_cast<const T *>(a.residual) + t * a.residual_pitch : nullptr;
  T *sum = a.sum_out ? static_cast<T *>(a.sum_out) + t * a.sum_pitch : nullptr;
  using P = Pack<T, VEC>;
  constexpr bool WIDE = !std::is_same<T, __half>::value, EARLY = VEC > 1;
  float down = 0.0f, lifted = 0.0f;
  // (as soon as h is there for wide accesses, beside the other sum for single elements: 4096 x 16384 bfloat16 74 us against 85,
  // 16384 x 4095 162 against 193)
  const auto scaled_squares = [&](const float (&v)[VEC]) {
    if constexpr (WIDE) down += squares<VEC>(v, kDown);
    if constexpr (TINY) lifted += squares<VEC>(v, kUp);
  };
  float h[NV][VEC];  // h, then h g
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const uint32_t i = (tid + j * threads) * VEC;
    P px{}, pr{};
    if (i < a.width) {
      px = *reinterpret_cast<const P *>(x + i);
      if (res) pr = *reinterpret_cast<const P *>(res + i);
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) h[j][e] = res ? to_float(px.v[e]) + to_float(pr.v[e]) : to_float(px.v[e]);
    if constexpr (EARLY) scaled_squares(h[j]);
  }
  float s = 0.0f, m = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const uint32_t i = (tid + j * threads) * VEC;
    if (i < a.width) {
      const Pack<float, VEC> g = *reinterpret_cast<const Pack<float, VEC> *>(a.gamma + i);
      P out;
      if constexpr (!EARLY) scaled_squares(h[j]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        out.v[e] = from_float<T>(h[j][e]);
        s += h[j][e] * h[j][e];
        h[j][e] *= g.v[e];
        m = max_nan(m, fabsf(h[j][e]));
      }
      if (sum) *reinterpret_cast<P *>(sum + i) = out;
    }
  }
  const auto reduce = [&]() {
    if constexpr (LANES > 0) {
#pragma unroll
      for (int o = LANES / 2; o > 0; o >>= 1) {
        s += __shfl_xor_sync(mask, s, o);
        m = max_nan(m, __shfl_xor_sync(mask, m, o));
      }
    } else {
      block_sum_max(s, m, parts);
    }
  };
  // (a second round rather than code of its own: that made every block 20 % longer)
  float factor = 1.0f;
#pragma unroll 1
  for (int round = 0; round < 2; ++round) {
    reduce();
    if (!WIDE || round) break;
    factor = factor_of(s, TINY);
    if (factor == 1.0f) break;  // (the same for the row)
    if constexpr (LANES == 0) __syncthreads();
    s = TINY && factor == kUp ? lifted : down;
  }
  const RowScale r = row_scale(s, m, a.width, a.eps, factor);
  int8_t *q = a.q + t * a.q_pitch;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const uint32_t i = (tid + j * threads) * VEC;
    if (i < a.width) {
      Pack<int8_t, VEC> out;
#pragma unroll
      for (int e = 0; e < VEC; ++e) out.v[e] = quantised(h[j][e], r);
      *reinterpret_cast<Pack<int8_t, VEC> *>(q + i) = out;
    }
  }
  if (tid == 0) a.scale[t] = r.scale;
}

// Rows too long for a block's registers are read twice (the second time from the L2 cache).
template <typename T>
__global__ void __launch_bounds__(1024) norm_long_kernel(const ClearNormArgs a) {
  __shared__ float2 parts[32];
  const size_t t = blockIdx.x;
  const T *x = static_cast<const T *>(a.x) + t * a.x_pitch;
  const T *res = a.residual ? static_cast<const T *>(a.residual) + t * a.residual_pitch : nullptr;
  T *sum = a.sum_out ? static_cast<T *>(a.sum_out) + t * a.sum_pitch : nullptr;
  float s = 0.0f, m = 0.0f;
  for (uint32_t i = threadIdx.x; i < a.width; i += blockDim.x) {
    const float h = to_float(x[i]) + (res ? to_float(res[i]) : 0.0f);
    s += h * h;
    m = max_nan(m, fabsf(h * a.gamma[i]));
  }
  block_sum_max(s, m, parts);
  const float factor = factor_of(s, a.eps < kTinyEps);
  if (factor != 1.0f) {  // (the same for the row; nothing is written yet)
    __syncthreads();
    s = 0.0f;
    for (uint32_t i = threadIdx.x; i < a.width; i += blockDim.x) {
      const float h = (to_float(x[i]) + (res ? to_float(res[i]) : 0.0f)) * factor;
      s += h * h;
    }
    block_sum_max(s, m, parts);
  }
  const RowScale r = row_scale(s, m, a.width, a.eps, factor);
  int8_t *q = a.q + t * a.q_pitch;
  for (uint32_t i = threadIdx.x; i < a.width; i += blockDim.x) {
    const float h = to_float(x[i]) + (res ? to_float(res[i]) : 0.0f);
    q[i] = quantised(h * a.gamma[i], r);
    if (sum) sum[i] = from_float<T>(h);
  }
  if (threadIdx.x == 0) a.scale[t] = r.scale;
}

template <typename T, int VEC, int NV, bool TINY>
cudaError_t launch_block(const ClearNormArgs &a, cudaStream_t s) {
  const uint32_t threads = ((a.width + VEC * NV - 1) / (VEC * NV) + 31) / 32 * 32;
  norm_kernel<T, VEC, NV, 0, TINY><<<a.tokens, threads, 0, s>>>(a);
  return cudaGetLastError();
}

// A quarter of a warp, then a warp per token while four packs a lane hold the row (scalars: eight), then blocks of up to 512 threads with two, up to
// 1024 with 32 elements each (scalars: 16).
template <typename T, int VEC, bool TINY>
cudaError_t launch_vec(const ClearNormArgs &a, cudaStream_t s) {
  constexpr int SMALL = VEC == 1 ? 8 : 4, MID = VEC == 1 ? 8 : 2, LARGE = VEC == 1 ? 16 : 32 / VEC;
  if (a.width <= 8u * VEC * SMALL) {
    norm_kernel<T, VEC, SMALL, 8, TINY><<<(a.tokens + 31) / 32, 256, 0, s>>>(a);
    return cudaGetLastError();
  }
  if (a.width <= 32u * VEC * SMALL) {
    norm_kernel<T, VEC, SMALL, 32, TINY><<<(a.tokens + 7) / 8, 256, 0, s>>>(a);
    return cudaGetLastError();
  }
  if (a.width <= 512u * VEC * MID) return launch_block<T, VEC, MID, TINY>(a, s);
  if (a.width <= 1024u * VEC * LARGE) return launch_block<T, VEC, LARGE, TINY>(a, s);
  norm_long_kernel<T><<<a.tokens, 1024, 0, s>>>(a);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_type(const ClearNormArgs &a, cudaStream_t s) {
  constexpr int VEC = 16 / sizeof(T);
  const auto at = [](const void *p) { return reinterpret_cast<uintptr_t>(p); };
  // (a pitch is used from the second row on only)
  const int64_t pitches = a.tokens > 1 ? (a.x_pitch | a.q_pitch | (a.residual ? a.residual_pitch : 0) | (a.sum_out ? a.sum_pitch : 0)) : 0;
  const bool wide = ((at(a.x) | at(a.residual) | at(a.sum_out)) & 15u) == 0 && (at(a.gamma) & (4 * VEC - 1)) == 0 &&
                    (at(a.q) & (VEC - 1)) == 0 && pitches % VEC == 0 && a.width % VEC == 0;
  if constexpr (!std::is_same<T, __half>::value) {
    if (a.eps < kTinyEps) return wide ? launch_vec<T, VEC, true>(a, s) : launch_vec<T, 1, true>(a, s);
  }
  return wide ? launch_vec<T, VEC, false>(a, s) : launch_vec<T, 1, false>(a, s);
}

}  // namespace

cudaError_t launch_clear_norm(const ClearNormArgs &a, int type, cudaStream_t s) {
  if (type == kOutF32) return launch_type<float>(a, s);
  if (type == kOutF16) return launch_type<__half>(a, s);
  return launch_type<__nv_bfloat16>(a, s);
}

}  // namespace rosetta
