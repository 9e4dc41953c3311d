// Product of 8-bit integers with scales for each token and channel:
//   acc[t][n] = sum_k q[t][k] w[n][k],   y = (acc scale[t]) w_scale[n] + bias[n].
// The packing of the weights, and the kernel for few tokens.
//
// Few tokens: bound by reading the weights once, and over 16 tokens by the latency of conversions and products of the few
// warps that the sums leave registers for.  A block takes 32 channels; its warps share out the steps of 64 inputs and join their
// integer sums in shared memory.  A warp copies its own weights and tokens ahead (cp.async, in the order of the lanes) and converts
// them from 8 bits to f16; a 16 x 8 x 16 product of f16 is exact (products below 2^14), and so are the f32 sums of 16 steps,
// which are then taken into integers.  More tokens are further groups of blocks, which read the weights from the L2.  4096
// inputs, 14336 channels (8.7 us at the copy rate): 1 token 11.3 us, 8 tokens 11.6, 16 12.7, 24 15.3, 32 17.5; 768 inputs, 3072
// channels: 1 token 2.1, 24 to 40 tokens 3.2, 64 4.3, 128 6.7.
#include <stdint.h>

#include "clear.h"
#include "dsmem.cuh"

namespace rosetta {

namespace {

// Pack: one 16-byte row of one chunk per thread.
__global__ void __launch_bounds__(256) pack_kernel(const int8_t *__restrict__ w, int64_t pitch, uint32_t channels,
                                                   uint32_t inner, uint32_t k_steps, int8_t *__restrict__ packed,
                                                   uint64_t rows16) {
  const uint64_t id = static_cast<uint64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (id >= rows16) return;
  const uint32_t row = id / 4 % kPackRows, chunk = (id % 4) ^ (row >> 1 & 3u);
  const uint64_t tile = id / (kPackRows * 4);
  const uint64_t n = tile / k_steps * kPackRows + row;
  const uint32_t k0 = tile % k_steps * kPackK + chunk * 16;
  uint32_t v[4] = {0u, 0u, 0u, 0u};
  if (n < channels) {
    const int8_t *src = w + static_cast<int64_t>(n) * pitch;
#pragma unroll
    for (uint32_t e = 0; e < 16; ++e)
      if (k0 + e < inner) v[e >> 2] |= static_cast<uint32_t>(static_cast<uint8_t>(src[k0 + e])) << (8 * (e & 3u));
  }
  reinterpret_cast<uint4 *>(packed)[id] = make_uint4(v[0], v[1], v[2], v[3]);
}

// four 8-bit integers to four f16: 1024 + (v + 128) by byte permute, minus 1152
__device__ __forceinline__ void int8x4_f16(uint32_t v, uint32_t &lo, uint32_t &hi) {
  const uint32_t u = v ^ 0x80808080u;
  const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
  uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
  const __half2 x = __hsub2(*reinterpret_cast<__half2 *>(&a), off), y = __hsub2(*reinterpret_cast<__half2 *>(&b), off);
  lo = *reinterpret_cast<const uint32_t *>(&x);
  hi = *reinterpret_cast<const uint32_t *>(&y);
}

__device__ __forceinline__ void mma_16x8x16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// 16 bytes of a token from input k on, which `row` points to; zeros from `inner` on
__device__ __forceinline__ uint4 token_bytes(const int8_t *row, uint32_t k, uint32_t inner) {
  uint32_t v[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (uint32_t e = 0; e < 16; ++e)
    if (k + e < inner) v[e >> 2] |= static_cast<uint32_t>(static_cast<uint8_t>(row[e])) << (8 * (e & 3u));
  return make_uint4(v[0], v[1], v[2], v[3]);
}

__device__ __forceinline__ void copy_async(uint32_t dst, const void *src, bool valid) {
  const uint32_t size = valid ? 16 : 0;  // (nothing is read for 0: zeros)
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(size) : "memory");
}

// Tiles of 32 channels over NB groups of eight tokens, the steps of 64 inputs shared out over WARPS warps; each
// warp copies its own steps, weights and tokens, DEPTH - 1 of them ahead.  Lane (g, t) = (lane / 4, lane % 4) of a warp takes,
// of one step, 16 bytes of channels g, g + 8, g + 16, g + 24 and of token g of each group: chunk t of the step.  Word i of
// those is its share of the i-th 16 x 8 x 16 product: the products take the inputs in another order than they are stored in,
// the same for both operands.
template <int NB, int WARPS, int DEPTH>
struct FewShape {
  static constexpr uint32_t PITCH = NB * 8 + 4;  // of a row of sums
  static constexpr uint32_t STEP = (4 + NB) * 512, RING = WARPS * DEPTH * STEP, SUMS = WARPS * 32 * PITCH * 4;
  static constexpr uint32_t SMEM = RING > SUMS ? RING : SUMS;
  static constexpr uint32_t BLOCKS = WARPS >= 12 ? 1 : NB == 4 ? 3 : 4;  // an SM
  static_assert(BLOCKS * (SMEM + 1024) <= 228 * 1024, "shared memory");
};

template <int NB, int WARPS, int DEPTH, bool ALIGNED>
__global__ void __launch_bounds__(32 * WARPS, FewShape<NB, WARPS, DEPTH>::BLOCKS) linear_few_kernel(const ClearLinearArgs a, int out_kind) {
  using S = FewShape<NB, WARPS, DEPTH>;
  extern __shared__ __align__(16) unsigned char smem[];
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
  const uint32_t n0 = blockIdx.x * 32, t0 = blockIdx.y * (NB * 8), tokens = min(a.tokens - t0, NB * 8u);
  // the next step to copy: its weights and, of this lane, each group's token
  const int8_t *w = a.packed + (static_cast<size_t>(n0 / kPackRows) * a.k_steps + warp) * kPackTile + n0 % kPackRows * kPackK + lane * 16;
  const int8_t *x[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) x[b] = a.q + (b * 8 + g < tokens ? static_cast<int64_t>(t0 + b * 8 + g) * a.q_pitch + warp * kPackK + t * 16 : 0);
  uint32_t next = warp;
  unsigned char *ring = smem + warp * (DEPTH * S::STEP) + lane * 16;
  const uint32_t ring_at = smem_addr(ring);
  const auto fetch = [&](uint32_t slot) {
    if (next < a.k_steps) {
#pragma unroll
      for (int r = 0; r < 4; ++r) copy_async(ring_at + slot * S::STEP + r * 512, w + r * (8 * kPackK), true);
      const bool whole = ALIGNED && (next + 1) * kPackK <= a.inner;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const bool in = b * 8 + g < tokens;
        if (whole)
          copy_async(ring_at + slot * S::STEP + (4 + b) * 512, x[b], in);
        else
          *reinterpret_cast<uint4 *>(ring + slot * S::STEP + (4 + b) * 512) =
              in ? token_bytes(x[b], next * kPackK + t * 16, a.inner) : make_uint4(0u, 0u, 0u, 0u);
        if (in) x[b] += WARPS * kPackK;
      }
      w += WARPS * kPackTile;
      next += WARPS;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  float d[2][NB][4] = {};
  int32_t acc[2][NB][4] = {};
  const auto take = [&]() {
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[m][b][i] += __float2int_rn(d[m][b][i]);
          d[m][b][i] = 0.0f;
        }
  };
#pragma unroll
  for (uint32_t i = 0; i + 1 < DEPTH; ++i) fetch(i);
  // of the channel that this lane writes, and of token `lane`
  const uint32_t n = n0 + lane;
  const float w_scale = n < a.channels ? a.w_scale[n] : 0.0f, bias = a.bias != nullptr && n < a.channels ? a.bias[n] : 0.0f;
  const float scale = lane < tokens ? a.scale[t0 + lane] : 0.0f;
  const uint32_t own = (g * 4 + (t ^ (g >> 1 & 3u))) * 16 - lane * 16;  // this lane's chunk of eight rows of weights
  uint32_t done = 0;  // steps since the sums were taken: 16 of 64 inputs are exact
  for (uint32_t k = warp, slot = 0; k < a.k_steps; k += WARPS) {
    asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 2) : "memory");
    __syncwarp();
    uint4 wv[4], xv[NB];
#pragma unroll
    for (int r = 0; r < 4; ++r) wv[r] = *reinterpret_cast<const uint4 *>(ring + slot * S::STEP + r * 512 + static_cast<int32_t>(own));
#pragma unroll
    for (int b = 0; b < NB; ++b) xv[b] = *reinterpret_cast<const uint4 *>(ring + slot * S::STEP + (4 + b) * 512);
    // into the place read in the step before this one
    fetch(slot == 0 ? DEPTH - 1 : slot - 1);
    if (++slot == DEPTH) slot = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto word = [&](const uint4 &v) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; };
      uint32_t f[2][4];
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        int8x4_f16(word(wv[2 * m]), f[m][0], f[m][2]);
        int8x4_f16(word(wv[2 * m + 1]), f[m][1], f[m][3]);
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        uint32_t b0, b1;
        int8x4_f16(word(xv[b]), b0, b1);
        mma_16x8x16(d[0][b], f[0], b0, b1);
        mma_16x8x16(d[1][b], f[1], b0, b1);
      }
    }
    if (++done == 1024 / kPackK) {
      done = 0;
      take();
    }
  }
  take();
  // the warps' sums, joined: exact in any order
  int32_t *parts = reinterpret_cast<int32_t *>(smem);  // [warp][channel][token]
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();
#pragma unroll
  for (int m = 0; m < 2; ++m)
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 4; i += 2)
        *reinterpret_cast<int2 *>(parts + (warp * 32 + m * 16 + i * 4 + g) * S::PITCH + b * 8 + 2 * t) =
            make_int2(acc[m][b][i], acc[m][b][i + 1]);
  __syncthreads();
  for (uint32_t tok = warp; tok < tokens; tok += WARPS) {
    const float token_scale = __shfl_sync(0xffffffffu, scale, tok);
    int32_t sum = 0;
#pragma unroll
    for (uint32_t v = 0; v < WARPS; ++v) sum += parts[(v * 32 + lane) * S::PITCH + tok];
    if (n >= a.channels) continue;
    const float y = clear_scaled(sum, token_scale, w_scale, a.bias != nullptr, bias);
    if (out_kind == kOutF32)
      clear_store<kOutF32>(a, t0 + tok, n, y);
    else if (out_kind == kOutF16)
      clear_store<kOutF16>(a, t0 + tok, n, y);
    else if (out_kind == kOutBf16)
      clear_store<kOutBf16>(a, t0 + tok, n, y);
    else
      clear_store<kOutCodes>(a, t0 + tok, n, y);
  }
}

bool aligned_of(const ClearLinearArgs &a) {
  return (reinterpret_cast<uintptr_t>(a.q) | static_cast<uintptr_t>(a.tokens > 1 ? a.q_pitch : 0)) % 16 == 0;
}

template <int NB, int WARPS, int DEPTH>
cudaError_t launch_few(const ClearLinearArgs &a, int out_kind, cudaStream_t s) {
  using S = FewShape<NB, WARPS, DEPTH>;
  auto kern = aligned_of(a) ? linear_few_kernel<NB, WARPS, DEPTH, true> : linear_few_kernel<NB, WARPS, DEPTH, false>;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(S::SMEM));
  if (e != cudaSuccess) return e;
  kern<<<dim3((a.channels + 31) / 32, (a.tokens + NB * 8 - 1) / (NB * 8)), 32 * WARPS, S::SMEM, s>>>(a, out_kind);
  return cudaGetLastError();
}

uint64_t blocks_of(const ClearLinearArgs &a, uint32_t nb) {
  return static_cast<uint64_t>((a.channels + 31) / 32) * ((a.tokens + nb * 8 - 1) / (nb * 8));
}

// An estimate of the time with groups of 8 nb tokens, from measurements.  Up to a block an SM: a start, and the steps of 16 warps
// (12 over 24 tokens: the sums leave no registers for more).  Else four warps a block and up to four blocks an SM, each
// with its steps.  Tokens that no 16-byte copy can take are read byte by byte.
uint64_t ns_of(const ClearLinearArgs &a, uint32_t nb, bool aligned, uint32_t sms) {
  static constexpr uint32_t kStart[4] = {1400, 2200, 3150, 3400}, kStep[4] = {710, 830, 1000, 850}, kBlock[4] = {300, 300, 600, 800},
                            kBlockStep[4] = {110, 155, 220, 290};
  const uint64_t blocks = blocks_of(a, nb), bytes = aligned ? 1 : 3;
  if (blocks <= sms) {
    const uint32_t warps = nb == 4 ? 12 : 16;
    return kStart[nb - 1] + (a.k_steps + warps - 1) / warps * kStep[nb - 1] * bytes;
  }
  const uint64_t steps = (a.k_steps + 3) / 4;
  return 1600 + 150 * steps + (kBlock[nb - 1] + kBlockStep[nb - 1] * steps) * bytes * blocks / sms;
}

uint32_t group_of(const ClearLinearArgs &a, uint32_t sms) {
  const bool aligned = aligned_of(a);
  uint32_t best = 1;
  for (uint32_t nb = 2; nb <= 4 && nb * 8 < a.tokens + 8; ++nb)
    if (ns_of(a, nb, aligned, sms) < ns_of(a, best, aligned, sms)) best = nb;
  return best;
}

template <int NB>
cudaError_t launch_few(const ClearLinearArgs &a, int out_kind, uint32_t sms, cudaStream_t s) {
  constexpr int DEPTH = NB > 2 ? 3 : 4;
  return blocks_of(a, NB) > sms ? launch_few<NB, 4, DEPTH>(a, out_kind, s) : launch_few<NB, NB == 4 ? 12 : 16, DEPTH>(a, out_kind, s);
}

}  // namespace

cudaError_t launch_clear_pack(const int8_t *weight, int64_t pitch, uint32_t channels, uint32_t inner, int8_t *packed,
                              cudaStream_t s) {
  const uint32_t k_steps = (inner + kPackK - 1) / kPackK;
  const uint64_t rows16 = static_cast<uint64_t>((channels + kPackRows - 1) / kPackRows) * k_steps * (kPackTile / 16);
  const uint64_t blocks = (rows16 + 255) / 256;  // < 2^31: checked with the sizes
  pack_kernel<<<static_cast<uint32_t>(blocks), 256, 0, s>>>(weight, pitch, channels, inner, k_steps, packed, rows16);
  return cudaGetLastError();
}

uint64_t linear_few_ns(const ClearLinearArgs &a, uint32_t sms) {
  if (a.tokens > 65535 * 8u) return ~0ull;  // (groups of a grid)
  return ns_of(a, group_of(a, sms), aligned_of(a), sms);
}

cudaError_t launch_clear_linear_few(const ClearLinearArgs &a, int out_kind, uint32_t sms, cudaStream_t s) {
  switch (group_of(a, sms)) {
    case 1: return launch_few<1>(a, out_kind, sms, s);
    case 2: return launch_few<2>(a, out_kind, sms, s);
    case 3: return launch_few<3>(a, out_kind, sms, s);
    default: return launch_few<4>(a, out_kind, sms, s);
  }
}

}  // namespace rosetta
