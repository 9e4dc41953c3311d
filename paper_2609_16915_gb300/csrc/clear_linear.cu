// Product of 8-bit integers with scales for each token and channel:
//   acc[t][n] = sum_k q[t][k] w[n][k],   y = (acc scale[t]) w_scale[n] + bias[n].
// The packing of the weights, and the kernel for few tokens.
//
// Few tokens: bound by reading the weights once.  A block takes 32 channels and up
// to 8 tokens; its eight warps share out the chunks of 16 inputs, a lane has one
// channel (the packed tiles make that 512 contiguous bytes a warp) and multiplies
// by dp4a, four products an instruction, with the tokens' bytes broadcast from
// shared memory.  Integer sums, so the warps' partial sums join exactly.
#include <stdint.h>

#include "clear.h"

namespace rosetta {

namespace {

// Pack: one 16-byte row of one chunk per thread.
__global__ void __launch_bounds__(256) pack_kernel(const int8_t *__restrict__ w, int64_t pitch, uint32_t channels,
                                                   uint32_t inner, uint32_t k_steps, int8_t *__restrict__ packed,
                                                   uint64_t rows16) {
  const uint64_t id = static_cast<uint64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (id >= rows16) return;
  const uint32_t row = id % kPackRows, chunk = id / kPackRows % 4;
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

constexpr uint32_t kFewWarps = 8, kFewSlab = 2048;  // bytes of a token's row in shared memory at a time

template <int TB, int OUT>
__global__ void __launch_bounds__(32 * kFewWarps) linear_few_kernel(const ClearLinearArgs a) {
  __shared__ __align__(16) int8_t xs[TB][kFewSlab];
  __shared__ int32_t part[kFewWarps][TB][32];
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t n = blockIdx.x * 32 + lane, t0 = blockIdx.y * TB;
  const int8_t *tiles = a.packed + static_cast<size_t>(blockIdx.x / 4) * a.k_steps * kPackTile + (blockIdx.x % 4 * 32 + lane) * 16;
  int32_t acc[TB] = {};
  for (uint32_t k0 = 0; k0 < a.inner; k0 += kFewSlab) {
    const uint32_t len = min(kFewSlab, a.inner - k0), padded = (len + 15) / 16 * 16;
    __syncthreads();
    for (uint32_t t = 0; t < TB; ++t) {
      const int8_t *src = a.q + static_cast<int64_t>(t0 + t) * a.q_pitch + k0;
      for (uint32_t i = threadIdx.x; i < padded; i += blockDim.x)
        xs[t][i] = t0 + t < a.tokens && i < len ? src[i] : static_cast<int8_t>(0);
    }
    __syncthreads();
    // chunk c of 16 inputs: bytes c * 128 * 16 of the tiles, which follow one another
    const int8_t *w = tiles + static_cast<size_t>(k0 / 16) * (kPackRows * 16);
#pragma unroll 4
    for (uint32_t c = warp; c < padded / 16; c += kFewWarps) {
      const int4 wv = __ldg(reinterpret_cast<const int4 *>(w + static_cast<size_t>(c) * (kPackRows * 16)));
#pragma unroll
      for (int t = 0; t < TB; ++t) {
        const int4 xv = *reinterpret_cast<const int4 *>(&xs[t][c * 16]);
        acc[t] = __dp4a(wv.w, xv.w, __dp4a(wv.z, xv.z, __dp4a(wv.y, xv.y, __dp4a(wv.x, xv.x, acc[t]))));
      }
    }
  }
#pragma unroll
  for (int t = 0; t < TB; ++t) part[warp][t][lane] = acc[t];
  __syncthreads();
  for (uint32_t t = warp; t < TB; t += kFewWarps) {
    if (t0 + t >= a.tokens || n >= a.channels) continue;
    int32_t sum = 0;
#pragma unroll
    for (uint32_t w = 0; w < kFewWarps; ++w) sum += part[w][t][lane];
    clear_store<OUT>(a, t0 + t, n, clear_scaled(sum, a.scale[t0 + t], a.w_scale[n], a.bias, n));
  }
}

template <int OUT>
cudaError_t launch_few(const ClearLinearArgs &a, cudaStream_t s) {
  const uint32_t blocks = (a.channels + 31) / 32;
  // the tokens of a block: as many as there are, in a power of two up to 8
  // (the grid's second dimension ends at 65535 blocks)
  for (uint64_t t0 = 0; t0 < a.tokens; t0 += 8ull * 65535) {
    ClearLinearArgs b = a;
    b.tokens = static_cast<uint32_t>(a.tokens - t0 < 8ull * 65535 ? a.tokens - t0 : 8ull * 65535);
    b.q += static_cast<int64_t>(t0) * a.q_pitch;
    b.scale += t0;
    const int64_t size = OUT == kOutF32 ? 4 : OUT == kOutCodes ? 1 : 2;
    b.out = static_cast<char *>(a.out) + static_cast<int64_t>(t0) * a.out_pitch * size;
    if (a.values) b.values += static_cast<int64_t>(t0) * a.values_pitch;
    const uint32_t tokens = b.tokens;
    if (tokens == 1)
      linear_few_kernel<1, OUT><<<dim3(blocks, 1), 32 * kFewWarps, 0, s>>>(b);
    else if (tokens == 2)
      linear_few_kernel<2, OUT><<<dim3(blocks, 1), 32 * kFewWarps, 0, s>>>(b);
    else if (tokens <= 4)
      linear_few_kernel<4, OUT><<<dim3(blocks, 1), 32 * kFewWarps, 0, s>>>(b);
    else
      linear_few_kernel<8, OUT><<<dim3(blocks, (tokens + 7) / 8), 32 * kFewWarps, 0, s>>>(b);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
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

cudaError_t launch_clear_linear(const ClearLinearArgs &a, int out_kind, cudaStream_t s) {
  switch (out_kind) {
    case kOutF32: return launch_few<kOutF32>(a, s);
    case kOutF16: return launch_few<kOutF16>(a, s);
    case kOutBf16: return launch_few<kOutBf16>(a, s);
    default: return launch_few<kOutCodes>(a, s);
  }
}

}  // namespace rosetta
