// Internal declarations of the decoder layer in the clear (rosetta_clear_*):
// argument structs and launchers of its kernels.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace rosetta {

struct ClearNormArgs {
  const void *x, *residual;  // residual null: none
  const float *gamma;
  void *sum_out;             // null: not wanted
  int8_t *q;
  float *scale;
  int64_t x_pitch, residual_pitch, sum_pitch, q_pitch;
  uint32_t tokens, width;
  float eps;
};

// Packed weights: [row tile][k step] tiles of 128 channels x 64 inputs, a row 64 bytes with its chunk c (of 16 inputs)
// at c ^ (row / 2 % 4): eight lanes read 128 bytes in a row of memory, and one chunk of eight rows every bank once.
constexpr uint32_t kPackRows = 128, kPackK = 64, kPackTile = kPackRows * kPackK;

enum ClearOut : int { kOutF32 = 0, kOutF16 = 1, kOutBf16 = 2, kOutCodes = 3 };  // 0 .. 2: rosetta_float_type

struct ClearLinearArgs {
  const int8_t *q;
  const float *scale;
  const int8_t *packed;
  const float *w_scale, *bias;  // bias null: none
  void *out;                    // floats, or the codes
  int64_t q_pitch, out_pitch;
  const int8_t *table;          // null: none
  int8_t *values;
  int64_t values_pitch;
  uint32_t tokens, channels, inner, k_steps;
  float lo, inv, top;           // code = clamp(floor((y - lo) * inv), 0, top)
  uint32_t *err_flag;
};

struct ClearAppendArgs {
  const void *src[2];           // k, v
  int64_t src_strides[2][3];    // batch, token, head
  int8_t *cache[2];
  int64_t cache_strides[3];     // page, head, row
  float *scale[2];
  const int32_t *page_table, *first;
  uint32_t batch, tokens, heads, dim, pages, page_tokens, table_pitch;
  uint32_t *err_flag;
};

struct ClearAttentionArgs {
  const void *q;
  void *out;
  int64_t q_strides[3], out_strides[3];
  const int8_t *k_cache, *v_cache;
  int64_t cache_strides[3];
  const float *k_scale, *v_scale;
  const int32_t *page_table, *lengths;
  uint32_t batch, tokens, heads, group, dim, pages, page_tokens, table_pitch;
  float softmax_scale;
  const uint32_t *mask;         // of a tree of drafted tokens; null: causal
  int64_t mask_strides[2];      // batch, token (words)
  uint32_t *err_flag;
};

struct ClearTreeArgs {
  const int32_t *parents;
  int64_t parents_pitch;
  uint32_t *mask;
  int64_t mask_strides[2];
  uint32_t batch, tokens;
  uint32_t *err_flag;
};

struct ClearVerifyArgs {
  const void *target, *draft;   // draft null: the drafted tokens were given, not drawn
  int64_t target_strides[2], draft_strides[2];  // batch, node
  const int32_t *tokens, *parents;
  const float *uniform;
  int64_t tokens_pitch, parents_pitch, uniform_pitch, path_pitch;
  int32_t *path, *count, *next;
  uint32_t batch, nodes, vocab;
  uint32_t *err_flag;
};

struct ClearKeepArgs {
  int8_t *cache[2];
  int64_t cache_strides[3];
  float *scale[2];
  const int32_t *page_table, *first, *path, *count;
  int64_t path_pitch;
  uint32_t batch, tokens, heads, dim, pages, page_tokens, table_pitch;
  uint32_t *err_flag;
};

struct ClearReadArgs {
  const int8_t *cache[2];
  int64_t cache_strides[3];
  const float *scale[2];
  const int32_t *page_table, *first, *lengths;
  void *out[2];
  int64_t out_strides[2][3];    // batch, token, head
  uint32_t batch, tokens, heads, dim, pages, page_tokens, table_pitch;
  uint32_t *err_flag;
};

// float types by rosetta_float_type
template <typename T>
__device__ __forceinline__ float to_float(T v);
template <>
__device__ __forceinline__ float to_float<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ float to_float<__half>(__half v) {
  return __half2float(v);
}
template <>
__device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) {
  return __bfloat162float(v);
}
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) {
  return v;
}
template <>
__device__ __forceinline__ __half from_float<__half>(float v) {
  return __float2half_rn(v);
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) {
  return __float2bfloat16_rn(v);
}

// A scaled sum of the linear product, each step rounded (no contraction): the
// codes are decided by exactly these single-precision values.
__device__ __forceinline__ float clear_scaled(int32_t acc, float scale, float w_scale, bool biased, float bias) {
  const float y = __fmul_rn(__fmul_rn(__int2float_rn(acc), scale), w_scale);
  return biased ? __fadd_rn(y, bias) : y;
}

__device__ __forceinline__ uint32_t clear_code(const ClearLinearArgs &a, float y) {
  // fmaxf drops a NaN: code 0
  return static_cast<uint32_t>(fminf(fmaxf(floorf(__fmul_rn(__fsub_rn(y, a.lo), a.inv)), 0.0f), a.top));
}

// Store one output of the linear product.
template <int OUT>
__device__ __forceinline__ void clear_store(const ClearLinearArgs &a, uint32_t t, uint32_t n, float y) {
  const int64_t at = static_cast<int64_t>(t) * a.out_pitch + n;
  if constexpr (OUT == kOutF32) {
    static_cast<float *>(a.out)[at] = y;
  } else if constexpr (OUT == kOutF16) {
    static_cast<__half *>(a.out)[at] = __float2half_rn(y);
  } else if constexpr (OUT == kOutBf16) {
    static_cast<__nv_bfloat16 *>(a.out)[at] = __float2bfloat16_rn(y);
  } else {
    const uint32_t code = clear_code(a, y);
    static_cast<uint8_t *>(a.out)[at] = static_cast<uint8_t>(code);
    if (a.values) a.values[static_cast<int64_t>(t) * a.values_pitch + n] = a.table[code];
  }
}

cudaError_t launch_clear_norm(const ClearNormArgs &a, int type, cudaStream_t s);
cudaError_t launch_clear_pack(const int8_t *weight, int64_t pitch, uint32_t channels, uint32_t inner, int8_t *packed,
                              cudaStream_t s);
// The linear product of few tokens, and the one on the tensor cores: estimates of their times, and the launches (work:
// linear_tc_bytes).  The first takes what few blocks finish, at every width up to 32 tokens and small matrices up to some hundred:
// 4096 inputs, 14336 channels, 32 tokens 17.8 us against 22.7, 40 tokens 26 against 22.7; 768 inputs, 3072 channels, 64 tokens
// 4.3 against 9.7, 256 as fast.
uint64_t linear_few_ns(const ClearLinearArgs &a, uint32_t sms);
uint64_t linear_tc_ns(const ClearLinearArgs &a, uint32_t sms);
cudaError_t launch_clear_linear_few(const ClearLinearArgs &a, int out_kind, uint32_t sms, cudaStream_t s);
size_t linear_tc_bytes(const ClearLinearArgs &a, uint32_t sms);
cudaError_t launch_clear_linear_tc(const ClearLinearArgs &a, int out_kind, void *work, uint32_t sms, cudaStream_t s);
cudaError_t launch_clear_append(const ClearAppendArgs &a, int type, cudaStream_t s);
// attention for few rows a cached head: whole 16-position tiles in a page, heads a multiple of 16; work:
// attend_few_bytes
bool attend_few_takes(const ClearAttentionArgs &a);
size_t attend_few_bytes(const ClearAttentionArgs &a, uint32_t sms);
cudaError_t launch_clear_attention_few(const ClearAttentionArgs &a, int type, void *work, uint32_t sms, cudaStream_t s);
// for many (prompts), on the tensor cores: the same, heads up to 128
bool attend_many_takes(const ClearAttentionArgs &a);
size_t attend_many_bytes(const ClearAttentionArgs &a, int type, uint32_t sms);
cudaError_t launch_clear_attention_many(const ClearAttentionArgs &a, int type, void *work, uint32_t sms, cudaStream_t s);
// and for every shape
cudaError_t launch_clear_attention(const ClearAttentionArgs &a, int type, cudaStream_t s);
// drafted tokens
cudaError_t launch_clear_tree_mask(const ClearTreeArgs &a, cudaStream_t s);
cudaError_t launch_clear_verify(const ClearVerifyArgs &a, int type, uint32_t sms, cudaStream_t s);
cudaError_t launch_clear_keep(const ClearKeepArgs &a, cudaStream_t s);
cudaError_t launch_clear_read(const ClearReadArgs &a, int type, cudaStream_t s);

}  // namespace rosetta
