// C ABI of the decoder layer in the clear (rosetta_clear_*): argument checks,
// the handle with its workspace, dispatch.  Declarations and their documentation:
// include/rosetta.h.
#include <cuda_runtime.h>
#include <math.h>

#include <new>
#include <vector>

#include "rosetta.h"
#include "clear.h"

using namespace rosetta;

struct rosetta_clear {
  int device = 0;
  uint32_t sms = 1;
  uint32_t *d_err = nullptr;  // 1: a page or length out of range; 2: a bounded wait gave up
  void *work = nullptr;       // the present workspace
  size_t work_bytes = 0;
  std::vector<void *> outgrown;  // earlier ones: a captured graph may hold them
};

namespace {

int cuda_fail(cudaError_t e) {
  return e == cudaErrorMemoryAllocation ? ROSETTA_ERR_OOM : ROSETTA_ERR_CUDA;
}

cudaStream_t as_stream(void *s) { return reinterpret_cast<cudaStream_t>(s); }

bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

size_t type_size(int type) { return type == ROSETTA_FLOAT32 ? 4 : 2; }

bool known_type(int type) { return type == ROSETTA_FLOAT32 || type == ROSETTA_FLOAT16 || type == ROSETTA_BFLOAT16; }

// Bytes from a buffer's start to the end of its last row.
size_t span(int64_t pitch, uint64_t rows, uint64_t width, size_t size) {
  return rows ? (static_cast<size_t>(pitch) * (rows - 1) + width) * size : 0;
}

bool overlaps(const void *a, size_t na, const void *b, size_t nb) {
  const char *pa = static_cast<const char *>(a), *pb = static_cast<const char *>(b);
  return a && b && pa < pb + nb && pb < pa + na;
}

constexpr int64_t kMostPitch = int64_t{1} << 40;

bool good_pitch(int64_t pitch, uint64_t width) { return pitch >= static_cast<int64_t>(width) && pitch <= kMostPitch; }

bool good_strides(const int64_t *s) {
  for (int i = 0; i < 3; ++i)
    if (s[i] < 0 || s[i] > kMostPitch) return false;
  return true;
}

// Do N dimensions of rows of `row` elements keep the rows apart?  (Each stride passes what the smaller ones span, in any order:
// what slices, permutations and gaps of a buffer give.)
template <int N>
bool separate_rows(const int64_t (&strides)[N], const uint64_t (&sizes)[N], uint64_t row) {
  bool taken[N] = {};
  uint64_t span = row;
  for (int n = 0; n < N; ++n) {
    int next = -1;
    for (int i = 0; i < N; ++i)
      if (!taken[i] && (next < 0 || strides[i] < strides[next])) next = i;
    taken[next] = true;
    if (sizes[next] <= 1) continue;
    if (static_cast<uint64_t>(strides[next]) < span) return false;
    span += static_cast<uint64_t>(strides[next]) * (sizes[next] - 1);
  }
  return true;
}

bool good_channels(uint32_t channels, uint32_t inner) {
  return channels >= 1 && channels <= (1u << 24) && inner >= 1 && inner <= 131071u;
}

constexpr uint32_t kMostTokens = 0x7fffffffu;

// The linear product's arguments, but for the outputs.
int linear_args(rosetta_clear *h, const int8_t *q, int64_t q_pitch, const float *scale, uint32_t tokens,
                const void *packed, const float *w_scale, const float *bias, uint32_t channels, uint32_t inner,
                ClearLinearArgs *a) {
  if (!h || !good_channels(channels, inner) || tokens > kMostTokens || !good_pitch(q_pitch, inner))
    return ROSETTA_ERR_INVALID_ARG;
  if (tokens && (!q || !scale || !packed || !w_scale)) return ROSETTA_ERR_INVALID_ARG;
  if (!aligned(scale, 4) || !aligned(w_scale, 4) || !aligned(bias, 4) || !aligned(packed, 16)) return ROSETTA_ERR_INVALID_ARG;
  a->q = q;
  a->scale = scale;
  a->packed = static_cast<const int8_t *>(packed);
  a->w_scale = w_scale;
  a->bias = bias;
  a->q_pitch = q_pitch;
  a->tokens = tokens;
  a->channels = channels;
  a->inner = inner;
  a->k_steps = (inner + kPackK - 1) / kPackK;
  a->err_flag = h->d_err;
  return ROSETTA_OK;
}

// Does an output of `bytes` bytes touch any of the product's inputs?
bool linear_overlap(const ClearLinearArgs &a, const void *out, size_t bytes) {
  return overlaps(out, bytes, a.q, span(a.q_pitch, a.tokens, a.inner, 1)) || overlaps(out, bytes, a.scale, 4ull * a.tokens) ||
         overlaps(out, bytes, a.packed, rosetta_clear_packed_bytes(a.channels, a.inner)) ||
         overlaps(out, bytes, a.w_scale, 4ull * a.channels) || overlaps(out, bytes, a.bias, 4ull * a.channels);
}

// Make the workspace hold `bytes`; what it outgrows stays until the handle is freed.
int ensure_work(rosetta_clear *h, size_t bytes, cudaStream_t s) {
  if (h->work_bytes >= bytes) return ROSETTA_OK;
  cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
  if (cudaStreamIsCapturing(s, &capture) != cudaSuccess) {
    cudaGetLastError();
    return ROSETTA_ERR_CUDA;
  }
  if (capture != cudaStreamCaptureStatusNone) return ROSETTA_ERR_OOM;
  try {
    h->outgrown.reserve(h->outgrown.size() + 1);
  } catch (...) {
    return ROSETTA_ERR_OOM;
  }
  // (at least doubled where there is room for it, so that what stays behind is no more than the present one)
  size_t want = bytes > 2 * h->work_bytes ? bytes : 2 * h->work_bytes;
  void *p = nullptr;
  cudaError_t e = cudaMalloc(&p, want);
  if (e == cudaErrorMemoryAllocation && want > bytes) {
    cudaGetLastError();
    want = bytes;
    e = cudaMalloc(&p, want);
  }
  if (e != cudaSuccess) {
    cudaGetLastError();
    return cuda_fail(e);
  }
  if (h->work) h->outgrown.push_back(h->work);
  h->work = p;
  h->work_bytes = want;
  return ROSETTA_OK;
}

int run_linear(rosetta_clear *h, const ClearLinearArgs &a, int kind, cudaStream_t s) {
  if (cudaSetDevice(h->device) != cudaSuccess) return ROSETTA_ERR_CUDA;
  cudaError_t e;
  if (linear_few_ns(a, h->sms) <= linear_tc_ns(a, h->sms)) {
    e = launch_clear_linear_few(a, kind, h->sms, s);
  } else {
    const int r = ensure_work(h, linear_tc_bytes(a, h->sms), s);
    if (r != ROSETTA_OK) return r;
    e = launch_clear_linear_tc(a, kind, h->work, h->sms, s);
  }
  return e == cudaSuccess ? ROSETTA_OK : cuda_fail(e);
}

// The cache's description, shared by the append and the attention.
bool good_cache(const int8_t *k_cache, const int8_t *v_cache, const int64_t *strides, const float *k_scale,
                const float *v_scale, uint32_t heads, uint32_t dim, uint32_t pages, uint32_t page_tokens,
                const int32_t *page_table, uint32_t table_pitch) {
  if (!strides || !good_strides(strides)) return false;
  if (dim < 4 || dim > 256 || dim % 4 || page_tokens < 1 || page_tokens > 1024 || heads < 1 || heads > 4096) return false;
  if (pages > 0x7fffffffu || static_cast<uint64_t>(table_pitch) * page_tokens > (1u << 30)) return false;
  if (strides[2] < static_cast<int64_t>(dim)) return false;
  for (int i = 0; i < 3; ++i)
    if (strides[i] % 4) return false;
  return k_cache && v_cache && k_scale && v_scale && page_table && aligned(k_cache, 4) && aligned(v_cache, 4) &&
         aligned(k_scale, 4) && aligned(v_scale, 4) && aligned(page_table, 4);
}

}  // namespace

extern "C" {

int rosetta_clear_init(rosetta_clear **out, int cuda_device, size_t workspace_bytes) {
  if (!out) return ROSETTA_ERR_INVALID_ARG;
  *out = nullptr;
  rosetta_clear *h = new (std::nothrow) rosetta_clear;
  if (!h) return ROSETTA_ERR_OOM;
  h->device = cuda_device;
  int sms = 0;
  cudaError_t e = cudaSetDevice(cuda_device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, cuda_device);
  if (e == cudaSuccess) e = cudaMalloc(&h->d_err, sizeof(uint32_t));
  if (e == cudaSuccess) e = cudaMemset(h->d_err, 0, sizeof(uint32_t));
  if (e == cudaSuccess && workspace_bytes) e = cudaMalloc(&h->work, workspace_bytes);
  if (e != cudaSuccess) {
    cudaGetLastError();
    rosetta_clear_destroy(h);
    return cuda_fail(e);
  }
  h->sms = static_cast<uint32_t>(sms);
  h->work_bytes = workspace_bytes;
  *out = h;
  return ROSETTA_OK;
}

int rosetta_clear_norm(rosetta_clear *h, int type, const void *x, int64_t x_pitch, const void *residual,
                       int64_t residual_pitch, const float *gamma, float eps, uint32_t tokens, uint32_t width,
                       void *sum_out, int64_t sum_pitch, int8_t *q, int64_t q_pitch, float *scale, void *stream) {
  if (!h || !known_type(type) || width < 1 || width > (1u << 20) || tokens > kMostTokens || !(eps >= 0.0f) || isinf(eps))
    return ROSETTA_ERR_INVALID_ARG;
  if (!good_pitch(x_pitch, width) || !good_pitch(q_pitch, width) || (residual && !good_pitch(residual_pitch, width)) ||
      (sum_out && !good_pitch(sum_pitch, width)))
    return ROSETTA_ERR_INVALID_ARG;
  if (tokens == 0) return ROSETTA_OK;
  const size_t size = type_size(type);
  if (!x || !gamma || !q || !scale || !aligned(x, size) || !aligned(residual, size) || !aligned(sum_out, size) ||
      !aligned(gamma, 4) || !aligned(scale, 4))
    return ROSETTA_ERR_INVALID_ARG;
  const size_t nx = span(x_pitch, tokens, width, size), nr = span(residual_pitch, tokens, width, size);
  const size_t ns = span(sum_pitch, tokens, width, size), nq = span(q_pitch, tokens, width, 1);
  const struct {
    const void *p;
    size_t n;
  } in[] = {{x, nx}, {residual, nr}, {gamma, 4ull * width}}, out[] = {{sum_out, ns}, {q, nq}, {scale, 4ull * tokens}};
  for (int o = 0; o < 3; ++o) {
    for (int i = 0; i < 3; ++i) {
      const bool in_place = o == 0 && ((i == 0 && sum_out == x && sum_pitch == x_pitch) ||
                                       (i == 1 && sum_out == residual && sum_pitch == residual_pitch));
      if (!in_place && overlaps(out[o].p, out[o].n, in[i].p, in[i].n)) return ROSETTA_ERR_INVALID_ARG;
    }
    for (int i = 0; i < o; ++i)
      if (overlaps(out[o].p, out[o].n, out[i].p, out[i].n)) return ROSETTA_ERR_INVALID_ARG;
  }
  if (cudaSetDevice(h->device) != cudaSuccess) return ROSETTA_ERR_CUDA;
  ClearNormArgs a{};
  a.x = x;
  a.residual = residual;
  a.gamma = gamma;
  a.sum_out = sum_out;
  a.q = q;
  a.scale = scale;
  a.x_pitch = x_pitch;
  a.residual_pitch = residual_pitch;
  a.sum_pitch = sum_pitch;
  a.q_pitch = q_pitch;
  a.tokens = tokens;
  a.width = width;
  a.eps = eps;
  const cudaError_t e = launch_clear_norm(a, type, as_stream(stream));
  return e == cudaSuccess ? ROSETTA_OK : cuda_fail(e);
}

size_t rosetta_clear_packed_bytes(uint32_t channels, uint32_t inner) {
  if (!good_channels(channels, inner)) return 0;
  return static_cast<size_t>((channels + kPackRows - 1) / kPackRows) * ((inner + kPackK - 1) / kPackK) * kPackTile;
}

int rosetta_clear_pack_weights(rosetta_clear *h, const int8_t *weight, int64_t pitch, uint32_t channels,
                               uint32_t inner, void *packed, void *stream) {
  const size_t bytes = rosetta_clear_packed_bytes(channels, inner);
  if (!h || !bytes || !weight || !packed || !good_pitch(pitch, inner) || !aligned(packed, 16) ||
      overlaps(packed, bytes, weight, span(pitch, channels, inner, 1)))
    return ROSETTA_ERR_INVALID_ARG;
  if (bytes / 16 / 256 >= 0x7fffffffu) return ROSETTA_ERR_INVALID_ARG;
  if (cudaSetDevice(h->device) != cudaSuccess) return ROSETTA_ERR_CUDA;
  const cudaError_t e = launch_clear_pack(weight, pitch, channels, inner, static_cast<int8_t *>(packed), as_stream(stream));
  return e == cudaSuccess ? ROSETTA_OK : cuda_fail(e);
}

int rosetta_clear_linear(rosetta_clear *h, const int8_t *q, int64_t q_pitch, const float *scale, uint32_t tokens,
                         const void *packed, const float *w_scale, const float *bias, uint32_t channels,
                         uint32_t inner, int type, void *out, int64_t out_pitch, void *stream) {
  ClearLinearArgs a{};
  const int r = linear_args(h, q, q_pitch, scale, tokens, packed, w_scale, bias, channels, inner, &a);
  if (r != ROSETTA_OK) return r;
  if (!known_type(type) || !good_pitch(out_pitch, channels)) return ROSETTA_ERR_INVALID_ARG;
  if (tokens == 0) return ROSETTA_OK;
  const size_t size = type_size(type);
  if (!out || !aligned(out, size) || linear_overlap(a, out, span(out_pitch, tokens, channels, size)))
    return ROSETTA_ERR_INVALID_ARG;
  a.out = out;
  a.out_pitch = out_pitch;
  return run_linear(h, a, type, as_stream(stream));
}

int rosetta_clear_linear_codes(rosetta_clear *h, const int8_t *q, int64_t q_pitch, const float *scale,
                               uint32_t tokens, const void *packed, const float *w_scale, const float *bias,
                               uint32_t channels, uint32_t inner, uint32_t bits, float lo, float hi, uint8_t *code,
                               int64_t code_pitch, const int8_t *table, int8_t *values, int64_t values_pitch,
                               void *stream) {
  ClearLinearArgs a{};
  const int r = linear_args(h, q, q_pitch, scale, tokens, packed, w_scale, bias, channels, inner, &a);
  if (r != ROSETTA_OK) return r;
  if (bits < 1 || bits > 8 || !isfinite(lo) || !isfinite(hi) || !(lo < hi) || !good_pitch(code_pitch, channels) ||
      !table != !values || (values && !good_pitch(values_pitch, channels)))
    return ROSETTA_ERR_INVALID_ARG;
  const double inv = static_cast<double>(1u << bits) / (static_cast<double>(hi) - lo);
  if (!isfinite(static_cast<float>(inv))) return ROSETTA_ERR_INVALID_ARG;
  if (tokens == 0) return ROSETTA_OK;
  const size_t nc = span(code_pitch, tokens, channels, 1), nv = span(values_pitch, tokens, channels, 1);
  if (!code || linear_overlap(a, code, nc) || overlaps(code, nc, table, size_t{1} << bits)) return ROSETTA_ERR_INVALID_ARG;
  if (values && (linear_overlap(a, values, nv) || overlaps(values, nv, table, size_t{1} << bits) || overlaps(values, nv, code, nc)))
    return ROSETTA_ERR_INVALID_ARG;
  a.out = code;
  a.out_pitch = code_pitch;
  a.table = table;
  a.values = values;
  a.values_pitch = values_pitch;
  a.lo = lo;
  a.inv = static_cast<float>(inv);
  a.top = static_cast<float>((1u << bits) - 1);
  return run_linear(h, a, kOutCodes, as_stream(stream));
}

int rosetta_clear_cache_append(rosetta_clear *h, int type, const void *k, const int64_t *k_strides, const void *v,
                               const int64_t *v_strides, uint32_t batch, uint32_t tokens, uint32_t heads, uint32_t dim,
                               int8_t *k_cache, int8_t *v_cache, const int64_t *cache_strides, float *k_scale,
                               float *v_scale, uint32_t pages, uint32_t page_tokens, const int32_t *page_table,
                               uint32_t table_pitch, const int32_t *first, void *stream) {
  if (!h || !known_type(type) || !k_strides || !v_strides || !good_strides(k_strides) || !good_strides(v_strides) ||
      tokens > kMostTokens || batch > 65535)
    return ROSETTA_ERR_INVALID_ARG;
  if (batch == 0 || tokens == 0) return ROSETTA_OK;
  const size_t size = type_size(type);
  if (!good_cache(k_cache, v_cache, cache_strides, k_scale, v_scale, heads, dim, pages, page_tokens, page_table, table_pitch) ||
      !k || !v || !first || !aligned(k, size) || !aligned(v, size) || !aligned(first, 4) || 2 * heads > 65535)
    return ROSETTA_ERR_INVALID_ARG;
  // what is written: no byte of the caches twice, keys' and values' among them
  const int64_t apart = v_cache > k_cache ? v_cache - k_cache : k_cache - v_cache;
  if (!separate_rows<4>({cache_strides[0], cache_strides[1], cache_strides[2], apart}, {pages, heads, page_tokens, 2}, dim) ||
      overlaps(k_scale, 4ull * pages * heads, v_scale, 4ull * pages * heads))
    return ROSETTA_ERR_INVALID_ARG;
  if (cudaSetDevice(h->device) != cudaSuccess) return ROSETTA_ERR_CUDA;
  ClearAppendArgs a{};
  a.src[0] = k;
  a.src[1] = v;
  a.cache[0] = k_cache;
  a.cache[1] = v_cache;
  a.scale[0] = k_scale;
  a.scale[1] = v_scale;
  for (int i = 0; i < 3; ++i) {
    a.src_strides[0][i] = k_strides[i];
    a.src_strides[1][i] = v_strides[i];
    a.cache_strides[i] = cache_strides[i];
  }
  a.page_table = page_table;
  a.first = first;
  a.batch = batch;
  a.tokens = tokens;
  a.heads = heads;
  a.dim = dim;
  a.pages = pages;
  a.page_tokens = page_tokens;
  a.table_pitch = table_pitch;
  a.err_flag = h->d_err;
  const cudaError_t e = launch_clear_append(a, type, as_stream(stream));
  return e == cudaSuccess ? ROSETTA_OK : cuda_fail(e);
}

int rosetta_clear_attention(rosetta_clear *h, int type, const void *q, const int64_t *q_strides, uint32_t batch,
                            uint32_t tokens, uint32_t heads, uint32_t group, uint32_t dim, const int8_t *k_cache,
                            const int8_t *v_cache, const int64_t *cache_strides, const float *k_scale,
                            const float *v_scale, uint32_t pages, uint32_t page_tokens, const int32_t *page_table,
                            uint32_t table_pitch, const int32_t *lengths, float softmax_scale, void *out,
                            const int64_t *out_strides, void *stream) {
  if (!h || !known_type(type) || !q_strides || !out_strides || !good_strides(q_strides) || !good_strides(out_strides) ||
      group < 1 || group > 128 || tokens > (1u << 24) || batch > 65535 || !isfinite(softmax_scale))
    return ROSETTA_ERR_INVALID_ARG;
  if (batch == 0 || tokens == 0) return ROSETTA_OK;
  const size_t size = type_size(type);
  if (!good_cache(k_cache, v_cache, cache_strides, k_scale, v_scale, heads, dim, pages, page_tokens, page_table, table_pitch) ||
      !q || !out || !lengths || !aligned(q, size) || !aligned(out, size) || !aligned(lengths, 4))
    return ROSETTA_ERR_INVALID_ARG;
  // (rows of q and out, over all batches: what the launches' grids count)
  if (static_cast<double>(batch) * tokens * heads * group > 2147483000.0) return ROSETTA_ERR_INVALID_ARG;
  const auto reach = [&](const int64_t *s) {
    return (static_cast<size_t>(batch - 1) * s[0] + static_cast<size_t>(tokens - 1) * s[1] +
            static_cast<size_t>(heads * group - 1) * s[2] + dim) * size;
  };
  if (overlaps(out, reach(out_strides), q, reach(q_strides)) ||
      !separate_rows<3>({out_strides[0], out_strides[1], out_strides[2]}, {batch, tokens, heads * group}, dim))
    return ROSETTA_ERR_INVALID_ARG;
  if (cudaSetDevice(h->device) != cudaSuccess) return ROSETTA_ERR_CUDA;
  ClearAttentionArgs a{};
  a.q = q;
  a.out = out;
  for (int i = 0; i < 3; ++i) {
    a.q_strides[i] = q_strides[i];
    a.out_strides[i] = out_strides[i];
    a.cache_strides[i] = cache_strides[i];
  }
  a.k_cache = k_cache;
  a.v_cache = v_cache;
  a.k_scale = k_scale;
  a.v_scale = v_scale;
  a.page_table = page_table;
  a.lengths = lengths;
  a.batch = batch;
  a.tokens = tokens;
  a.heads = heads;
  a.group = group;
  a.dim = dim;
  a.pages = pages;
  a.page_tokens = page_tokens;
  a.table_pitch = table_pitch;
  a.softmax_scale = softmax_scale;
  a.err_flag = h->d_err;
  const cudaStream_t s = as_stream(stream);
  cudaError_t e;
  if (attend_many_takes(a)) {
    const int r = ensure_work(h, attend_many_bytes(a, type, h->sms), s);
    if (r != ROSETTA_OK) return r;
    e = launch_clear_attention_many(a, type, h->work, h->sms, s);
  } else if (attend_few_takes(a)) {
    const int r = ensure_work(h, attend_few_bytes(a, h->sms), s);
    if (r != ROSETTA_OK) return r;
    e = launch_clear_attention_few(a, type, h->work, h->sms, s);
  } else {
    e = launch_clear_attention(a, type, s);
  }
  return e == cudaSuccess ? ROSETTA_OK : cuda_fail(e);
}

int rosetta_clear_sync_status(rosetta_clear *h, void *stream) {
  if (!h) return ROSETTA_ERR_INVALID_ARG;
  if (cudaSetDevice(h->device) != cudaSuccess) return ROSETTA_ERR_CUDA;
  cudaError_t e = cudaStreamSynchronize(as_stream(stream));
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) return cuda_fail(e);
  uint32_t flag = 0;
  e = cudaMemcpy(&flag, h->d_err, sizeof(flag), cudaMemcpyDeviceToHost);
  if (e == cudaSuccess && flag) e = cudaMemset(h->d_err, 0, sizeof(flag));
  if (e != cudaSuccess) return cuda_fail(e);
  if (flag == 2) return ROSETTA_ERR_TIMEOUT;
  return flag ? ROSETTA_ERR_INVALID_ARG : ROSETTA_OK;
}

void rosetta_clear_destroy(rosetta_clear *h) {
  if (!h) return;
  cudaSetDevice(h->device);
  cudaDeviceSynchronize();
  cudaFree(h->d_err);
  cudaFree(h->work);
  for (void *p : h->outgrown) cudaFree(p);
  delete h;
}

}  // extern "C"
