// Rows of the paged 8-bit cache moved and read back.
//
// Keeping: rows first + path[i] become rows first + i, under a page's scale
//   s' = max of the scales of the pages that its rows come from,  q' = rint(q (s / s')).
// A unit of work is one cached head of one sequence, keys or values, page after page: path[i] >= i and increasing, so what is
// written never lies before what is still to be read but for the rows in the unit's registers.  Bound by the chain of a
// unit (path, pages, scales and rows, one after another): what 256 sequences accepted of 64 drafted tokens, 8 heads of 128,
// 8.7 us, one sequence 3.6.
//
// Reading: out = q s[page][head].  Bound by its bytes, one read and two or four written for each value: 32 uneven sequences of up to
// 4096 positions, 8 heads of 128, into bfloat16 84 us, 5.1 TB/s; all of 4096 143 us, 5.6 TB/s; 16 of 4096
// into single precision 107 us, 6.3 TB/s.
#include <stdint.h>

#include "clear.h"

namespace rosetta {

namespace {

// The low byte of rint(v), |v| < 2^22: v + 1.5 * 2^23 has it in its last bits (ties to even).
__device__ __forceinline__ int8_t rint_byte(float v) { return static_cast<int8_t>(__float_as_uint(v + 12582912.0f)); }

template <int VEC>
struct alignas(VEC) Bytes {
  int8_t v[VEC];
};

template <int VEC>
__device__ __forceinline__ Bytes<VEC> rescaled(Bytes<VEC> q, float ratio) {
#pragma unroll
  for (int e = 0; e < VEC; ++e) q.v[e] = rint_byte(fminf(fmaxf(q.v[e] * ratio, -128.0f), 127.0f));
  return q;
}

// Shared memory of a unit: the path, and of each row of the present page where it comes from and under which scale.
__host__ __device__ constexpr uint32_t keep_bytes(uint32_t tokens, uint32_t page_tokens) { return (tokens + 1) / 2 * 8 + page_tokens * 12 + page_tokens % 2 * 4; }

// WARPS of a unit: one (four units a block) or four.  VEC bytes an access, of which a thread keeps `KEPT` between reading and
// writing.  (64 registers a thread: 256 sequences are resident at once; with 96 they are not, 11.3 us, and 40 spill, 12.4.)
template <int WARPS, int VEC>
__global__ void __launch_bounds__(128, 8) keep_kernel(const ClearKeepArgs a) {
  constexpr uint32_t THREADS = 32 * WARPS, KEPT = VEC == 16 ? 2 : 4;
  extern __shared__ __align__(8) unsigned char smem[];
  __shared__ float s_most[4];
  const uint32_t tid = threadIdx.x % THREADS, own = threadIdx.x / THREADS, unit = blockIdx.x * (4 / WARPS) + own;
  const uint32_t kv = unit & 1u, head = unit >> 1, b = blockIdx.y;
  if (head >= a.heads) return;  // (whole warps; there is no barrier where a block has several units)
  const auto meet = [] {
    if constexpr (WARPS == 1)
      __syncwarp();
    else
      __syncthreads();
  };
  int32_t *s_path = reinterpret_cast<int32_t *>(smem + own * keep_bytes(a.tokens, a.page_tokens));
  int64_t *s_from = reinterpret_cast<int64_t *>(s_path + (a.tokens + 1) / 2 * 2);
  float *s_scale = reinterpret_cast<float *>(s_from + a.page_tokens);
  const int64_t first = a.first[b];
  const int32_t given = a.count[b];
  const int32_t *path = a.path + static_cast<int64_t>(b) * a.path_pitch;
  for (uint32_t i = tid; i < a.tokens; i += THREADS) s_path[i] = path[i];
  if (first < 0 || given == 0) return;
  const uint32_t count = given > 0 ? static_cast<uint32_t>(given) : 0u;
  meet();
  bool bad = given < 0 || count > a.tokens;
  for (uint32_t i = tid; i < min(count, a.tokens); i += THREADS) {
    const int32_t v = s_path[i];
    bad |= v < 0 || static_cast<uint32_t>(v) >= a.tokens || (i && v <= s_path[i - 1]);
  }
  // (a path that is none moves nothing)
  if (WARPS == 1 ? __any_sync(0xffffffffu, bad) : __syncthreads_or(bad)) {
    if (tid == 0) atomicMax(a.err_flag, 1u);
    return;
  }
  const uint32_t page_rows = a.page_tokens, packs = a.dim / VEC;
  const int32_t *table = a.page_table + static_cast<size_t>(b) * a.table_pitch;
  int8_t *cache = a.cache[kv] + static_cast<int64_t>(head) * a.cache_strides[1];
  const int64_t line = a.cache_strides[2], end = first + count;
  const auto page_of = [&](uint32_t slot) {
    const int32_t page = slot < a.table_pitch ? table[slot] : -1;
    if (page >= 0 && static_cast<uint32_t>(page) < a.pages) return page;
    atomicMax(a.err_flag, 1u);
    return -1;
  };
  const uint32_t last_slot = static_cast<uint32_t>((end - 1) / page_rows);  // (positions and slots below 2^32)
  for (uint32_t slot = static_cast<uint32_t>(first) / page_rows; slot <= last_slot; ++slot) {
    const int64_t row0 = static_cast<int64_t>(slot) * page_rows, lo = first > row0 ? first : row0, hi = end < row0 + page_rows ? end : row0 + page_rows;
    const int32_t page = page_of(slot);
    if (page < 0) continue;  // (the same for the unit)
    int8_t *dst = cache + page * a.cache_strides[0];
    float *scale = a.scale[kv] + static_cast<size_t>(page) * a.heads + head;
    const uint32_t old_rows = static_cast<uint32_t>(lo - row0), rows = static_cast<uint32_t>(hi - lo);
    const float was = *scale;
    // the largest scale, a NaN where there is one
    float most = old_rows ? was : -__int_as_float(0x7f800000);
    const auto take = [&](float v) { most = v != v || most != most ? __int_as_float(0x7fc00000) : fmaxf(most, v); };
    for (uint32_t i = tid; i < rows; i += THREADS) {
      const uint32_t from = static_cast<uint32_t>(first + s_path[lo - first + i]), at = from / page_rows;
      const int32_t of = at == slot ? page : page_of(at);
      s_from[i] = of < 0 ? -1 : of * a.cache_strides[0] + from % page_rows * line;
      s_scale[i] = of < 0 ? 0.0f : of == page ? was : a.scale[kv][static_cast<size_t>(of) * a.heads + head];
      if (of >= 0) take(s_scale[i]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) take(__shfl_xor_sync(0xffffffffu, most, o));
    if constexpr (WARPS > 1) {
      if (tid % 32 == 0) s_most[tid / 32] = most;
      __syncthreads();
#pragma unroll
      for (uint32_t w = 0; w < WARPS; ++w) take(s_most[w]);
    } else {
      __syncwarp();
    }
    const float now = most, div = now > 0.0f ? now : 1.0f;
    const bool number = now == now;  // (a NaN: bytes as they are)
    if (old_rows && now != was && number) {
      const float ratio = was / div;
      for (uint32_t i = tid; i < old_rows * packs; i += THREADS) {
        Bytes<VEC> *p = reinterpret_cast<Bytes<VEC> *>(dst + i / packs * line + i % packs * VEC);
        *p = rescaled(*p, ratio);
      }
    }
    // a few packs a thread at a time, all read before any is written; what stays as it is is not touched
    const int64_t to = page * a.cache_strides[0] + old_rows * line;
    for (uint32_t i0 = 0; i0 < rows * packs; i0 += THREADS * KEPT) {
      Bytes<VEC> kept[KEPT];
      int8_t *at[KEPT];
#pragma unroll
      for (uint32_t k = 0; k < KEPT; ++k) {
        const uint32_t i = i0 + k * THREADS + tid, row = i / packs, d = (i - row * packs) * VEC;
        at[k] = nullptr;
        if (row >= rows || s_from[row] < 0) continue;
        const float s = s_scale[row];
        const bool other = number && s != now;
        if (!other && s_from[row] == to + row * line) continue;
        at[k] = cache + to + row * line + d;
        kept[k] = *reinterpret_cast<const Bytes<VEC> *>(cache + s_from[row] + d);
        if (other) kept[k] = rescaled(kept[k], s / div);
      }
      meet();
#pragma unroll
      for (uint32_t k = 0; k < KEPT; ++k)
        if (at[k]) *reinterpret_cast<Bytes<VEC> *>(at[k]) = kept[k];
      meet();
    }
    if (tid == 0 && most != -__int_as_float(0x7f800000)) *scale = now;
    meet();  // (the rows' list is free again)
  }
}

template <int VEC>
cudaError_t launch_keep(const ClearKeepArgs &a, cudaStream_t s) {
  // a warp a unit where the path is short (256 sequences of 64 tokens 9 us against 19, 64 of 200 5.6 against 5.2); shared memory: 32 KB
  // at most
  const uint32_t bytes = keep_bytes(a.tokens, a.page_tokens);
  if (a.tokens <= 128 && bytes <= 8192)
    keep_kernel<1, VEC><<<dim3((2 * a.heads + 3) / 4, a.batch), 128, 4 * bytes, s>>>(a);
  else
    keep_kernel<4, VEC><<<dim3(2 * a.heads, a.batch), 128, bytes, s>>>(a);
  return cudaGetLastError();
}

// ---- reading ----

// A byte (biased by 128, as the last one of 2^23's word) as a number.
__device__ __forceinline__ float number_of(uint32_t biased, uint32_t select) {
  return __uint_as_float(__byte_perm(biased, 0x4b000000u, select)) - 8388736.0f;
}

template <typename T>
__device__ __forceinline__ uint32_t two_of(float x, float y) {
  const T a = from_float<T>(x), b = from_float<T>(y);
  return static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(&a)) | static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(&b)) << 16;
}

// 32 bytes: a whole sector at once
__device__ __forceinline__ void store_sector(void *to, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
               "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}

// A thread takes VEC bytes of ROWS rows, in flight at once, `apart` positions from each other.  WIDE: outputs in whole sectors.
template <typename T, int VEC, bool WIDE, uint32_t ROWS>
__global__ void __launch_bounds__(256) read_kernel(const ClearReadArgs a, uint32_t packs, uint32_t apart) {
  const uint32_t b = blockIdx.z, head = blockIdx.y >> 1, kv = blockIdx.y & 1u;
  const uint32_t in_block = threadIdx.x / packs, d = threadIdx.x % packs * VEC;
  if (in_block >= apart) return;
  const int64_t most = static_cast<int64_t>(a.table_pitch) * a.page_tokens, given = a.lengths[b], first = a.first[b];
  if (given > most && threadIdx.x == 0) atomicMax(a.err_flag, 1u);
  const int64_t len = given < most ? given : most;
  const int32_t *table = a.page_table + static_cast<size_t>(b) * a.table_pitch;
  const int8_t *cache = a.cache[kv] + static_cast<int64_t>(head) * a.cache_strides[1] + d;
  const uint32_t row0 = blockIdx.x * (apart * ROWS) + in_block;
  Bytes<VEC> q[ROWS];
  float s[ROWS];
  int32_t page[ROWS];
  uint32_t in_page[ROWS];
#pragma unroll
  for (uint32_t k = 0; k < ROWS; ++k) {
    const uint32_t i = row0 + k * apart;
    const int64_t at = first + i;
    page[k] = -1;
    if (i >= a.tokens || at < 0 || at >= len) continue;
    const uint32_t slot = static_cast<uint32_t>(at) / a.page_tokens;  // (below 2^30)
    in_page[k] = static_cast<uint32_t>(at) - slot * a.page_tokens;
    page[k] = table[slot];
    if (page[k] < 0 || static_cast<uint32_t>(page[k]) >= a.pages) {
      atomicMax(a.err_flag, 1u);
      page[k] = -1;
    }
  }
#pragma unroll
  for (uint32_t k = 0; k < ROWS; ++k) {
    if (page[k] < 0) continue;
    q[k] = *reinterpret_cast<const Bytes<VEC> *>(cache + page[k] * a.cache_strides[0] + in_page[k] * a.cache_strides[2]);
    s[k] = a.scale[kv][static_cast<size_t>(page[k]) * a.heads + head];
  }
#pragma unroll
  for (uint32_t k = 0; k < ROWS; ++k) {
    if (page[k] < 0) continue;
    T *out = static_cast<T *>(a.out[kv]) + static_cast<int64_t>(b) * a.out_strides[kv][0] + static_cast<int64_t>(row0 + k * apart) * a.out_strides[kv][1] +
             static_cast<int64_t>(head) * a.out_strides[kv][2] + d;
    const uint32_t *words = reinterpret_cast<const uint32_t *>(&q[k]);
    float v[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) v[e] = number_of(words[e / 4] ^ 0x80808080u, 0x7440u + e % 4) * s[k];
    if constexpr (WIDE && sizeof(T) == 2) {
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = two_of<T>(v[2 * e], v[2 * e + 1]);
      store_sector(out, w);
    } else if constexpr (WIDE) {
#pragma unroll
      for (int h = 0; h < VEC; h += 8) {
        uint32_t w[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(v[h + e]);
        store_sector(out + h, w);
      }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) out[e] = from_float<T>(v[e]);
    }
  }
}

template <typename T, int VEC, bool WIDE>
cudaError_t launch_read(const ClearReadArgs &a, cudaStream_t s) {
  // four rows a thread where that leaves enough blocks to fill the GPU (32 uneven sequences of up to 4096 82 us, one row 91), else one
  // (2 of 131 tokens 2.5 us against 5)
  const uint32_t packs = a.dim / VEC, apart = 256 / packs;
  const auto blocks = [&](uint32_t rows) { return dim3((a.tokens + apart * rows - 1) / (apart * rows), 2 * a.heads, a.batch); };
  const dim3 four = blocks(4);
  if (static_cast<uint64_t>(four.x) * four.y * four.z >= 1024)
    read_kernel<T, VEC, WIDE, 4><<<four, 256, 0, s>>>(a, packs, apart);
  else
    read_kernel<T, VEC, WIDE, 1><<<blocks(1), 256, 0, s>>>(a, packs, apart);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_read(const ClearReadArgs &a, cudaStream_t s) {
  uintptr_t in = static_cast<uintptr_t>(a.cache_strides[0] | a.cache_strides[1] | a.cache_strides[2] | a.dim), out = 0;
  for (int kv = 0; kv < 2; ++kv) {
    in |= reinterpret_cast<uintptr_t>(a.cache[kv]);
    out |= reinterpret_cast<uintptr_t>(a.out[kv]);
    for (int i = 0; i < 3; ++i) out |= static_cast<uintptr_t>(a.out_strides[kv][i] * sizeof(T));
  }
  return in % 16 == 0 && out % 32 == 0 ? launch_read<T, 16, true>(a, s) : launch_read<T, 4, false>(a, s);
}

}  // namespace

cudaError_t launch_clear_keep(const ClearKeepArgs &a, cudaStream_t s) {
  uintptr_t at = reinterpret_cast<uintptr_t>(a.cache[0]) | reinterpret_cast<uintptr_t>(a.cache[1]) | a.dim;
  for (int i = 0; i < 3; ++i) at |= static_cast<uintptr_t>(a.cache_strides[i]);
  return at % 16 == 0 ? launch_keep<16>(a, s) : launch_keep<4>(a, s);
}

cudaError_t launch_clear_read(const ClearReadArgs &a, int type, cudaStream_t s) {
  if (type == kOutF32) return launch_read<float>(a, s);
  if (type == kOutF16) return launch_read<__half>(a, s);
  return launch_read<__nv_bfloat16>(a, s);
}

}  // namespace rosetta
