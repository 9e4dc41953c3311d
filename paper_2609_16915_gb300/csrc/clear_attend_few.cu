// Causal attention over the paged 8-bit cache for few query rows a cached head: decoding.
//
// Bound by reading keys and values once (two 8-bit rows a position and cached head, 79.8 us of copies at the
// measured rate for 64 sequences of up to 8192 positions, 8 heads of 128: 108 us, 5.0 TB/s; all of 8192: 185 us, 5.8 TB/s),
// and as closely by converting each value for at most 8 rows.  Query rows of one cached head (its
// group's heads, and the tokens of a short run) share what is read: they are the columns of
//   S^T = K Q^T (16 positions x 8 rows x 16 dimensions a product)  and  O^T = V^T P^T (16 dimensions x 8 rows x
// 16 positions), with the 8-bit values made f16 in registers (exact) and the scales kept outside the
// products.  In units of log 2, with sv a power of two,
//   P = 2^(s - m),  l = sum P,  O = sum P (vs / sv) 2^7 V,  out = O sv 2^-7 / l,
// where m is no more than 8 below the largest s + log2(vs / sv) that the row has seen: what is rounded to f16 is at most 2^15,
// and 2^-14 (the least normal f16) is far below the largest of the row's own terms, whatever the scales of pages without
// weight in it or out of its sight.  (A reference of the scores alone, and terms over the largest scale, lost those bits.)
// Single-precision queries are split into two f16 each, and the weights too but for bfloat16, whose own rounding hides that of
// 11 bits (float16 outputs 2.1e-4 off, their rounding alone, against 3.0e-4; 64 sequences of up to 8192 110 us against 108).  The tensor cores cut sums off
// instead of rounding them, so single precision adds each tile's products to the outputs (rounded) and the halves' scores at the end.
//
// A block of four warps takes one cached head, one group of 8 NB rows and one range of the positions; a warp
// takes every fourth tile of 16 positions, copied ahead into a ring of its own by cp.async (lanes read what others
// of the warp copied: __syncwarp after each wait, no block-wide barrier but one each 256 tiles).  Blocks of one sequence join through partial results (m, l, O) in the
// workspace and attend_join_kernel; a sequence that fits one range is written at once.
#include <stdint.h>

#include <type_traits>

#include "clear_attend.cuh"
#include "dsmem.cuh"

namespace rosetta {

namespace {

constexpr int kWarps = 4;
constexpr uint32_t kSegment = 256;      // tiles whose pages and scales are in shared memory at a time
constexpr float kRaise = 8.0f, kLift = 128.0f;
constexpr float kLog2e = 1.44269504088896340736f;

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ void mma_16x8x16(float (&d)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}

// an 8 x 8 matrix of f16, two of a row in each lane, transposed
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

// bytes (biased by 128) of a permuted word pair as f16: 1024 + u, minus 1152
__device__ __forceinline__ uint32_t biased_f16(uint32_t u, uint32_t select) {
  const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
  uint32_t v = __byte_perm(u, 0x64646464u, select);
  const __half2 h = __hsub2(*reinterpret_cast<__half2 *>(&v), off);
  return *reinterpret_cast<const uint32_t *>(&h);
}

__device__ __forceinline__ void copy_async(uint32_t dst, const void *src, bool valid) {
  const uint32_t size = valid ? 16 : 0;  // (nothing is read for 0: zeros)
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(size) : "memory");
}

// DP: the head's dimension, rounded up to 64, 128 or 256
template <int DP>
struct Few {
  static constexpr uint32_t TILE = 16 * DP * 2;                      // bytes of a tile's keys and values
  static constexpr uint32_t DEPTH = DP == 64 ? 6 : DP == 128 ? 3 : 2;  // tiles of a warp's ring
  static constexpr uint32_t RING = kWarps * DEPTH * TILE;
  static constexpr uint32_t BLOCKS = DP == 256 ? 2 : 4;              // an SM
};

__device__ __forceinline__ int64_t length_of(const ClearAttentionArgs &a, uint32_t b) {
  const int64_t len = a.lengths[b], most = static_cast<int64_t>(a.table_pitch) * a.page_tokens;
  if (len > most && threadIdx.x == 0) atomicMax(a.err_flag, 1u);
  return len > most ? most : len;
}

// TREE: under a mask.  A row sees every position before the drafted ones, and of those the bits of its own row of the mask.
template <typename T, int DP, int NB, bool TREE>
__global__ void __launch_bounds__(32 * kWarps, NB == 1 ? Few<DP>::BLOCKS : 2) attend_few_kernel(const AttendArgs f) {
  using F = Few<DP>;
  constexpr bool SPLIT = sizeof(T) == 4;     // queries and weights in two halves
  constexpr int H = SPLIT ? 2 : 1;
  constexpr int HP = std::is_same<T, __nv_bfloat16>::value ? 1 : 2;  // parts of a weight
  constexpr int KC = DP / 16;                // products of 16 dimensions
  constexpr int MT = DP / 16;                // tiles of 16 dimensions of O^T
  constexpr int VB = DP / 8;                 // bytes of a value row in a lane
  const ClearAttentionArgs &a = f.a;
  extern __shared__ __align__(16) unsigned char ring[];
  __shared__ int32_t s_page[kSegment];
  __shared__ int64_t s_at[kSegment];  // where the tiles lie in the caches
  __shared__ float s_ks[kSegment], s_vs[kSegment];
  __shared__ int32_t s_top[kWarps];
  __shared__ uint32_t s_mask[TREE ? 8 * NB : 1][33];  // the rows' words (up to 32)
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
  const uint32_t split = blockIdx.x % f.splits, group = blockIdx.x / f.splits % f.groups;
  const uint32_t own_head = blockIdx.x / f.splits / f.groups, bh = f.first + own_head, kh = bh % a.heads, b = bh / a.heads;
  const uint32_t rows = a.tokens * a.group, row0 = group * (8 * NB);
  const int64_t len = length_of(a, b);
  const uint32_t end = group_end<TREE>(a, len, min(row0 + 8 * NB, rows) - 1);
  const uint32_t share = split_share(f, end), lo = split * share, hi = min(end, lo + share);
  if (split > 0 && lo >= end) return;
  const bool alone = end <= share;  // (the first block of an empty sequence writes its zeros)

  // the rows' last positions, and their queries as B operands: row g of a group of eight, dimensions 16 t + 4 c
  // (+ 64 for every four c)
  int32_t last[NB][2];  // of rows 2 t, 2 t + 1
  float factor[NB][2];
  uint32_t qf[H][NB][KC][2];
  float o[NB][MT][4] = {}, m[NB][2], l[NB][2] = {};
  int32_t most = kNoScale, unit = 0;  // of the value scales so far: the largest exponent, and that of sv
#pragma unroll
  for (int n = 0; n < NB; ++n) m[n][0] = m[n][1] = neg_inf();
  const int32_t *table = a.page_table + static_cast<size_t>(b) * a.table_pitch;
  unsigned char *own = ring + warp * (F::DEPTH * F::TILE);
  const uint32_t own_addr = smem_addr(own);
  const uint32_t tiles_hi = (hi + 15) / 16;
  // A warp copies a tile's rows in the order of its lanes, 16 bytes each (other orders of the same bytes took up to 40 % longer),
  // with the chunks of a row moved so that the reads below meet few banks twice: keys, chunk t of each 64 bytes of row g;
  // values, VB bytes at VB g of rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9.
  // (16 rows of a page lie within 2^31 bytes: attend_few_takes)
  constexpr int CH = DP / 16;  // 16-byte chunks of a row
  const auto move = [](uint32_t row) {  // of a value row's chunks
    const uint32_t r = row >> 1 & 3u;
    return CH == 4 ? r : CH == 8 ? 2 * r : (r & 1u) | (r & 2u) << 1;
  };
  const int64_t head_at = static_cast<int64_t>(kh) * a.cache_strides[1];
  const uint32_t row_step = static_cast<uint32_t>(a.cache_strides[2]);
  const uint32_t k_dst = lane / CH * DP + ((lane % CH) ^ (CH >= 8 ? (lane / CH & 1u) * 4 : 0u)) * 16;
  const bool inside = lane % CH * 16 < a.dim;
  // of a lane's copies of a tile: place in the first, way on to the next (zero where it reads nothing)
  const uint32_t lane_at = inside ? lane / CH * row_step + lane % CH * 16 : 0, lane_on = inside ? 512 / DP * row_step : 0;
  int32_t whole = 0x7fffffff;  // the last position that every row sees
  if constexpr (TREE) {
    if (static_cast<int64_t>(hi) > len - a.tokens) {  // (the block meets before it uses them)
      const uint32_t words = (a.tokens + 31) / 32;
      for (uint32_t i = threadIdx.x; i < 8 * NB * words; i += blockDim.x) {
        const uint32_t r = row0 + i / words;
        s_mask[i / words][i % words] = r < rows ? a.mask[static_cast<int64_t>(b) * a.mask_strides[0] + static_cast<int64_t>(r / a.group) * a.mask_strides[1] + i % words] : 0u;
      }
    }
  }
  for (uint32_t seg = lo / 16; seg < tiles_hi; seg += kSegment) {
    const uint32_t count = min(kSegment, tiles_hi - seg);
    __syncthreads();
    int32_t top = kNoScale;
    for (uint32_t i = threadIdx.x; i < count; i += blockDim.x) {
      int32_t page = table[(seg + i) * 16 / a.page_tokens];
      if (page < 0 || static_cast<uint32_t>(page) >= a.pages) {
        atomicMax(a.err_flag, 1u);
        page = -1;
      }
      s_page[i] = page;
      s_at[i] = page < 0 ? 0 : page * a.cache_strides[0] + head_at + static_cast<int64_t>((seg + i) * 16 % a.page_tokens) * a.cache_strides[2];
      const size_t at = static_cast<size_t>(page) * a.heads + kh;
      s_ks[i] = page < 0 ? 0.0f : a.k_scale[at];
      float v = page < 0 ? 0.0f : a.v_scale[at];
      if (fabsf(v) == -neg_inf()) v = __int_as_float(0x7fc00000);  // no number either: kept out of the maximum
      s_vs[i] = v;
      top = max(top, scale_exponent(v));
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) s_top[warp] = top;
    __syncthreads();
    most = max(most, max(max(s_top[0], s_top[1]), max(s_top[2], s_top[3])));
    const int32_t grown = scale_unit(most) - unit;  // (the same for the block)
    if (grown != 0) {
      // from here on s + log2(vs / sv) counts from a larger sv: m goes down by as much, or as far as l has room, and O the rest
      unit += grown;
      if (seg != lo / 16) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int32_t down = min(grown, max(0, 100 + 127 - static_cast<int32_t>(__float_as_uint(l[n][e]) >> 23)));
            m[n][e] -= static_cast<float>(down);
            l[n][e] = scalbnf(l[n][e], down);
            const float keep = scalbnf(1.0f, down - grown);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              o[n][i][e] *= keep;
              o[n][i][e + 2] *= keep;
            }
          }
      }
    }
    const float vlift = scalbnf(kLift, -unit);

    const auto issue = [&](uint32_t i, uint32_t slot) {
      if (i < count) {
        const bool in = s_page[i] >= 0 && inside;
        const int8_t *kt = a.k_cache + s_at[i], *vt = a.v_cache + s_at[i];
        const uint32_t dst = own_addr + slot * F::TILE, vdst = dst + 16 * DP;
#pragma unroll
        for (int i = 0; i < DP / 32; ++i) {
          const uint32_t from = lane_at + i * lane_on;
          copy_async(dst + i * 512 + k_dst, kt + from, in);
          const uint32_t row = i * (512 / DP) + lane / CH;
          copy_async(vdst + row * DP + ((lane % CH) ^ move(row)) * 16, vt + from, in);
        }
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (uint32_t i = 0; i + 1 < F::DEPTH; ++i) issue(warp + i * kWarps, i);
    if (seg == lo / 16) {  // (once, with the first tiles on their way)
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        const uint32_t row = row0 + n * 8 + g;
        const T *q = static_cast<const T *>(a.q) + static_cast<int64_t>(b) * a.q_strides[0] +
                     static_cast<int64_t>(row / a.group) * a.q_strides[1] +
                     static_cast<int64_t>(kh * a.group + row % a.group) * a.q_strides[2];
        // four consecutive elements an access, kept as they are where their f16 will be
        const bool four = (reinterpret_cast<uintptr_t>(a.q) | static_cast<uintptr_t>((a.q_strides[0] | a.q_strides[1] | a.q_strides[2]) * sizeof(T))) % (4 * sizeof(T)) == 0;
        struct alignas(4 * sizeof(T)) Four {
          T v[4];
        };
        const auto place = [](int c) { return 64 * (c / 4) + 4 * (c % 4); };
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const uint32_t d = 16 * t + place(c);
          Four x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x.v[e] = from_float<T>(0.0f);
          if (row < rows && d < a.dim) {  // (dim is a multiple of 16)
            if (four) {
              x = *reinterpret_cast<const Four *>(q + d);
            } else {
#pragma unroll
              for (int e = 0; e < 4; ++e) x.v[e] = q[d + e];
            }
          }
          const uint32_t *bits = reinterpret_cast<const uint32_t *>(&x);
#pragma unroll
          for (int h = 0; h < H; ++h) qf[h][n][c][0] = bits[2 * h], qf[h][n][c][1] = bits[2 * h + 1];
        }
        const auto given = [&](int c, float (&v)[4]) {
          if constexpr (H == 2) {
            v[0] = __uint_as_float(qf[0][n][c][0]), v[1] = __uint_as_float(qf[0][n][c][1]);
            v[2] = __uint_as_float(qf[H - 1][n][c][0]), v[3] = __uint_as_float(qf[H - 1][n][c][1]);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint16_t half = static_cast<uint16_t>(qf[0][n][c][e / 2] >> (e % 2 * 16));
              v[e] = to_float(*reinterpret_cast<const T *>(&half));
            }
          }
        };
        float top = 0.0f;
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          float v[4];
          given(c, v);
#pragma unroll
          for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(v[e]));
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // a power of two that brings the row's largest value to [1, 2): exact (within the range of exponents)
        const int ex = min(max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -126), 126);
        const float down = __int_as_float((127 - ex) << 23), up = __int_as_float((127 + ex) << 23);
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          float v[4];
          given(c, v);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] *= down;
#pragma unroll
          for (int h = 0; h < H; ++h)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
              const __half2 x = __floats2half2_rn(v[2 * p], v[2 * p + 1]);
              qf[h][n][c][p] = *reinterpret_cast<const uint32_t *>(&x);
              v[2 * p] -= __low2float(x);
              v[2 * p + 1] -= __high2float(x);
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          factor[n][i] = __shfl_sync(0xffffffffu, up, (2 * t + i) * 4) * (a.softmax_scale * kLog2e);
          const uint32_t r = row0 + n * 8 + 2 * t + i;
          last[n][i] = r < rows ? static_cast<int32_t>(TREE ? len - a.tokens - 1 : len - a.tokens + r / a.group) : -1;
        }
      }
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (row0 + n * 8 + 2 * t + e < rows) whole = min(whole, last[n][e]);
      whole = min(whole, __shfl_xor_sync(0xffffffffu, whole, 1));
      whole = min(whole, __shfl_xor_sync(0xffffffffu, whole, 2));
    }
    uint32_t slot = 0;
    for (uint32_t i = warp; i < count; i += kWarps) {
      asm volatile("cp.async.wait_group %0;" ::"n"(F::DEPTH - 2) : "memory");
      __syncwarp();
      const unsigned char *tile = own + slot * F::TILE;
      // ---- scores: positions g, g + 8 (rows of S^T), query rows 2 t, 2 t + 1 ----
      float s[NB][4] = {}, fine[NB][4] = {};  // (fine: of the queries' second halves)
#pragma unroll
      for (int j = 0; j < DP / 64; ++j) {
        const uint32_t chunk = (t + 4 * j) ^ (CH >= 8 ? (g & 1u) * 4 : 0u);
        const uint4 x = reinterpret_cast<const uint4 *>(tile)[g * CH + chunk];
        const uint4 y = reinterpret_cast<const uint4 *>(tile)[(g + 8) * CH + chunk];
        const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t u = xw[c] ^ 0x80808080u, v = yw[c] ^ 0x80808080u;
          const uint32_t k[4] = {biased_f16(u, 0x4140), biased_f16(v, 0x4140), biased_f16(u, 0x4342), biased_f16(v, 0x4342)};
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int h = 0; h < H; ++h) mma_16x8x16(h == 0 ? s[n] : fine[n], k, qf[h][n][j * 4 + c]);
        }
      }
      if constexpr (H == 2) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[n][e] += fine[n][e];
      }
      const float ks = s_ks[i], vs = s_vs[i] * vlift, above = scale_above(s_vs[i], unit), limit = kRaise - above;
      bool raise = false;
      // (rows past the last are scored too, of queries of zeros; nothing of them is written)
      const bool part = s_page[i] < 0 || static_cast<int32_t>((seg + i) * 16 + 15) > whole;
      if (part) {
        const int32_t p0 = static_cast<int32_t>((seg + i) * 16 + g);
        const bool in = s_page[i] >= 0;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            bool seen = in && p0 + e / 2 * 8 <= last[n][e % 2];
            if constexpr (TREE) {
              const int32_t j = p0 + e / 2 * 8 - static_cast<int32_t>(len - a.tokens);  // (of rows past the last no more than zeros)
              if (in && j >= 0 && j < static_cast<int32_t>(a.tokens)) seen = (s_mask[n * 8 + 2 * t + e % 2][j / 32] >> (j % 32) & 1u) != 0u;
            }
            s[n][e] = seen ? s[n][e] * (ks * factor[n][e % 2]) : neg_inf();
            raise |= s[n][e] > m[n][e % 2] + limit;
          }
      } else {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[n][e] *= ks * factor[n][e % 2];
            raise |= s[n][e] > m[n][e % 2] + limit;
          }
      }
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float top = fmaxf(fmaxf(s[n][e], s[n][e + 2]) + above, m[n][e]);
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
            const float keep = m[n][e] == neg_inf() ? 0.0f : ex2(m[n][e] - top);
            m[n][e] = top;
            l[n][e] *= keep;
#pragma unroll
            for (int j = 0; j < MT; ++j) {
              o[n][j][e] *= keep;
              o[n][j][e + 2] *= keep;
            }
          }
      }
      uint32_t pf[HP][NB][2];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float base = m[n][e % 2] == neg_inf() ? 0.0f : m[n][e % 2];
          p[e] = ex2(s[n][e] - base);
          l[n][e % 2] += p[e];
          p[e] = part && s[n][e] == neg_inf() ? 0.0f : p[e] * vs;  // (no product with the scale of a page that a row does not see)
        }
#pragma unroll
        for (int h = 0; h < HP; ++h)
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            const __half2 x = __floats2half2_rn(p[2 * r], p[2 * r + 1]);
            pf[h][n][r] = transposed(*reinterpret_cast<const uint32_t *>(&x));
            p[2 * r] -= __low2float(x);
            p[2 * r + 1] -= __high2float(x);
          }
      }
      // ---- O^T: four dimensions of four positions to two 16 x 8 x 16 operands ----
      const unsigned char *vt = tile + 16 * DP;
      constexpr int VW = VB == 8 ? 2 : 4;  // words of a lane's access
#pragma unroll
      for (int j = 0; j < VB / (4 * VW); ++j) {
        uint32_t w[4][VW];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          if constexpr (VB == 8) {
            const uint2 x = *reinterpret_cast<const uint2 *>(vt + (2 * t + p % 2 + p / 2 * 8) * DP + ((g >> 1) ^ move(2 * t)) * 16 + (g & 1u) * 8);
            w[p][0] = x.x ^ 0x80808080u;
            w[p][1] = x.y ^ 0x80808080u;
          } else {
            const uint4 x = *reinterpret_cast<const uint4 *>(vt + (2 * t + p % 2 + p / 2 * 8) * DP + ((g * (VB / 16) + j) ^ move(2 * t)) * 16);
            w[p][0] = x.x ^ 0x80808080u;
            w[p][1] = x.y ^ 0x80808080u;
            w[p][2] = x.z ^ 0x80808080u;
            w[p][3] = x.w ^ 0x80808080u;
          }
        }
#pragma unroll
        for (int c = 0; c < VW; ++c) {
          const uint32_t x0 = __byte_perm(w[0][c], w[1][c], 0x5140), x1 = __byte_perm(w[0][c], w[1][c], 0x7362);
          const uint32_t y0 = __byte_perm(w[2][c], w[3][c], 0x5140), y1 = __byte_perm(w[2][c], w[3][c], 0x7362);
          const uint32_t v0[4] = {biased_f16(x0, 0x4140), biased_f16(x0, 0x4342), biased_f16(y0, 0x4140), biased_f16(y0, 0x4342)};
          const uint32_t v1[4] = {biased_f16(x1, 0x4140), biased_f16(x1, 0x4342), biased_f16(y1, 0x4140), biased_f16(y1, 0x4342)};
#pragma unroll
          for (int n = 0; n < NB; ++n) {
            if constexpr (H == 1) {
#pragma unroll
              for (int h = 0; h < HP; ++h) {
                mma_16x8x16(o[n][(j * VW + c) * 2], v0, pf[h][n]);
                mma_16x8x16(o[n][(j * VW + c) * 2 + 1], v1, pf[h][n]);
              }
            } else {
              float tile0[4] = {}, tile1[4] = {};
#pragma unroll
              for (int h = HP - 1; h >= 0; --h) {
                mma_16x8x16(tile0, v0, pf[h][n]);
                mma_16x8x16(tile1, v1, pf[h][n]);
              }
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                o[n][(j * VW + c) * 2][e] += tile0[e];
                o[n][(j * VW + c) * 2 + 1][e] += tile1[e];
              }
            }
          }
        }
      }
      issue(i + (F::DEPTH - 1) * kWarps, slot == 0 ? F::DEPTH - 1 : slot - 1);  // the slot read a round before
      if (++slot == F::DEPTH) slot = 0;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  }

  // ---- join the warps: [warp][row][dimension] and (m, l) in the ring ----
#pragma unroll
  for (int n = 0; n < NB; ++n)
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int off = 4; off <= 16; off <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], off);
  constexpr int PITCH = DP + 4;
  float *joined = reinterpret_cast<float *>(ring);
  float *stats = joined + kWarps * 8 * PITCH;  // [warp][8 rows][2]
  const float back = scalbnf(1.0f / kLift, unit);
  for (int n = 0; n < NB; ++n) {
    __syncthreads();
#pragma unroll
    for (int q = 0; q < NB; ++q) {
      if (q != n) continue;
#pragma unroll
      for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) joined[(warp * 8 + 2 * t + e % 2) * PITCH + VB * g + 2 * j + e / 2] = o[q][j][e];
      if (g == 0)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          stats[(warp * 8 + 2 * t + e) * 2] = m[q][e];
          stats[(warp * 8 + 2 * t + e) * 2 + 1] = l[q][e];
        }
    }
    __syncthreads();
    // warp w joins rows 2 w, 2 w + 1
    for (uint32_t r = warp * 2; r < warp * 2 + 2; ++r) {
      const uint32_t row = row0 + n * 8 + r;
      if (row >= rows) break;
      float top = neg_inf(), keep[kWarps], sum = 0.0f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) top = fmaxf(top, stats[(w * 8 + r) * 2]);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float mw = stats[(w * 8 + r) * 2];
        keep[w] = mw == neg_inf() ? 0.0f : ex2(mw - top);
        // (a warp that saw nothing but NaN has a NaN sum under m = -inf)
        sum += mw == neg_inf() ? stats[(w * 8 + r) * 2 + 1] : stats[(w * 8 + r) * 2 + 1] * keep[w];
      }
      const float scale = alone ? (sum == 0.0f ? 0.0f : 1.0f / sum) : 1.0f;
      const size_t at = (static_cast<size_t>(own_head) * f.splits + split) * rows + row;
      float *part = f.part + at * a.dim;
      T *out = static_cast<T *>(a.out) + static_cast<int64_t>(b) * a.out_strides[0] +
               static_cast<int64_t>(row / a.group) * a.out_strides[1] +
               static_cast<int64_t>(kh * a.group + row % a.group) * a.out_strides[2];
      for (uint32_t d = lane; d < a.dim; d += 32) {
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) v += keep[w] * joined[(w * 8 + r) * PITCH + d];
        if (alone)
          out[d] = from_float<T>(v * scale * back);  // (back is a power of two that may be tiny)
        else
          part[d] = v * back;
      }
      if (!alone && lane == 0) f.stats[at] = make_float2(sum, top);
    }
  }
}

constexpr int kJoinWarps = 8;

// Joins the splits of a row: WARPS warps a row (8: a block a row; 1: eight rows a block), a warp every WARPS-th split, a lane
// four dimensions (and 128 further on).
template <typename T, int WARPS>
__global__ void __launch_bounds__(32 * kJoinWarps) attend_join_kernel(const AttendArgs f, uint32_t group_rows) {
  __shared__ float s_o[kJoinWarps][256], s_m[kJoinWarps], s_l[kJoinWarps];
  const ClearAttentionArgs &a = f.a;
  const uint32_t warp = threadIdx.x / 32 % WARPS, lane = threadIdx.x % 32, rows = a.tokens * a.group;
  const uint32_t id = blockIdx.x * (kJoinWarps / WARPS) + threadIdx.x / (32 * WARPS);
  const bool real = id < f.count * rows;
  const uint32_t own_head = real ? id / rows : 0, bh = f.first + own_head, row = id % rows, kh = bh % a.heads, b = bh / a.heads;
  const int64_t most = static_cast<int64_t>(a.table_pitch) * a.page_tokens, given = a.lengths[b], len = given > most ? most : given;
  const uint32_t last_row = min(row / group_rows * group_rows + group_rows, rows) - 1;
  const uint32_t end = a.mask ? group_end<true>(a, len, last_row) : group_end<false>(a, len, last_row);
  const uint32_t share = split_share(f, end), count = (end + share - 1) / share;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (!real || end <= share) return;  // (whole rows; written already)
  const size_t at = static_cast<size_t>(own_head) * f.splits * rows + row;
  float top = neg_inf(), sum = 0.0f;
  float4 o[2] = {};
  for (uint32_t s0 = warp; s0 < count; s0 += 32 * WARPS) {  // lane i: split s0 + WARPS i
    const uint32_t mine = s0 + WARPS * lane, n = min(32u, (count - s0 + WARPS - 1) / WARPS);
    const float2 lm = mine < count ? f.stats[at + static_cast<size_t>(mine) * rows] : make_float2(0.0f, neg_inf());
    float t = fmaxf(top, lm.y);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, off));
    const float fade = top == neg_inf() ? 0.0f : ex2(top - t);
    const float keep = lm.y == neg_inf() ? 0.0f : ex2(lm.y - t);
    float add = lm.y == neg_inf() ? lm.x : lm.x * keep;  // (a NaN sum under m = -inf stays)
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) add += __shfl_xor_sync(0xffffffffu, add, off);
    sum = sum * fade + add;
    top = t;
#pragma unroll
    for (int i = 0; i < 2; ++i) o[i] = make_float4(o[i].x * fade, o[i].y * fade, o[i].z * fade, o[i].w * fade);
    const float *src = f.part + (at + static_cast<size_t>(s0) * rows) * a.dim + lane * 4;
    const size_t step = static_cast<size_t>(WARPS) * rows * a.dim;
#pragma unroll 4
    for (uint32_t j = 0; j < n; ++j, src += step) {
      const float k = __shfl_sync(0xffffffffu, keep, j);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (lane * 4 + 128 * i < a.dim) {
          const float4 v = *reinterpret_cast<const float4 *>(src + 128 * i);
          o[i] = make_float4(o[i].x + k * v.x, o[i].y + k * v.y, o[i].z + k * v.z, o[i].w + k * v.w);
        }
    }
  }
  T *out = static_cast<T *>(a.out) + static_cast<int64_t>(b) * a.out_strides[0] + static_cast<int64_t>(row / a.group) * a.out_strides[1] +
           static_cast<int64_t>(kh * a.group + row % a.group) * a.out_strides[2];
  if constexpr (WARPS == 1) {
    const float scale = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint32_t d = lane * 4 + 128 * i;
      if (d >= a.dim) continue;
      out[d] = from_float<T>(o[i].x * scale);
      out[d + 1] = from_float<T>(o[i].y * scale);
      out[d + 2] = from_float<T>(o[i].z * scale);
      out[d + 3] = from_float<T>(o[i].w * scale);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) *reinterpret_cast<float4 *>(&s_o[warp][lane * 4 + 128 * i]) = o[i];
    if (lane == 0) {
      s_m[warp] = top;
      s_l[warp] = sum;
    }
    __syncthreads();
    top = neg_inf();
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) top = fmaxf(top, s_m[w]);
    sum = 0.0f;
    float v = 0.0f;
    const uint32_t d = threadIdx.x;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) {
      const float keep = s_m[w] == neg_inf() ? 0.0f : ex2(s_m[w] - top);
      sum += s_m[w] == neg_inf() ? s_l[w] : s_l[w] * keep;
      v += keep * s_o[w][d];
    }
    if (d < a.dim) out[d] = from_float<T>(sum == 0.0f ? 0.0f : v / sum);
  }
}

// Splits of a sequence.  Ranges of 1024 positions, or 512 or 256 where those leave SMs without a block; no more of them
// than fill the SMs four times over (uneven lengths then even out).  Longer ranges cost less to begin and to join
// (8 sequences of 4096, 8 heads: 1024 positions a tenth less than 512), shorter ones balance better.
void split(AttendArgs *f, uint32_t sms) {
  const ClearAttentionArgs &a = f->a;
  const uint64_t blocks = static_cast<uint64_t>(a.batch) * a.heads * f->groups, most = static_cast<uint64_t>(a.table_pitch) * a.page_tokens;
  f->least = 1024;
  while (f->least > 256 && blocks * ((most + f->least - 1) / f->least) < 2 * sms) f->least /= 2;
  const uint64_t longest = (most + f->least - 1) / f->least, want = (16ull * sms + blocks - 1) / blocks;
  f->splits = static_cast<uint32_t>(want < longest ? want : longest);
  if (f->splits < 1) f->splits = 1;
  if (f->splits > 1024) f->splits = 1024;
  const uint64_t least = (most + kWarps * kMostPositions - 1) / (kWarps * kMostPositions);  // (a warp takes a quarter)
  if (f->splits < least) f->splits = static_cast<uint32_t>(least);
}

uint32_t group_rows_of(const ClearAttentionArgs &a) { return a.tokens * a.group <= 8 ? 8 : 16; }

template <typename T, int DP, int NB, bool TREE>
cudaError_t launch(const AttendArgs &f, cudaStream_t s) {
  auto kern = attend_few_kernel<T, DP, NB, TREE>;
  constexpr uint32_t join = (kWarps * 8 * (DP + 4) + kWarps * 8 * 2) * 4;
  constexpr uint32_t smem = Few<DP>::RING > join ? Few<DP>::RING : join;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
  if (e != cudaSuccess) return e;
  kern<<<f.count * f.groups * f.splits, 32 * kWarps, smem, s>>>(f);
  return cudaGetLastError();
}

template <typename T, int DP>
cudaError_t launch(const AttendArgs &f, cudaStream_t s) {
  if (f.a.mask) return group_rows_of(f.a) == 8 ? launch<T, DP, 1, true>(f, s) : launch<T, DP, 2, true>(f, s);
  return group_rows_of(f.a) == 8 ? launch<T, DP, 1, false>(f, s) : launch<T, DP, 2, false>(f, s);
}

template <typename T>
cudaError_t launch(const AttendArgs &f, cudaStream_t s) {
  if (f.a.dim <= 64) return launch<T, 64>(f, s);
  if (f.a.dim <= 128) return launch<T, 128>(f, s);
  return launch<T, 256>(f, s);
}

}  // namespace

bool attend_few_takes(const ClearAttentionArgs &a) {
  return a.dim % 16 == 0 && a.page_tokens % 16 == 0 && a.cache_strides[2] < (1 << 26) &&
         (reinterpret_cast<uintptr_t>(a.k_cache) | reinterpret_cast<uintptr_t>(a.v_cache) |
          static_cast<uintptr_t>(a.cache_strides[0] | a.cache_strides[1] | a.cache_strides[2])) % 16 == 0;
}

namespace {

AttendArgs few_args(const ClearAttentionArgs &a, void *work, uint32_t sms) {
  AttendArgs f{a, nullptr, nullptr, 0, 0, 1, 1, 1, false, false};
  const uint32_t rows = a.tokens * a.group, gr = group_rows_of(a);
  f.groups = (rows + gr - 1) / gr;
  split(&f, sms);
  attend_place(&f, work);
  return f;
}

template <typename T>
cudaError_t launch_join(const AttendArgs &f, uint32_t group_rows, cudaStream_t s) {
  const uint64_t rows = static_cast<uint64_t>(f.count) * f.a.tokens * f.a.group;
  const bool many = f.splits > 8;  // a warp reads eight partial rows as fast as eight warps would start
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<uint32_t>(many ? rows : (rows + kJoinWarps - 1) / kJoinWarps));
  cfg.blockDim = dim3(32 * kJoinWarps);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return many ? cudaLaunchKernelEx(&cfg, attend_join_kernel<T, kJoinWarps>, f, group_rows)
              : cudaLaunchKernelEx(&cfg, attend_join_kernel<T, 1>, f, group_rows);
}

}  // namespace

cudaError_t launch_attend_join(const AttendArgs &f, int type, uint32_t group_rows, cudaStream_t s) {
  if (type == kOutF32) return launch_join<float>(f, group_rows, s);
  if (type == kOutF16) return launch_join<__half>(f, group_rows, s);
  return launch_join<__nv_bfloat16>(f, group_rows, s);
}

size_t attend_few_bytes(const ClearAttentionArgs &a, uint32_t sms) { return attend_part_bytes(few_args(a, nullptr, sms)); }

cudaError_t launch_clear_attention_few(const ClearAttentionArgs &a, int type, void *work, uint32_t sms, cudaStream_t s) {
  return attend_each(few_args(a, work, sms), [&](const AttendArgs &f) {
    const cudaError_t e = type == kOutF32 ? launch<float>(f, s) : type == kOutF16 ? launch<__half>(f, s) : launch<__nv_bfloat16>(f, s);
    return e != cudaSuccess || f.splits == 1 ? e : launch_attend_join(f, type, group_rows_of(a), s);
  });
}

}  // namespace rosetta
