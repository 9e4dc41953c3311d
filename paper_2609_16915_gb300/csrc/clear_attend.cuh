// What both attention kernels share: the ranges that a sequence's positions are split into, and the join of their
// partial results.
#pragma once
#include <stdint.h>

#include "clear.h"

namespace rosetta {

struct AttendArgs {
  ClearAttentionArgs a;
  float *part;              // [batch, head of this launch][split][rows of all groups]: O [dim]
  float2 *stats;            // the same: l, m
  uint32_t first, count;    // cached heads, of all sequences, that this launch takes
  uint32_t splits, groups;  // ranges of a sequence's positions at most, row groups of a cached head
  uint32_t least;           // positions of a range at least
  bool by_length;           // blocks of the longest sequences first
  bool runs;                // a range may be longer than one accumulator takes: it adds up in the place of its partial result
};

// The tensor cores cut the terms of their sums off instead of rounding them: an output comes out up to 7e-9 of itself short for
// every position that one accumulator has taken (values of one sign; 1e-9 otherwise).  So no accumulator takes more
// positions than this (2^-12, half a unit of float16's rounding), and single
// precision adds its accumulators up much sooner (its running sums of longer ranges round off more than 2^-18).
constexpr uint32_t kMostPositions = 1u << 15;

// Value scales as exponents of two.  Weights for the product with V are 2^(s - m) vs / sv with the running maximum m of
// s + log2(vs / sv), so that each row's largest term is near the largest f16 whatever other pages' scales are.  sv = 2^unit keeps
// the sums of weights in range: 1 for scales within 2^20 of 1 (a row's words then do not depend on pages that it does not
// see), or near the largest one.
constexpr int32_t kNoScale = -1000;
constexpr float kLeastAbove = -80.0f;  // scales further below sv are taken as if this far: 2^-100 of sv still keeps ten bits

// floor(log2 |v|); less than every number's for 0, NaN and infinity
__device__ __forceinline__ int32_t scale_exponent(float v) {
  const int32_t e = static_cast<int32_t>(__float_as_uint(v) >> 23 & 255u);
  return v == 0.0f || e == 255 ? kNoScale : e - 127;
}

__device__ __forceinline__ int32_t scale_unit(int32_t most) {
  return most == kNoScale || (most >= -20 && most <= 20) ? 0 : max(most, -100);
}

// What a page's scale adds to its scores in the running maximum: at least log2 |v / sv|, less than 1 more.
__device__ __forceinline__ float scale_above(float v, int32_t unit) {
  const float up = static_cast<float>(static_cast<int32_t>(__float_as_uint(v) >> 23 & 255u) - 126 - unit);
  return fminf(fmaxf(up, kLeastAbove), 24.0f);  // (24: no number)
}

// Positions of each range of a sequence of `end`: whole tiles of all warps.
__device__ __forceinline__ uint32_t split_share(const AttendArgs &f, uint32_t end) {
  const uint32_t share = (end + f.splits - 1) / f.splits;
  return ((share < f.least ? f.least : share) + 63) / 64 * 64;
}

// Positions that the rows of a group see at most: up to the last token of the group; under a mask (TREE) all of them.
template <bool TREE>
__device__ __forceinline__ uint32_t group_end(const ClearAttentionArgs &a, int64_t len, uint32_t last_row) {
  const int64_t end = TREE ? len : len - a.tokens + 1 + last_row / a.group;
  return end > 0 ? static_cast<uint32_t>(end) : 0u;
}

// Word `i` of a mask row, its bits from a position of the drafted ones on: before them (i < 0) all are seen, behind them none.
__device__ __forceinline__ uint32_t mask_word(const uint32_t *row, uint32_t tokens, int32_t i) {
  if (i < 0) return ~0u;
  const uint32_t from = static_cast<uint32_t>(i) * 32;
  if (from >= tokens) return 0u;
  return tokens - from < 32 ? row[i] & ((1u << (tokens - from)) - 1u) : row[i];
}

// Join the splits of every row; group_rows: rows that one block's ranges were laid out for.
cudaError_t launch_attend_join(const AttendArgs &f, int type, uint32_t group_rows, cudaStream_t s);

// Partial results take kMostPart bytes at most, or what one cached head of one sequence needs: beyond that the heads go
// in several launches (each many times what fills the GPU).
constexpr size_t kMostPart = size_t{256} << 20;

inline size_t attend_part_rows(const AttendArgs &f) { return static_cast<size_t>(f.splits) * f.a.tokens * f.a.group; }  // of a head
inline uint32_t attend_heads_at_once(const AttendArgs &f) {
  const size_t heads = static_cast<size_t>(f.a.batch) * f.a.heads, each = attend_part_rows(f) * (f.a.dim + 2) * sizeof(float);
  if ((f.splits == 1 && !f.runs) || heads * each <= kMostPart) return static_cast<uint32_t>(heads);
  const size_t most = each < kMostPart ? kMostPart / each : 1, launches = (heads + most - 1) / most;
  return static_cast<uint32_t>((heads + launches - 1) / launches);  // (about as many each time)
}
// Bytes of the partial results, and their place in the workspace (rows of 16 floats at least: the statistics behind
// them are aligned).
inline size_t attend_part_bytes(const AttendArgs &f) {
  return f.splits == 1 && !f.runs ? 0 : attend_heads_at_once(f) * attend_part_rows(f) * (f.a.dim + 2) * sizeof(float);
}
inline void attend_place(AttendArgs *f, void *work) {
  f->first = 0;
  f->count = attend_heads_at_once(*f);
  f->part = static_cast<float *>(work);
  f->stats = reinterpret_cast<float2 *>(f->part + f->count * attend_part_rows(*f) * f->a.dim);
}
// launch(f) for all heads, the last time with fewer.
template <typename F>
cudaError_t attend_each(AttendArgs f, F launch) {
  const uint32_t heads = f.a.batch * f.a.heads;
  for (; f.first < heads; f.first += f.count) {
    if (f.count > heads - f.first) f.count = heads - f.first;
    const cudaError_t e = launch(f);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace rosetta
