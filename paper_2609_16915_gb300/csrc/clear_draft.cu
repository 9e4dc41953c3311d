// A tree of drafted tokens: its mask, and its verification against the target's probabilities.
//
// Mask: bit j of row t says whether node j is t or an ancestor of it.  A thread takes a word of a row and walks from the
// node towards its root (parents come before their children, so the walk ends, and ends early for a word of later nodes).
//
// Verification.  From the root, node after node, the children of the accepted node n are tried in order.  With target
// row p and draft row q of n, which they were drawn from (one by one, with replacement),
//   s = 0, Z = 1;  child of token x, number u:  accepted where u q(x) Z < max(p(x) - s q(x), 0),
//   else  s' = s + Z,  Z' = sum_y max(p(y) - s' q(y), 0)
// (what is left of p after a rejection, max(w - Z q, 0), is max(p - s' q, 0): one number instead of a row).  Without
// draft rows a child is given, not drawn: accepted where u R < p(x), else its p(x) leaves R, which begins at 1.  The first
// token whose running sum of what is left passes u_0 of all of it is next.
//
// All sums are of whole multiples of 2^-56, so no order changes them, and they are compared as integers.  (64 bits all the way: the next
// token is where a running sum over the vocabulary passes a number, and sums in single precision would now and then pass it at
// another token.)
// What is read: p(x) and q(x) of every node at once, and whole rows only where a sum is wanted: of nodes whose children were rejected
// and of the last one, of that a warp's run again.  Bound by the chain of these steps (nodes, their probabilities, a row at a time, each with a
// meeting of the cluster) and by 13 instructions a pair of probabilities: a sequence of 5 nodes over 50257 tokens 8 us; 64 of 64
// nodes over 128256 with draft rows 54 us, of which one target row of each takes 17.
#include <stdint.h>

#include "clear.h"
#include "dsmem.cuh"
#include "pairs.cuh"

namespace rosetta {

namespace {

constexpr uint64_t kOne = 1ull << 56, kMost = 1ull << 62;  // sums stay at kMost: no probabilities
constexpr uint32_t kMostThreads = 512, kMostWarps = kMostThreads / 32;

__global__ void __launch_bounds__(256) tree_mask_kernel(const ClearTreeArgs a) {
  extern __shared__ int32_t up[];
  const uint32_t b = blockIdx.y, words = (a.tokens + 31) / 32;
  const int32_t *parents = a.parents + static_cast<int64_t>(b) * a.parents_pitch;
  for (uint32_t i = threadIdx.x; i < a.tokens; i += blockDim.x) {
    int32_t p = parents[i];
    if (p < -1 || p >= static_cast<int32_t>(i)) {
      atomicMax(a.err_flag, 1u);
      p = -1;
    }
    up[i] = p;
  }
  __syncthreads();
  const uint32_t id = blockIdx.x * blockDim.x + threadIdx.x;
  if (id >= a.tokens * words) return;
  const int32_t t = static_cast<int32_t>(id / words), w = static_cast<int32_t>(id % words);
  uint32_t bits = 0;
  for (int32_t j = t; j >= w * 32; j = up[j])
    if (j / 32 == w) bits |= 1u << (j % 32);
  a.mask[static_cast<int64_t>(b) * a.mask_strides[0] + t * a.mask_strides[1] + w] = bits;
}

__device__ __forceinline__ uint64_t add_most(uint64_t a, uint64_t b) {  // both kMost at most
  const uint64_t s = a + b;
  return s < kMost ? s : kMost;
}

// a b of two fixed-point numbers, rounded down (2^57 and 2^62 at most)
__device__ __forceinline__ uint64_t times(uint64_t a, uint64_t b) { return __umul64hi(a, b) << 8 | (a * b) >> 56; }

__device__ __forceinline__ uint64_t less(uint64_t a, uint64_t b) { return a > b ? a - b : 0; }

// A probability p in [0, 2] as whole multiples of 2^-56, from additions that round to a grid each: p + 4 in the last bits of its word has
// p to 2^-21, what is left over (exact) plus 1.5 x 2^-21 has it to 2^-44, and what is left of that plus 1.5 x 2^-33 to 2^-56.  (Converting
// to 64-bit integers instead: 33 MB of rows 35 us.)
constexpr float kGrid1 = 4.0f, kGrid2 = 1.5f / 2097152.0f, kGrid3 = 1.5f / 8589934592.0f;
__device__ __forceinline__ uint64_t joined(uint32_t s1, uint32_t s2, uint32_t s3) {  // of sums of the words' differences to the grids'
  return (static_cast<uint64_t>(s1) << 35) + static_cast<uint64_t>(static_cast<int64_t>(static_cast<int32_t>(s2)) << 12) +
         static_cast<uint64_t>(static_cast<int64_t>(static_cast<int32_t>(s3)));
}
__device__ __forceinline__ uint64_t fixed(float p, bool &bad) {  // what is no probability counts as zero
  const bool in = p >= 0.0f && p <= 2.0f;  // (rounded sums may pass 1)
  bad |= !in;
  if (!in) p = 0.0f;
  const float t1 = __fadd_rn(p, kGrid1), r = __fsub_rn(p, __fsub_rn(t1, kGrid1)), t2 = __fadd_rn(r, kGrid2);
  const float t3 = __fadd_rn(__fsub_rn(r, __fsub_rn(t2, kGrid2)), kGrid3);
  return joined(__float_as_uint(t1) - __float_as_uint(kGrid1), __float_as_uint(t2) - __float_as_uint(kGrid2),
                __float_as_uint(t3) - __float_as_uint(kGrid3));
}

// the words of two probabilities on the three grids
struct Words {
  float2 t1, t2, t3;
};
__device__ __forceinline__ Words words_of(float x, float y) {
  const uint64_t p = pair_of(x, y), minus = pair_of(-1.0f, -1.0f), g1 = pair_of(kGrid1, kGrid1), g2 = pair_of(kGrid2, kGrid2), g3 = pair_of(kGrid3, kGrid3);
  const uint64_t t1 = add2(p, g1), r = add2(p, fma2(t1, minus, g1)), t2 = add2(r, g2), t3 = add2(add2(r, fma2(t2, minus, g2)), g3);
  return {floats_of(t1), floats_of(t2), floats_of(t3)};
}

// a number in [0, 1) in units of 2^-64
__device__ __forceinline__ uint64_t fraction(float u) {
  if (!(u > 0.0f)) return 0;
  return u >= 1.0f ? ~0ull : __float2ull_rz(u * 18446744073709551616.0f);
}

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Pack {
  T v[VEC];
};

// A cluster of CTAs for each sequence; a warp takes a run of the vocabulary.
template <typename T, bool DRAFT>
__global__ void __launch_bounds__(kMostThreads, 2) verify_kernel(const ClearVerifyArgs a, uint32_t ranks, uint32_t run) {
  constexpr int VEC = 4;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ uint64_t s_warp[2][kMostWarps], s_total[2];
  __shared__ uint32_t s_bad;
  const uint32_t nodes = a.nodes, tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
  const uint32_t threads = blockDim.x, warps = threads / 32;
  const uint32_t rank = blockIdx.x % ranks, b = blockIdx.x / ranks;
  // of each node: p and q of its token under its parent, its number, parent, token; the tokens rejected at the present
  // node and their p (DRAFT has none)
  uint64_t *s_p = reinterpret_cast<uint64_t *>(smem), *s_u = s_p + nodes, *s_q = s_u + nodes, *s_gone_p = s_q;
  int32_t *s_up = reinterpret_cast<int32_t *>(s_q + nodes), *s_token = s_up + nodes, *s_path = s_token + nodes;
  int32_t *s_gone = s_path + nodes;
  const T *target = static_cast<const T *>(a.target) + static_cast<int64_t>(b) * a.target_strides[0];
  const T *draft = DRAFT ? static_cast<const T *>(a.draft) + static_cast<int64_t>(b) * a.draft_strides[0] : nullptr;
  const float *uniform = a.uniform + static_cast<int64_t>(b) * a.uniform_pitch;
  bool bad = false;
  // Each CTA gathers every ranks-th node and all take it over, so that they decide alike whatever becomes of the buffers meanwhile.
  for (uint32_t c = rank + tid * ranks; c < nodes; c += threads * ranks) {
    int32_t up = c ? a.parents[static_cast<int64_t>(b) * a.parents_pitch + c] : -1;
    const int32_t x = a.tokens[static_cast<int64_t>(b) * a.tokens_pitch + c];
    if (up < -1 || up >= static_cast<int32_t>(c) || (up >= 0 && (x < 0 || static_cast<uint32_t>(x) >= a.vocab))) {
      bad = true;
      up = -1;
    }
    s_up[c] = up;
    s_token[c] = x;
    s_u[c] = fraction(uniform[c]);
    s_p[c] = up >= 0 ? fixed(to_float(target[static_cast<int64_t>(up) * a.target_strides[1] + x]), bad) : 0;
    if constexpr (DRAFT) s_q[c] = up >= 0 ? fixed(to_float(draft[static_cast<int64_t>(up) * a.draft_strides[1] + x]), bad) : 0;
  }
  __syncwarp();  // (here and below: the cluster's barrier wants whole warps)
  if (ranks > 1) {
    cluster_sync_shared();
    for (uint32_t c = tid; c < nodes; c += threads) {
      const uint32_t from = c % ranks;
      if (from == rank) continue;
      const uint32_t up = dsmem_ld_u32(dsmem_map(smem_addr(s_up + c), from)), x = dsmem_ld_u32(dsmem_map(smem_addr(s_token + c), from));
      const uint64_t u = dsmem_ld_u64(dsmem_map(smem_addr(s_u + c), from)), p = dsmem_ld_u64(dsmem_map(smem_addr(s_p + c), from));
      const uint64_t q = DRAFT ? dsmem_ld_u64(dsmem_map(smem_addr(s_q + c), from)) : 0;
      s_up[c] = static_cast<int32_t>(up);
      s_token[c] = static_cast<int32_t>(x);
      s_u[c] = u;
      s_p[c] = p;
      if constexpr (DRAFT) s_q[c] = q;
    }
  }
  __syncthreads();
  if (static_cast<uint32_t>(s_token[0]) >= a.vocab) {  // the root is no token: nothing stands behind it (the same for the cluster)
    if (rank == 0) {
      for (uint32_t i = tid; i < nodes; i += threads) a.path[static_cast<int64_t>(b) * a.path_pitch + i] = -1;
      if (tid == 0) {
        a.count[b] = 0;
        a.next[b] = -1;
        atomicMax(a.err_flag, 1u);
      }
    }
    __syncwarp();
    if (ranks > 1) cluster_sync_shared();  // (the nodes are read until here)
    return;
  }

  const uint32_t lo = (rank * warps + warp) * run, hi = min(a.vocab, lo + run);  // this warp's run
  const auto row_of = [&](const T *rows, const int64_t (&strides)[2], uint32_t n) { return rows + static_cast<int64_t>(n) * strides[1]; };
  // s q in two floats, the second to 2^-48 of it, for s other than 0 and 1; what is left of p (whole multiples of 2^-56 again, none of them
  // below zero) counts from kLeast on
  float high = 0.0f, low = 0.0f;
  const auto take = [&](uint64_t s) {
    high = __ull2float_rn(s) * 0x1p-56f;
    low = __ll2float_rn(static_cast<int64_t>(s - __float2ull_rn(high * 0x1p56f))) * 0x1p-56f;
  };
  constexpr float kLeast = 0x1p-55f;
  // what is left of a token
  const auto one = [&](const T *p, const T *q, uint32_t x, uint64_t s) {
    const uint64_t w = fixed(to_float(p[x]), bad);
    if (!DRAFT || s == 0) return w;
    const uint64_t v = fixed(to_float(q[x]), bad);
    if (s == kOne) return less(w, v);
    const float px = to_float(p[x]), given = to_float(q[x]), qx = given >= 0.0f && given <= 2.0f ? given : 0.0f, h = __fmul_rn(qx, high), l = __fmaf_rn(qx, low, __fmaf_rn(qx, high, -h));
    if (w == 0 || !(__fsub_rn(px, h) > __fadd_rn(l, kLeast))) return uint64_t{0};
    const float t2 = __fadd_rn(l, kGrid2), t3 = __fadd_rn(__fsub_rn(l, __fsub_rn(t2, kGrid2)), kGrid3);
    return w - fixed(h, bad) - joined(0, __float_as_uint(t2) - __float_as_uint(kGrid2), __float_as_uint(t3) - __float_as_uint(kGrid3));
  };
  // what is left of this thread's share of the warp's run.  Rows that lie alike to 16 bytes are read in such pieces, but for their ends.
  const auto own_sum = [&](const T *p, const T *q, uint64_t s) {
    uint64_t sum = 0;
    const auto away = [](const T *row, uint32_t x) { return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(row + x) / sizeof(T) % VEC); };
    const bool both = DRAFT && s != 0;
    uint32_t x = min(lo, hi), end = x;
    if (!both || away(p, 0) == away(q, 0)) {
      x = min(hi, x + (VEC - away(p, x)) % VEC);  // the first piece
      end = x + (hi - x) / VEC * VEC;
      const uint32_t edge = lo < hi ? x - lo + (hi - end) : 0;  // tokens outside the pieces: fewer than 2 VEC
      if (lane < edge) sum = one(p, q, lane < x - lo ? lo + lane : end + lane - (x - lo), s);
      const uint64_t begun = sum;
      const uint64_t s_high = pair_of(high, high), s_low = pair_of(low, low);
      uint32_t largest = 0;  // of the numbers' bits: past 2.0's where one is none
      // Two pieces of each row are asked for at once; what lies behind the end counts as zeros.  Of the row itself, or after one
      // rejection (s = 1, max(p - q, 0)), the words' sums: 64 tokens at a time fit them, 2^63 of them together.  (Longer pieces and
      // more of them, unrolled, are slower: the code of a kernel that runs through once comes from far away.)
      for (uint32_t at = x + lane * VEC; at < end;) {
        uint32_t s1 = 0, s2 = 0, s3 = 0;
        uint64_t part = 0;
#pragma unroll 1
        for (uint32_t turn = 0; turn < 64 / VEC / 2 && at < end; ++turn, at += 2 * 32 * VEC) {
          Pack<T, VEC> pv[2], qv[2];
#pragma unroll
          for (uint32_t i = 0; i < 2; ++i) {
            const uint32_t own = at + i * 32 * VEC;
#pragma unroll
            for (int e = 0; e < VEC; ++e) pv[i].v[e] = qv[i].v[e] = from_float<T>(0.0f);
            if (own < end) {
              pv[i] = *reinterpret_cast<const Pack<T, VEC> *>(p + own);
              if (both) qv[i] = *reinterpret_cast<const Pack<T, VEC> *>(q + own);
            }
          }
          if (both && s != kOne) {
#pragma unroll
            for (uint32_t i = 0; i < 2; ++i)
#pragma unroll
              for (int e = 0; e < VEC; e += 2) {
                const float px = to_float(pv[i].v[e]), py = to_float(pv[i].v[e + 1]), qx = to_float(qv[i].v[e]), qy = to_float(qv[i].v[e + 1]);
                largest = max(max(largest, max(__float_as_uint(px), __float_as_uint(py))), max(__float_as_uint(qx), __float_as_uint(qy)));
                const uint64_t q2 = pair_of(qx, qy), h2 = mul2(q2, s_high), minus = pair_of(-1.0f, -1.0f);
                const uint64_t l2 = fma2(q2, s_low, fma2(q2, s_high, mul2(h2, minus)));
                const float2 h = floats_of(h2), limit = floats_of(add2(l2, pair_of(kLeast, kLeast))), off = floats_of(add2(pair_of(px, py), mul2(h2, minus)));
                const Words w = words_of(px, py), v = words_of(h.x, h.y);
                const uint64_t g2 = pair_of(kGrid2, kGrid2), g3 = pair_of(kGrid3, kGrid3), u2 = add2(l2, g2);
                const float2 t2 = floats_of(u2), t3 = floats_of(add2(add2(l2, fma2(u2, minus, g2)), g3));
                if (off.x > limit.x) {
                  s1 += __float_as_uint(w.t1.x) - __float_as_uint(v.t1.x);
                  s2 += __float_as_uint(w.t2.x) - __float_as_uint(v.t2.x) - (__float_as_uint(t2.x) - __float_as_uint(kGrid2));
                  s3 += __float_as_uint(w.t3.x) - __float_as_uint(v.t3.x) - (__float_as_uint(t3.x) - __float_as_uint(kGrid3));
                }
                if (off.y > limit.y) {
                  s1 += __float_as_uint(w.t1.y) - __float_as_uint(v.t1.y);
                  s2 += __float_as_uint(w.t2.y) - __float_as_uint(v.t2.y) - (__float_as_uint(t2.y) - __float_as_uint(kGrid2));
                  s3 += __float_as_uint(w.t3.y) - __float_as_uint(v.t3.y) - (__float_as_uint(t3.y) - __float_as_uint(kGrid3));
                }
              }
            continue;
          }
#pragma unroll
          for (uint32_t i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < VEC; e += 2) {
              // (of the row itself q is zeros: its words are the grids' own)
              const float px = to_float(pv[i].v[e]), py = to_float(pv[i].v[e + 1]), qx = to_float(qv[i].v[e]), qy = to_float(qv[i].v[e + 1]);
              const Words w = words_of(px, py), v = words_of(qx, qy);
              largest = max(max(largest, max(__float_as_uint(px), __float_as_uint(py))), max(__float_as_uint(qx), __float_as_uint(qy)));
              if (px > qx) {
                s1 += __float_as_uint(w.t1.x) - __float_as_uint(v.t1.x);
                s2 += __float_as_uint(w.t2.x) - __float_as_uint(v.t2.x);
                s3 += __float_as_uint(w.t3.x) - __float_as_uint(v.t3.x);
              }
              if (py > qy) {
                s1 += __float_as_uint(w.t1.y) - __float_as_uint(v.t1.y);
                s2 += __float_as_uint(w.t2.y) - __float_as_uint(v.t2.y);
                s3 += __float_as_uint(w.t3.y) - __float_as_uint(v.t3.y);
              }
            }
        }
        part += joined(s1, s2, s3);
        sum = add_most(sum, part < kMost ? part : kMost);
      }
      if (largest > 0x40000000u) {  // one by one
        sum = begun;
#pragma unroll 1
        for (uint32_t at = x + lane * VEC; at < end; at += 32 * VEC)
#pragma unroll 1
          for (int e = 0; e < VEC; ++e) sum = add_most(sum, one(p, q, at + e, s));
      }
      return sum;
    }
    if constexpr (DRAFT) {
#pragma unroll 2
      for (x += lane; x < hi; x += 32) sum = add_most(sum, one(p, q, x, s));
    }
    return sum;
  };
  uint32_t turn = 0;
  uint64_t before = 0;  // the sum of the CTAs before this one
  // the sum of what is left of node n's row, over the cluster; the warps' sums stay in s_warp[turn ^ 1]
  const auto row_sum = [&](uint32_t n, uint64_t s, uint32_t gone) {
    const T *p = row_of(target, a.target_strides, n), *q = DRAFT ? row_of(draft, a.draft_strides, n) : nullptr;
    if constexpr (DRAFT) take(s);
    uint64_t sum = own_sum(p, q, s);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum = add_most(sum, __shfl_xor_sync(0xffffffffu, sum, o));
    if (lane == 0) s_warp[turn][warp] = sum;
    __syncthreads();
    if (!DRAFT && gone) {
      for (uint32_t i = tid; i < gone; i += threads) {
        const uint32_t w = static_cast<uint32_t>(s_gone[i]) / run;
        // (a sum that stopped at kMost is none to take from; the others are below it from beginning to end)
        if (w / warps == rank && *const_cast<volatile uint64_t *>(&s_warp[turn][w % warps]) < kMost)
          atomicAdd(reinterpret_cast<unsigned long long *>(&s_warp[turn][w % warps]), 0ull - s_gone_p[i]);
      }
      __syncthreads();
    }
    uint64_t total = 0;
    for (uint32_t w = 0; w < warps; ++w) total = add_most(total, s_warp[turn][w]);
    before = 0;
    if (ranks > 1) {
      if (tid == 0) s_total[turn] = total;
      __syncwarp();
      cluster_sync_shared();
      const uint32_t at = smem_addr(&s_total[turn]);
      const uint64_t of = lane < ranks ? dsmem_ld_u64(dsmem_map(at, lane)) : 0;
      total = 0;
      for (uint32_t r = 0; r < ranks; ++r) {
        if (r == rank) before = total;
        total = add_most(total, __shfl_sync(0xffffffffu, of, r));
      }
    }
    turn ^= 1;
    return total;
  };

  // ---- the walk: every warp for itself, all alike; it stops where a sum is wanted, and at its end ----
  uint32_t n = 0, length = 1, gone = 0, c0 = 1;
  uint64_t s = 0, z = kOne, left = kOne, off = 0, total;  // (off: of the rejected tokens that were given, which left may not hold in full)
  bool stale = false, ended = false;  // (stale: z is that of the s before)
  if (tid == 0) s_path[0] = 0;
  while (true) {
    while (!ended) {
      uint32_t hit = 0;
      for (; c0 < nodes; c0 += 32) {
        hit = __ballot_sync(0xffffffffu, c0 + lane < nodes && s_up[min(c0 + lane, nodes - 1)] == static_cast<int32_t>(n));
        if (hit) break;
      }
      ended = hit == 0;
      if (ended) break;
      const uint32_t c = c0 + __ffs(hit) - 1;
      const uint64_t u = s_u[c];
      bool yes;
      if constexpr (DRAFT) {
        // (Z only falls, but for rows that add up to a little more than 1: what the one before would accept needs no sum)
        yes = __umul64hi(u, times(s_q[c], stale ? z + (z >> 6) : z)) < less(s_p[c], times(s_q[c], s));
        if (!yes && stale) break;
        if (!yes) {
          s = add_most(s, z);
          stale = true;
        }
      } else {
        uint64_t p = s_p[c];
        bool again = false;  // a token that has been rejected here
        for (uint32_t i = lane; i < gone; i += 32) again |= s_gone[i] == s_token[c];
        if (__any_sync(0xffffffffu, again)) p = 0;
        yes = __umul64hi(u, left) < p;
        if (!yes && p) {
          left = less(left, p);
          off = add_most(off, p);
          __syncthreads();  // (all have looked at the list)
          if (tid == 0) {
            s_gone[gone] = s_token[c];
            s_gone_p[gone] = p;
          }
          ++gone;
          __syncthreads();
        }
      }
      c0 = c + 1;
      if (yes) {
        if (tid == 0) s_path[length] = static_cast<int32_t>(c);
        ++length;
        n = c;
        s = 0;
        z = left = kOne;
        off = 0;
        gone = 0;
        stale = false;
      }
    }
    total = row_sum(n, s, gone);
    // given: it is the row that adds up to too much or does not, the rejected tokens in it (so that the runs' sizes do not matter)
    if (!DRAFT && add_most(total, off) == kMost) total = kMost;
    if (!ended) {
      z = total;
      stale = false;
    } else if (total == 0 && (s != 0 || gone != 0)) {  // nothing is left: the target's row itself
      s = off = 0;
      gone = 0;
    } else {
      break;
    }
  }

  // ---- the next token ----
  if (tid == 0) s_bad = 0;
  __syncthreads();
  if (bad) s_bad = 1;
  __syncthreads();
  if (tid == 0 && (s_bad || total == 0 || total >= kMost)) atomicMax(a.err_flag, 1u);
  if (rank == 0) {
    for (uint32_t i = tid; i < nodes; i += threads) a.path[static_cast<int64_t>(b) * a.path_pitch + i] = i < length ? s_path[i] : -1;
    if (tid == 0) {
      a.count[b] = static_cast<int32_t>(length);
      if (total == 0 || total >= kMost) a.next[b] = -1;
    }
  }
  const uint64_t goal = __umul64hi(s_u[0], total);  // the first running sum above it
  const uint32_t last = turn ^ 1;
  uint32_t owner = 0;  // the warp in whose run it passes
  for (; owner < warps && total < kMost; ++owner) {
    if (before <= goal && goal < before + s_warp[last][owner]) break;
    before = add_most(before, s_warp[last][owner]);
  }
  if (owner < warps && total < kMost) {  // (the same for the CTA)
    const T *p = row_of(target, a.target_strides, n), *q = DRAFT ? row_of(draft, a.draft_strides, n) : nullptr;
    // a thread takes consecutive tokens of the run
    const uint32_t first = (rank * warps + owner) * run, size = min(a.vocab, first + run) - first, each = (size + threads - 1) / threads;
    const uint32_t from = first + min(size, tid * each), to = min(first + size, from + each);
    uint64_t own = 0;
#pragma unroll 4
    for (uint32_t x = from; x < to; ++x) own += one(p, q, x, s);
    if constexpr (!DRAFT) {
      for (uint32_t i = 0; i < gone; ++i)
        if (static_cast<uint32_t>(s_gone[i]) >= from && static_cast<uint32_t>(s_gone[i]) < to) own -= s_gone_p[i];
    }
    uint64_t sum = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint64_t v = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= static_cast<uint32_t>(o)) sum += v;
    }
    if (lane == 31) s_warp[turn][warp] = sum;
    __syncthreads();
    uint64_t at = before + sum - own;
    for (uint32_t w = 0; w < warp; ++w) at += s_warp[turn][w];
    if (at <= goal && goal < at + own) {
      uint32_t x = from;
      for (; x + 1 < to; ++x) {
        bool here = true;
        if constexpr (!DRAFT)
          for (uint32_t i = 0; i < gone; ++i) here = here && s_gone[i] != static_cast<int32_t>(x);
        if (here) at += one(p, q, x, s);
        if (at > goal) break;
      }
      a.next[b] = static_cast<int32_t>(x);
    }
  }
  __syncwarp();
  if (ranks > 1) cluster_sync_shared();  // (the others' sums are read until here)
}

template <typename T, bool DRAFT>
cudaError_t launch(const ClearVerifyArgs &a, uint32_t sms, cudaStream_t s) {
  // As many CTAs for each sequence as are resident at once for all of them, of 2048 tokens at least, and eight at most (the portable
  // cluster); 512 threads each, or 256 where those leave room for more of them (64 sequences of 128256 tokens: eight of 256 55 us, four of
  // 512 63; 300 of 32000: two of 256 41, one of 512 50; 4 of 6000: two of 512 10.3, eight 10.7).
  uint32_t ranks = 8;
  while (ranks > 1 && (static_cast<uint64_t>(a.batch) * ranks > 4ull * sms || a.vocab < 2048 * ranks)) ranks /= 2;
  const uint32_t threads = static_cast<uint64_t>(a.batch) * ranks > 2ull * sms && ranks > 1 ? 256 : 512, parts = ranks * (threads / 32);
  const uint32_t run = ((a.vocab + parts - 1) / parts + 31) / 32 * 32;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.batch * ranks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = static_cast<size_t>(a.nodes) * (8 * 3 + 4 * 4);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = ranks;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, verify_kernel<T, DRAFT>, a, ranks, run);
}

template <typename T>
cudaError_t launch(const ClearVerifyArgs &a, uint32_t sms, cudaStream_t s) {
  return a.draft ? launch<T, true>(a, sms, s) : launch<T, false>(a, sms, s);
}

}  // namespace

cudaError_t launch_clear_tree_mask(const ClearTreeArgs &a, cudaStream_t s) {
  const uint32_t words = (a.tokens + 31) / 32;
  tree_mask_kernel<<<dim3((a.tokens * words + 255) / 256, a.batch), 256, a.tokens * sizeof(int32_t), s>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_clear_verify(const ClearVerifyArgs &a, int type, uint32_t sms, cudaStream_t s) {
  if (type == kOutF32) return launch<float>(a, sms, s);
  if (type == kOutF16) return launch<__half>(a, sms, s);
  return launch<__nv_bfloat16>(a, sms, s);
}

}  // namespace rosetta
