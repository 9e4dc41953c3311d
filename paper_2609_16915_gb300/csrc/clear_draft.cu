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
// All sums are of whole multiples of 2^-56, so no order changes them, and they are compared as integers.
// What is read: p(x) and q(x) of every node at once, and whole rows only of nodes whose children have been rejected,
// twice where they are the last (the second time by one warp).  Latency bound for a few sequences; for many by reading one or two rows of each.
#include <stdint.h>

#include "clear.h"
#include "dsmem.cuh"

namespace rosetta {

namespace {

constexpr uint64_t kOne = 1ull << 56, kMost = 1ull << 62;  // sums stay at kMost: no probabilities
constexpr uint32_t kThreads = 512, kWarps = kThreads / 32;

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

// a probability in units of 2^-56; what is none counts as zero
__device__ __forceinline__ uint64_t fixed(float p, bool &bad) {
  const bool in = p >= 0.0f && p <= 2.0f;  // (rounded sums may pass 1)
  bad |= !in;
  return in ? __float2ull_rn(p * 72057594037927936.0f) : 0;
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

// A cluster of CTAs for each sequence; a warp takes a run of the vocabulary, a lane VEC of every 32 VEC.
template <typename T, bool DRAFT, int VEC>
__global__ void __launch_bounds__(kThreads) verify_kernel(const ClearVerifyArgs a, uint32_t ranks, uint32_t run) {
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ uint64_t s_warp[2][kWarps], s_total[2];
  __shared__ uint32_t s_bad;
  const uint32_t nodes = a.nodes, tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
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
  for (uint32_t c = rank + tid * ranks; c < nodes; c += kThreads * ranks) {
    int32_t up = c ? a.parents[static_cast<int64_t>(b) * a.parents_pitch + c] : -1;
    const int32_t x = c ? a.tokens[static_cast<int64_t>(b) * a.tokens_pitch + c] : 0;
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
  if (ranks > 1) {
    cluster_sync_shared();
    for (uint32_t c = tid; c < nodes; c += kThreads) {
      const uint32_t from = c % ranks;
      if (from == rank) continue;
      s_up[c] = static_cast<int32_t>(dsmem_ld_u32(dsmem_map(smem_addr(s_up + c), from)));
      s_token[c] = static_cast<int32_t>(dsmem_ld_u32(dsmem_map(smem_addr(s_token + c), from)));
      s_u[c] = dsmem_ld_u64(dsmem_map(smem_addr(s_u + c), from));
      s_p[c] = dsmem_ld_u64(dsmem_map(smem_addr(s_p + c), from));
      if constexpr (DRAFT) s_q[c] = dsmem_ld_u64(dsmem_map(smem_addr(s_q + c), from));
    }
  }
  __syncthreads();

  const uint32_t lo = (rank * kWarps + warp) * run, hi = min(a.vocab, lo + run);  // this warp's run
  const auto row_of = [&](const T *rows, const int64_t (&strides)[2], uint32_t n) { return rows + static_cast<int64_t>(n) * strides[1]; };
  // what is left of VEC tokens from x on
  const auto load = [&](const T *p, const T *q, uint32_t x, uint64_t s, uint64_t (&w)[VEC]) {
    if (VEC > 1 && x + VEC > hi) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        w[e] = x + e < hi ? fixed(to_float(p[x + e]), bad) : 0;
        if (DRAFT && x + e < hi) w[e] = less(w[e], times(fixed(to_float(q[x + e]), bad), s));
      }
      return;
    }
    const Pack<T, VEC> pv = *reinterpret_cast<const Pack<T, VEC> *>(p + x);
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[e] = fixed(to_float(pv.v[e]), bad);
    if constexpr (DRAFT) {
      if (s != 0) {
        const Pack<T, VEC> qv = *reinterpret_cast<const Pack<T, VEC> *>(q + x);
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[e] = less(w[e], times(fixed(to_float(qv.v[e]), bad), s));
      }
    }
  };
  uint32_t turn = 0;
  uint64_t before = 0;  // the sum of the CTAs before this one
  // the sum of what is left of node n's row, over the cluster; the warps' sums stay in s_warp[turn ^ 1]
  const auto row_sum = [&](uint32_t n, uint64_t s, uint32_t gone) {
    const T *p = row_of(target, a.target_strides, n), *q = DRAFT ? row_of(draft, a.draft_strides, n) : nullptr;
    uint64_t sum = 0;
    for (uint32_t x = lo + lane * VEC; x < hi; x += 32 * VEC) {
      uint64_t w[VEC];
      load(p, q, x, s, w);
#pragma unroll
      for (int e = 1; e < VEC; ++e) w[0] += w[e];  // (2^60)
      sum = add_most(sum, w[0]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum = add_most(sum, __shfl_xor_sync(0xffffffffu, sum, o));
    if (lane == 0) s_warp[turn][warp] = sum;
    __syncthreads();
    if (!DRAFT && gone) {
      for (uint32_t i = tid; i < gone; i += kThreads) {
        const uint32_t w = static_cast<uint32_t>(s_gone[i]) / run;
        if (w / kWarps == rank) atomicAdd(reinterpret_cast<unsigned long long *>(&s_warp[turn][w % kWarps]), 0ull - s_gone_p[i]);
      }
      __syncthreads();
    }
    uint64_t total = 0;
#pragma unroll
    for (uint32_t w = 0; w < kWarps; ++w) total = add_most(total, s_warp[turn][w]);
    before = 0;
    if (ranks > 1) {
      if (tid == 0) s_total[turn] = total;
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

  // ---- the walk: every warp for itself, all alike ----
  uint32_t n = 0, length = 1, gone = 0;
  uint64_t s = 0, z = kOne, left = kOne;
  bool stale = false;  // z is that of the s before
  if (tid == 0) s_path[0] = 0;
  for (uint32_t c0 = 1; c0 < nodes;) {
    const uint32_t hit = __ballot_sync(0xffffffffu, c0 + lane < nodes && s_up[min(c0 + lane, nodes - 1)] == static_cast<int32_t>(n));
    if (hit == 0) {
      c0 += 32;
      continue;
    }
    const uint32_t c = c0 + __ffs(hit) - 1;
    c0 = c + 1;
    const uint64_t u = s_u[c];
    bool yes;
    if constexpr (DRAFT) {
      if (stale) z = row_sum(n, s, 0);
      stale = false;
      yes = __umul64hi(u, times(s_q[c], z)) < less(s_p[c], times(s_q[c], s));
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
        __syncthreads();  // (all have looked at the list)
        if (tid == 0) {
          s_gone[gone] = s_token[c];
          s_gone_p[gone] = p;
        }
        ++gone;
        __syncthreads();
      }
    }
    if (yes) {
      if (tid == 0) s_path[length] = static_cast<int32_t>(c);
      ++length;
      n = c;
      s = 0;
      z = left = kOne;
      stale = false;
      gone = 0;
      __syncthreads();
    }
  }

  // ---- the next token ----
  uint64_t total = row_sum(n, s, gone);
  if (total == 0 && (s != 0 || gone != 0)) {  // nothing is left: the target's row itself
    s = 0;
    gone = 0;
    total = row_sum(n, s, gone);
  }
  if (tid == 0) s_bad = 0;
  __syncthreads();
  if (bad) s_bad = 1;
  __syncthreads();
  if (tid == 0 && (s_bad || total == 0 || total >= kMost)) atomicMax(a.err_flag, 1u);
  if (rank == 0) {
    for (uint32_t i = tid; i < nodes; i += kThreads) a.path[static_cast<int64_t>(b) * a.path_pitch + i] = i < length ? s_path[i] : -1;
    if (tid == 0) {
      a.count[b] = static_cast<int32_t>(length);
      if (total == 0 || total >= kMost) a.next[b] = -1;
    }
  }
  const uint64_t goal = __umul64hi(s_u[0], total);  // the first running sum above it
  const uint32_t last = turn ^ 1;
  for (uint32_t w = 0; w < warp; ++w) before = add_most(before, s_warp[last][w]);
  if (total < kMost && before <= goal && goal < before + s_warp[last][warp]) {
    const T *p = row_of(target, a.target_strides, n), *q = DRAFT ? row_of(draft, a.draft_strides, n) : nullptr;
    for (uint32_t x0 = lo; x0 < hi; x0 += 32 * VEC) {
      const uint32_t x = x0 + lane * VEC;
      uint64_t w[VEC] = {};
      if (x < hi) load(p, q, x, s, w);
      if constexpr (!DRAFT) {
        for (uint32_t i = 0; i < gone; ++i) {
          const uint32_t e = static_cast<uint32_t>(s_gone[i]) - x;
#pragma unroll
          for (int j = 0; j < VEC; ++j)
            if (e == static_cast<uint32_t>(j)) w[j] = 0;
        }
      }
      uint64_t own = 0, sum;
#pragma unroll
      for (int e = 0; e < VEC; ++e) own += w[e];
      sum = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint64_t v = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= static_cast<uint32_t>(o)) sum += v;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, before + sum > goal);
      if (past) {
        if (lane == static_cast<uint32_t>(__ffs(past) - 1)) {
          uint64_t at = before + sum - own;
          int e = 0;
          while (e + 1 < VEC && at + w[e] <= goal) at += w[e++];
          a.next[b] = static_cast<int32_t>(x + e);
        }
        break;
      }
      before += __shfl_sync(0xffffffffu, sum, 31);
    }
  }
  if (ranks > 1) cluster_sync_shared();  // (the others' sums are read until here)
}

template <typename T, bool DRAFT, int VEC>
cudaError_t launch(const ClearVerifyArgs &a, uint32_t sms, cudaStream_t s) {
  const uint32_t ranks = 1;
  const uint32_t parts = ranks * kWarps, each = 32 * VEC;
  const uint32_t run = ((a.vocab + parts - 1) / parts + each - 1) / each * each;
  const size_t smem = static_cast<size_t>(a.nodes) * (8 * 3 + 4 * 4);
  verify_kernel<T, DRAFT, VEC><<<a.batch * ranks, kThreads, smem, s>>>(a, ranks, run);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch(const ClearVerifyArgs &a, uint32_t sms, cudaStream_t s) {
  constexpr int WIDE = 16 / sizeof(T);
  uintptr_t at = reinterpret_cast<uintptr_t>(a.target) | static_cast<uintptr_t>((a.target_strides[0] | a.target_strides[1]) * sizeof(T));
  if (!a.draft) return at % 16 == 0 ? launch<T, false, WIDE>(a, sms, s) : launch<T, false, 1>(a, sms, s);
  at |= reinterpret_cast<uintptr_t>(a.draft) | static_cast<uintptr_t>((a.draft_strides[0] | a.draft_strides[1]) * sizeof(T));
  return at % 16 == 0 ? launch<T, true, WIDE>(a, sms, s) : launch<T, true, 1>(a, sms, s);
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
