// The 8-bit linear product on the tensor cores (tcgen05, accumulators in tensor memory).
//
//   acc[t][n] = sum_k q[t][k] w[n][k]   exactly, in f16: sm_103a's tensor cores have no
// integer kind, but every 8-bit integer is an f16, every product of two (at most 2^14) is exact
// in the f32 accumulator, and so is every sum of up to 1024 of them (at most 2^24).  So the
// accumulators are drained into 32-bit integers every 1024 inputs, and any order of summation
// gives the same words.
//
// A tile is 128 channels (rows of the MMA) x NT tokens (its columns): the weights stay 8-bit up
// to the SM.  Per 64-input step
//   2 copy warps     weight tile (8 KB) and token tile (NT x 64 f16, from tokens_kernel) by
//                    cp.async.bulk into two rings
//   8 or 16 convert warps  a thread a row: 64 bytes to 64 f16 (byte permute into 1024 + u, one
//                    subtraction), stored to tensor memory as the MMA's A operand
//   MMA warp         four tcgen05.mma (K = 16), A from tensor memory, B from shared memory
//   4 or 8 drain warps  every 1024 inputs the accumulators are read back, added up as integers,
//                    and after the last scaled and stored while the next tile runs
// Bound by the products and, between them, by the drains that exactness asks for (tensor pipe 69 % active): 4096 tokens, 4096
// inputs, 14336 channels 315 us, 1.53 PFLOP/s (82 % of the measured bf16 rate), 1024 tokens 86 us; from 33 to 256 tokens by
// the way of a step through copy, conversion and product, and by 7 us to begin and to end (33 tokens 22.7 us, 256 33).
// A launch is persistent over the tiles; where there are few tiles, a cluster of up to eight CTAs
// shares out one tile's inputs and joins the integer sums through distributed shared memory.
//
// Every wait gives up after about two seconds and sets the error flag; the CTA then waits (again
// bounded) for the copies it issued, and frees the tensor memory only when nothing it issued can
// still be in flight.
#include <stdint.h>

#include "clear.h"
#include "dsmem.cuh"
#include "tcgen.cuh"

namespace rosetta {

namespace {

constexpr uint32_t CHUNK_STEPS = 1024 / kPackK;

template <uint32_t NT>
struct Shape {
  // as many as fit: the way of a step through copy, conversion and product takes 2 - 3 us
  static constexpr uint32_t W_STAGES = NT == 64 ? 14 : 8;                 // weight tiles
  static constexpr uint32_t STAGES = NT == 64 ? 12 : NT == 128 ? 9 : 5;  // token tiles and A operands
  static constexpr uint32_t B_TILE = NT * kPackK * 2;
  static constexpr uint32_t DRAIN_WARPS = NT == 256 ? 8 : 4;
  static constexpr uint32_t COLS = NT / (DRAIN_WARPS / 4);                 // of one drain thread
  static constexpr uint32_t CONVERT_GROUPS = NT == 256 ? 2 : 4;            // warpgroups that take turns
  static constexpr uint32_t CONVERT_WARPS = 4 * CONVERT_GROUPS;
  static constexpr uint32_t WARPS = CONVERT_WARPS + DRAIN_WARPS + 4;       // whole warpgroups
  static constexpr uint32_t A_COL = NT;                                    // first column of the A operands
  static constexpr uint32_t TMEM = NT + STAGES * 32 <= 256 ? 256 : 512;
  static constexpr uint32_t RING = W_STAGES * kPackTile + STAGES * B_TILE;
  static_assert(RING <= 225 * 1024 && NT + STAGES * 32 <= 512, "shared and tensor memory");
  // over half an SM's shared memory: two CTAs of a cluster on one SM would wait for each other's
  // tensor memory
  static constexpr uint32_t SMEM = RING > 120 * 1024 ? RING : 120 * 1024;
  // Registers a thread: 96 at launch for 20 warps (80 for 24), then 64 for the conversion, 32 for the
  // copy and MMA warps, the rest for the sums: 256 x 64 + 256 x 160 + 128 x 32 = 61440 of 61440
  // (512 x 64 + 128 x 168 + 128 x 32 = 58368 of 61440)
  static constexpr uint32_t LAUNCH_REGS = 65536 / (WARPS * 32) / 8 * 8, DRAIN_REGS = NT == 256 ? 160 : 168;
  // (more than was launched would wait forever)
  static_assert(CONVERT_WARPS * 64 + DRAIN_WARPS * DRAIN_REGS + 4 * 32 <= WARPS * LAUNCH_REGS, "register shares");
};

// Instruction descriptor, kind::f16: D f32, A and B f16, both K-major, M = 128.
template <uint32_t NT>
constexpr uint32_t kIdescF16 = (1u << 4) | ((NT >> 3) << 17) | ((128u >> 4) << 24);

// One lane of the warp, the same each time.  The MMA warp runs converged and its instructions are predicated on this
// lane, so that descriptors stay in uniform registers.
__device__ __forceinline__ uint32_t elected() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p;
}

template <uint32_t NT>
__device__ __forceinline__ void mma_f16(uint32_t d, uint32_t a, uint64_t bdesc, uint32_t accumulate, uint32_t elect) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(bdesc), "r"(kIdescF16<NT>), "r"(accumulate), "r"(elect)
      : "memory");
}

__device__ __forceinline__ void commit(uint32_t bar, uint32_t elect) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
      "r"(elect)
      : "memory");
}

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]),
      "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]),
      "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
      : "memory");
}

// 16 consecutive f32 columns of this thread's lane (complete after tmem_ld_wait)
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, "
      "[%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr));
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// mbar_wait that reads no clock where the phase is complete already
__device__ __forceinline__ bool wait_quick(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done || mbar_wait(bar, parity);
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

}  // namespace

// The tokens' 8-bit rows as f16 tiles [token tile][k step][NT x 64], zeros beyond the sizes: 8 values
// (16 bytes written) a thread.  A tile has the no-swizzle K-major layout of the tensor cores: core matrices
// of 8 rows x 16 bytes, K-adjacent ones 128 bytes apart, groups of 8 rows 1024 bytes apart.
__global__ void __launch_bounds__(256) tokens_kernel(const int8_t *__restrict__ q, int64_t pitch, uint32_t tokens,
                                                     uint32_t inner, uint32_t k_steps, uint32_t nt, uint4 *__restrict__ tiles,
                                                     uint64_t items) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint64_t id = static_cast<uint64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
  if (id >= items) return;
  // neighbouring threads: the row within 8, then k within the step, so that a warp writes 512 bytes in a row
  const uint32_t r = id & 7u, kg = (id >> 3) & 7u;
  const uint64_t group = id >> 6;  // [tile][k step][row group]
  const uint32_t groups = nt / 8, rg = group % groups;
  const uint64_t ts = group / groups;
  const uint32_t ks = ts % k_steps;
  const uint64_t t = ts / k_steps * nt + rg * 8 + r;
  const uint32_t k0 = ks * kPackK + kg * 8;
  uint32_t w[2] = {0u, 0u};
  if (t < tokens) {
    const int8_t *src = q + static_cast<int64_t>(t) * pitch + k0;
    if (k0 + 8 <= inner && (reinterpret_cast<uintptr_t>(src) & 7u) == 0) {
      const uint2 v = __ldg(reinterpret_cast<const uint2 *>(src));
      w[0] = v.x;
      w[1] = v.y;
    } else {
#pragma unroll
      for (uint32_t e = 0; e < 8; ++e)
        if (k0 + e < inner) w[e >> 2] |= static_cast<uint32_t>(static_cast<uint8_t>(src[e])) << (8 * (e & 3u));
    }
  }
  uint4 o;
  int8x4_f16(w[0], o.x, o.y);
  int8x4_f16(w[1], o.z, o.w);
  tiles[ts * (nt * 8) + rg * 64 + kg * 8 + r] = o;
}

template <uint32_t NT, int OUT>
__global__ void __launch_bounds__(Shape<NT>::WARPS * 32, 1)
    linear_tc_kernel(const ClearLinearArgs a, const uint8_t *__restrict__ tok, uint32_t row_tiles, uint32_t tok_tiles) {
  using S = Shape<NT>;
  extern __shared__ __align__(1024) unsigned char smem[];
  // wfull, wempty [S::W_STAGES]; bfull, afull, empty [STAGES]; dfull, dempty, free
  __shared__ __align__(8) uint64_t bars[2 * S::W_STAGES + 3 * S::STAGES + 3];
  __shared__ uint32_t tmem_slot;
  __shared__ uint32_t s_fail, s_unsafe;
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t base = smem_addr(smem), bar0 = smem_addr(bars);
  const auto wfull = [&](uint32_t s) { return bar0 + 8u * s; };
  const auto wempty = [&](uint32_t s) { return bar0 + 8u * (S::W_STAGES + s); };
  const auto bfull = [&](uint32_t s) { return bar0 + 8u * (2 * S::W_STAGES + s); };
  const auto afull = [&](uint32_t s) { return bar0 + 8u * (2 * S::W_STAGES + S::STAGES + s); };
  const auto empty = [&](uint32_t s) { return bar0 + 8u * (2 * S::W_STAGES + 2 * S::STAGES + s); };
  const uint32_t dfull = bar0 + 8u * (2 * S::W_STAGES + 3 * S::STAGES), dempty = dfull + 8u, free_bar = dempty + 8u;
  const uint32_t b_ring = base + S::W_STAGES * kPackTile;

  if (warp == 0) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_slot)),
                 "r"(S::TMEM)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (threadIdx.x == 0) {
    s_fail = s_unsafe = 0u;
    for (uint32_t s = 0; s < S::W_STAGES; ++s) {
      mbar_init(wfull(s), 1);
      mbar_init(wempty(s), 4);
    }
    for (uint32_t s = 0; s < S::STAGES; ++s) {
      mbar_init(bfull(s), 1);
      mbar_init(afull(s), 4);
      mbar_init(empty(s), 1);
    }
    mbar_init(dfull, 1);
    mbar_init(dempty, S::DRAIN_WARPS);
    mbar_init(free_bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;

  // the cluster's CTAs share out a tile's steps
  uint32_t rank = 0, ranks = 1;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
  const uint32_t per = (a.k_steps + ranks - 1) / ranks;
  const uint32_t k0 = min(a.k_steps, rank * per), steps = min(a.k_steps, k0 + per) - k0;
  const uint32_t tiles = row_tiles * tok_tiles;
  const uint32_t first = blockIdx.x / ranks, stride = gridDim.x / ranks;
  const auto give_up = [&]() {
    atomicExch(a.err_flag, 2u);
    atomicExch(&s_fail, 1u);
  };

  if (warp < S::CONVERT_WARPS) {
    // ---- weights to f16, in tensor memory ----
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    const uint32_t mine = first < tiles ? (tiles - 1 - first) / stride + 1 : 0;  // tiles of this CTA
    // warpgroup g takes the steps g, g + CONVERT_GROUPS, ...
    for (uint32_t it = warp / 4; it < mine * steps; it += S::CONVERT_GROUPS) {
      const uint32_t ws = it % S::W_STAGES, s = it % S::STAGES;
      if (!__all_sync(0xffffffffu, wait_quick(wfull(ws), (it / S::W_STAGES) & 1u))) {
        give_up();
        goto done;
      }
      uint32_t v[32];
      const uint32_t turn = threadIdx.x >> 1 & 3u;  // how this row's chunks are moved
      const uint4 *src = reinterpret_cast<const uint4 *>(smem + ws * kPackTile) + threadIdx.x % kPackRows * 4;
#pragma unroll
      for (uint32_t c = 0; c < 4; ++c) {
        const uint4 w = src[c ^ turn];
        int8x4_f16(w.x, v[c * 8 + 0], v[c * 8 + 1]);
        int8x4_f16(w.y, v[c * 8 + 2], v[c * 8 + 3]);
        int8x4_f16(w.z, v[c * 8 + 4], v[c * 8 + 5]);
        int8x4_f16(w.w, v[c * 8 + 6], v[c * 8 + 7]);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(wempty(ws));
      if (it >= S::STAGES && !__all_sync(0xffffffffu, wait_quick(empty(s), (it / S::STAGES - 1) & 1u))) {
        give_up();
        goto done;
      }
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      tmem_st32(tmem + (((warp % 4) * 32u) << 16) + S::A_COL + s * 32u, v);
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(afull(s));
    }
  } else if (warp < S::CONVERT_WARPS + S::DRAIN_WARPS) {
    // ---- sums: lane = channel, this warp's quarter of tensor memory, COLS tokens ----
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(S::DRAIN_REGS));
    const uint32_t col0 = (warp - S::CONVERT_WARPS) / 4 * S::COLS;
    const uint32_t quarter = tmem + (((warp % 4) * 32u) << 16);
    uint32_t chunk = 0;
    for (uint32_t tile = first; tile < tiles; tile += stride) {
      int32_t acc[S::COLS];
#pragma unroll
      for (uint32_t i = 0; i < S::COLS; ++i) acc[i] = 0;
      for (uint32_t k = 0; k < steps; k += CHUNK_STEPS, ++chunk) {
        if (!__all_sync(0xffffffffu, wait_quick(dfull, chunk & 1u))) {
          give_up();
          goto done;
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
        for (uint32_t c = 0; c < S::COLS; c += 16) {
          uint32_t v[16];
          tmem_ld16(quarter + col0 + c, v);
#pragma unroll
          for (uint32_t i = 0; i < 16; ++i) acc[c + i] += __float2int_rn(__uint_as_float(v[i]));
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(dempty);
      }
      const uint32_t t0 = tile % tok_tiles * NT + col0, n = tile / tok_tiles * kPackRows + (warp % 4) * 32 + lane;
      if (ranks == 1) {
        if (n < a.channels) {
          const float w_scale = a.w_scale[n], bias = a.bias ? a.bias[n] : 0.0f;
          if constexpr (OUT != kOutCodes && NT == 256) {
#pragma unroll
            for (uint32_t i = 0; i < S::COLS; ++i)
              if (t0 + i < a.tokens) clear_store<OUT>(a, t0 + i, n, clear_scaled(acc[i], __ldg(a.scale + t0 + i), w_scale, a.bias != nullptr, bias));
          } else {
            // a few tokens at a time, all of whose loads (scales, table entries) go before their stores, which hold loads back:
            // 4096 tokens, 4096 x 14336 with a table 367 us against 481, 333 tokens, 1021 x 2999 12.0 against 12.5 (floats of
            // 256 columns are 1 % faster one by one)
            constexpr uint32_t STEP = 8;
#pragma unroll
            for (uint32_t i = 0; i < S::COLS; i += STEP) {
              if (t0 + i >= a.tokens) break;
              float y[STEP];
#pragma unroll
              for (uint32_t e = 0; e < STEP; ++e) y[e] = __ldg(a.scale + min(t0 + i + e, a.tokens - 1));
#pragma unroll
              for (uint32_t e = 0; e < STEP; ++e) y[e] = clear_scaled(acc[i + e], y[e], w_scale, a.bias != nullptr, bias);
              if constexpr (OUT != kOutCodes) {
#pragma unroll
                for (uint32_t e = 0; e < STEP; ++e)
                  if (t0 + i + e < a.tokens) clear_store<OUT>(a, t0 + i + e, n, y[e]);
              } else {
                uint32_t code[STEP];
                int8_t value[STEP];
#pragma unroll
                for (uint32_t e = 0; e < STEP; ++e) code[e] = clear_code(a, y[e]);
                if (a.values) {
#pragma unroll
                  for (uint32_t e = 0; e < STEP; ++e) value[e] = __ldg(a.table + code[e]);
                }
                uint8_t *out = static_cast<uint8_t *>(a.out) + static_cast<int64_t>(t0 + i) * a.out_pitch + n;
                int8_t *to = a.values + static_cast<int64_t>(t0 + i) * a.values_pitch + n;
#pragma unroll
                for (uint32_t e = 0; e < STEP; ++e, out += a.out_pitch, to += a.values_pitch) {
                  if (t0 + i + e >= a.tokens) break;
                  *out = static_cast<uint8_t>(code[e]);
                  if (a.values) *to = value[e];
                }
              }
            }
          }
        }
      } else {
        // (one tile per cluster) the rings are idle now: this CTA's sums into them, [token][channel]
        int32_t *part = reinterpret_cast<int32_t *>(smem);
#pragma unroll
        for (uint32_t i = 0; i < S::COLS; ++i) part[(col0 + i) * kPackRows + (warp % 4) * 32 + lane] = acc[i];
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
    const uint32_t role = warp - S::CONVERT_WARPS - S::DRAIN_WARPS;
    if (role == 0 && lane == 0) {
      // ---- weight copies ----
      uint32_t slot = 0, par = 1, issued = 0;  // the first round's wait is for the phase before the first: none
      bool ok = true;
      for (uint32_t tile = first; tile < tiles && ok; tile += stride) {
        const int8_t *src = a.packed + (static_cast<size_t>(tile / tok_tiles) * a.k_steps + k0) * kPackTile;
        for (uint32_t k = 0; k < steps; ++k, ++issued, src += kPackTile) {
          if (!wait_quick(wempty(slot), par)) {
            ok = false;
            break;
          }
          expect_tx(wfull(slot), kPackTile);
          bulk_load(base + slot * kPackTile, src, kPackTile, wfull(slot));
          if (++slot == S::W_STAGES) {
            slot = 0;
            par ^= 1u;
          }
        }
      }
      if (!ok) give_up();
      // the copies issued land before the shared memory is released, whichever warp gave up
      for (uint32_t i = issued > S::W_STAGES ? issued - S::W_STAGES : 0; i < issued; ++i)
        if (!mbar_wait(wfull(i % S::W_STAGES), (i / S::W_STAGES) & 1u)) {
          atomicExch(&s_unsafe, 1u);
          give_up();
        }
    } else if (role == 1 && lane == 0) {
      // ---- token copies, after the kernel that makes the tiles ----
      asm volatile("griddepcontrol.wait;" ::: "memory");
      uint32_t slot = 0, par = 1, issued = 0;
      bool ok = true;
      for (uint32_t tile = first; tile < tiles && ok; tile += stride) {
        const uint8_t *src = tok + (static_cast<size_t>(tile % tok_tiles) * a.k_steps + k0) * S::B_TILE;
        for (uint32_t k = 0; k < steps; ++k, ++issued, src += S::B_TILE) {
          if (!wait_quick(empty(slot), par)) {
            ok = false;
            break;
          }
          expect_tx(bfull(slot), S::B_TILE);
          bulk_load(b_ring + slot * S::B_TILE, src, S::B_TILE, bfull(slot));
          if (++slot == S::STAGES) {
            slot = 0;
            par ^= 1u;
          }
        }
      }
      if (!ok) give_up();
      for (uint32_t i = issued > S::STAGES ? issued - S::STAGES : 0; i < issued; ++i)
        if (!mbar_wait(bfull(i % S::STAGES), (i / S::STAGES) & 1u)) {
          atomicExch(&s_unsafe, 1u);
          give_up();
        }
    } else if (role == 2) {
      // ---- MMAs ----
      const uint32_t elect = elected();
      const auto ready = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, wait_quick(bar, parity)); };
      uint32_t slot = 0, par = 0, dpar = 1;
      for (uint32_t tile = first; tile < tiles; tile += stride)
        for (uint32_t k = 0; k < steps; ++k) {
          bool ok = ready(bfull(slot), par) && ready(afull(slot), par);
          if (k % CHUNK_STEPS == 0) {  // the accumulators have been read
            ok = ok && ready(dempty, dpar);
            dpar ^= 1u;
          }
          if (!ok) {
            give_up();
            goto done;
          }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint64_t sb = smem_desc(b_ring + slot * S::B_TILE);
          const uint32_t sa = tmem + S::A_COL + slot * 32u;
#pragma unroll
          for (uint32_t kk = 0; kk < kPackK / 16; ++kk)  // 256 bytes on: 16 in the descriptor's units
            mma_f16<NT>(tmem, sa + kk * 8u, sb + kk * 16u, (k % CHUNK_STEPS | kk) != 0, elect);
          commit(empty(slot), elect);
          if (k % CHUNK_STEPS == CHUNK_STEPS - 1 || k + 1 == steps) commit(dfull, elect);
          if (++slot == S::STAGES) {
            slot = 0;
            par ^= 1u;
          }
        }
      // no commit arrives after the CTA's end: the last one of every slot in use
      const uint32_t total = first < tiles ? ((tiles - 1 - first) / stride + 1) * steps : 0;
      for (uint32_t i = total > S::STAGES ? total - S::STAGES : 0; i < total; ++i)
        if (!ready(empty(i % S::STAGES), (i / S::STAGES) & 1u)) {
          give_up();
          goto done;
        }
    }
  }
done:
  __syncwarp();
  __syncthreads();
  const bool fail = s_fail != 0u;
  if (ranks > 1) {
    // every CTA of the cluster arrives, failed or not
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (!fail && first < tiles) {
      // this CTA's share of the tokens: sums over the cluster
      const uint32_t t0 = first % tok_tiles * NT, n0 = first / tok_tiles * kPackRows;
      const uint32_t share = (NT + ranks - 1) / ranks;
      for (uint32_t i = threadIdx.x; i < share * kPackRows; i += blockDim.x) {
        const uint32_t col = rank * share + i / kPackRows, n = n0 + i % kPackRows;
        if (col >= NT || t0 + col >= a.tokens || n >= a.channels) continue;
        int32_t sum = 0;
        for (uint32_t r = 0; r < ranks; ++r)
          sum += static_cast<int32_t>(dsmem_ld_u32(dsmem_map(base + (col * kPackRows + i % kPackRows) * 4u, r)));
        clear_store<OUT>(a, t0 + col, n, clear_scaled(sum, a.scale[t0 + col], a.w_scale[n], a.bias != nullptr, a.bias ? a.bias[n] : 0.0f));
      }
    }
    // no CTA leaves while another reads its shared memory
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  if (fail) {
    // what was issued ends by itself: the tensor memory is freed after it (a CTA that kept it would end in an error of
    // the whole context), and only where this wait too gives up, or copies may be in flight, it stays allocated
    if (warp == S::CONVERT_WARPS + S::DRAIN_WARPS + 2) {
      commit(free_bar, elected());
      if (!mbar_wait(free_bar, 0)) atomicExch(&s_unsafe, 1u);
    }
    __syncthreads();
  }
  if (warp == 0 && !s_unsafe)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::TMEM) : "memory");
}

namespace {

// Columns of a tile, and CTAs that share out its inputs.
struct Plan {
  uint32_t columns, ranks;
  uint64_t ns;
};

// A cluster is doubled while the GPU holds all of them at once (of 152 SMs 76 clusters of two, 36 of four, 15 of eight: a
// second round costs more than it saves, 2048 inputs and channels, 64 tokens 15.9 us with eight and 10.3 with four) and
// four steps are left to each CTA.
uint32_t ranks_of(uint64_t tiles, uint32_t k_steps, uint32_t sms) {
  uint32_t ranks = 1;
  while (ranks < 8 && tiles <= (ranks == 1 ? sms / 2 : ranks == 2 ? sms * 9 / 38 : sms / 10) && k_steps >= ranks * 2 * 4) ranks *= 2;
  return ranks;
}

// The columns by an estimate of the time: a start and an end, longer for more columns and for the join of a cluster's sums, and
// so much a step, as measured.  Wide tiles save conversions of weights, narrow ones make more CTAs: 256 tokens, 4096 inputs,
// 14336 channels 33.2 us with 256 columns, 49 with 128, 54 with 64; 768 inputs, 3072 channels 17.2, 12.1, 9.8.
Plan plan_of(const ClearLinearArgs &a, uint32_t sms) {
  const uint32_t row_tiles = (a.channels + kPackRows - 1) / kPackRows;
  Plan best = {64, 1, ~0ull};
  for (uint32_t nt = 256; nt >= 64; nt /= 2) {
    if (nt > 64 && a.tokens <= nt / 2) continue;
    const uint64_t tiles = static_cast<uint64_t>(row_tiles) * ((a.tokens + nt - 1) / nt);
    const uint32_t ranks = ranks_of(tiles, a.k_steps, sms);
    const uint64_t steps = ranks > 1 ? (a.k_steps + ranks - 1) / ranks : (tiles + sms - 1) / sms * a.k_steps;
    const uint64_t ns = (nt == 256 ? (ranks > 1 ? 14500 : 11000) : nt == 128 ? 10000 : ranks > 1 ? 9300 : 8500) +
                        steps * (nt == 256 ? 275 : nt == 128 ? 285 : 210);
    if (ns < best.ns) best = {nt, ranks, ns};
  }
  return best;
}

template <uint32_t NT, int OUT>
cudaError_t launch_tc(const ClearLinearArgs &a, uint32_t ranks, void *work, uint32_t sms, cudaStream_t s) {
  using S = Shape<NT>;
  const uint32_t row_tiles = (a.channels + kPackRows - 1) / kPackRows, tok_tiles = (a.tokens + NT - 1) / NT;
  const uint64_t items = static_cast<uint64_t>(tok_tiles) * a.k_steps * NT * 8;
  tokens_kernel<<<static_cast<uint32_t>((items + 255) / 256), 256, 0, s>>>(a.q, a.q_pitch, a.tokens, a.inner, a.k_steps, NT,
                                                                          static_cast<uint4 *>(work), items);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  auto kern = linear_tc_kernel<NT, OUT>;
  e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(S::SMEM));
  if (e != cudaSuccess) return e;
  const uint64_t tiles = static_cast<uint64_t>(row_tiles) * tok_tiles;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ranks > 1 ? static_cast<uint32_t>(tiles) * ranks : static_cast<uint32_t>(tiles < sms ? tiles : sms));
  cfg.blockDim = dim3(S::WARPS * 32);
  cfg.dynamicSmemBytes = S::SMEM;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = ranks;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kern, a, static_cast<const uint8_t *>(work), row_tiles, tok_tiles);
}

template <int OUT>
cudaError_t launch_out(const ClearLinearArgs &a, void *work, uint32_t sms, cudaStream_t s) {
  const Plan p = plan_of(a, sms);
  return p.columns == 64    ? launch_tc<64, OUT>(a, p.ranks, work, sms, s)
         : p.columns == 128 ? launch_tc<128, OUT>(a, p.ranks, work, sms, s)
                            : launch_tc<256, OUT>(a, p.ranks, work, sms, s);
}

}  // namespace

uint64_t linear_tc_ns(const ClearLinearArgs &a, uint32_t sms) { return plan_of(a, sms).ns; }

size_t linear_tc_bytes(const ClearLinearArgs &a, uint32_t sms) {
  const uint32_t nt = plan_of(a, sms).columns;
  return static_cast<size_t>((a.tokens + nt - 1) / nt) * a.k_steps * nt * (kPackK * 2);
}

cudaError_t launch_clear_linear_tc(const ClearLinearArgs &a, int out_kind, void *work, uint32_t sms, cudaStream_t s) {
  switch (out_kind) {
    case kOutF32: return launch_out<kOutF32>(a, work, sms, s);
    case kOutF16: return launch_out<kOutF16>(a, work, sms, s);
    case kOutBf16: return launch_out<kOutBf16>(a, work, sms, s);
    default: return launch_out<kOutCodes>(a, work, sms, s);
  }
}

}  // namespace rosetta
