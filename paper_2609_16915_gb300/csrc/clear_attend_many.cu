// Causal attention over the paged 8-bit cache for many query rows: prompts.
//
// Bound by the issue of the softmax's and the conversions' instructions (about 60 % of the issue slots; the tensor pipe is
// active for 35 % of the time, DRAM for 5 %): 8 x 256 queries at 4096 positions, 32 heads over 8 of 128, 167 us, 797 TFLOP/s
// of 4 D operations per row and visible position.  tcgen05, scores, weights and outputs in tensor memory.
//
// A block takes 256 query rows of one cached head (its group's heads, token by token), as two tiles of 128, and walks
// over the positions 64 at a time:
//   4 + 4 convert warps  the 8-bit keys and values, copied ahead from the pages by cp.async (four tiles in flight), to f16
//                    in shared memory, both K-major and exact: keys [position][dimension], with the sign of their
//                    scale, values transposed by byte permutes to [dimension][position]
//   MMA warp         S = Q K^T, 128 x 64 a tile, two of them ahead; O += P V with P from tensor memory
//   2 x 8 softmax warps  two threads a row, 32 positions each: scores from tensor memory, times the page's key scale and the row's
//                    factor, 2^(s - m + 7) with the running maximum m of s + log2(vs / sv) raised only where it is passed
//                    by 8 (then O is scaled down in place), P vs / sv as f16 over the scores' columns
// With two score tiles a row tile, one row tile's next scores are there when its softmax is done: the handing over
// between warps and tensor cores (about 900 clocks a round) runs under the exponentials.
// Rows and pages that are not seen have weight 0; a page whose value scale is not a number has the scale zero and a key scale
// of NaN, which reaches exactly the rows that see it.
//
// Every wait gives up after about two seconds and sets the error flag; the block then waits (again bounded) for the
// products it issued before it frees the tensor memory.
#include <stdint.h>

#include <type_traits>

#include "clear_attend.cuh"
#include "dsmem.cuh"
#include "pairs.cuh"
#include "tcgen.cuh"

namespace rosetta {

namespace {

constexpr uint32_t ROWS = 128, POS = 64, TILE_WARPS = 8, CONVERT_WARPS = 8;  // (TILE_WARPS: softmax warps of a row tile)
// Single precision: one row tile, its queries in two halves.
template <typename T>
constexpr bool kSplit = sizeof(T) == 4;
// Weights in two halves: all but bfloat16, whose own rounding hides that of weights to 11 bits (float16 outputs 2.1e-4 off, their rounding alone, against 3.0e-4; 8 x 256 queries at
// 4096 positions 186 us against 167).
template <typename T>
constexpr bool kFine = !std::is_same<T, __nv_bfloat16>::value;
template <typename T>
constexpr uint32_t kSoftWarps = kSplit<T> ? TILE_WARPS : 2 * TILE_WARPS;
template <typename T>
constexpr uint32_t kWarps = kSoftWarps<T> + CONVERT_WARPS + 1;  // (25 leave 72 registers a thread)
constexpr uint32_t RING = 3, STAGED = 4;  // f16 tiles of keys and of values; 8-bit tiles of both
// Single precision adds its accumulators to a sum of their own every FOLD tiles: 256 positions lose up to 2e-6 (8 x 256 queries
// at 4096 positions 305 us; 285 with 8 tiles, 265 without, where 4096 positions lose up to 3e-5).
constexpr uint32_t FOLD = 4;
// No accumulator takes more than this many tiles: a longer range's outputs so far, and its sum of weights, are then added up
// aside (the outputs in the place of the row's partial result).
constexpr uint32_t RUN = kMostPositions / POS;
static_assert(RUN % FOLD == 0, "runs are whole folds");
constexpr float kRaise = 8.0f, kLift = 7.0f;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr uint32_t V_GROUP = POS * 16;  // bytes of eight dimensions of a value tile

template <int DP>
struct Many {
  static constexpr uint32_t Q_TILE = ROWS * DP * 2, K_TILE = POS * DP * 2, V_TILE = DP / 8 * V_GROUP, RAW = POS * DP;
  static constexpr uint32_t K_AT = 2 * Q_TILE, V_AT = K_AT + RING * K_TILE, RAW_AT = V_AT + RING * V_TILE;
  static constexpr uint32_t SMEM = RAW_AT + STAGED * 2 * RAW;
  static constexpr uint32_t O_COL = 4 * POS;  // score tiles of the two row tiles: two of 64 columns each
};

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint32_t half2_bits(__half2 h) { return *reinterpret_cast<const uint32_t *>(&h); }
__device__ __forceinline__ __half2 bits_half2(uint32_t v) { return *reinterpret_cast<const __half2 *>(&v); }

// no swizzle, K-major: core matrices of 8 rows x 16 bytes, K-adjacent ones 128 bytes apart, groups of 8 rows
// `group` bytes apart
__device__ __forceinline__ uint64_t desc_of(uint32_t saddr, uint32_t group) {
  return static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4) | (static_cast<uint64_t>(128u >> 4) << 16) |
         (static_cast<uint64_t>(group >> 4) << 32) | (1ull << 46);
}

// kind::f16: D f32, A and B f16, both K-major, M = 128
__host__ __device__ constexpr uint32_t idesc(uint32_t n) { return (1u << 4) | ((n >> 3) << 17) | ((128u >> 4) << 24); }

// One lane of the warp, the same each time.  The MMA warp runs converged and its instructions are predicated on this
// lane, so that descriptors stay in uniform registers: with one lane branching off, issuing a product cost about 60 clocks.
__device__ __forceinline__ uint32_t elected() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p;
}

__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t id, uint32_t accumulate, uint32_t elect) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(id), "r"(accumulate), "r"(elect)
      : "memory");
}

__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t id, uint32_t accumulate, uint32_t elect) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(id), "r"(accumulate), "r"(elect)
      : "memory");
}

__device__ __forceinline__ void commit(uint32_t bar, uint32_t elect) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar),
      "r"(elect)
      : "memory");
}

// 32 consecutive columns of this thread's lane (complete after tmem_wait_ld)
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float *v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]),
        "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
        "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_ld16f(uint32_t taddr, float (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
        "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
      : "r"(taddr)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void tmem_st16f(uint32_t taddr, const float (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(
          taddr),
      "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]),
      "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(
          taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
      "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// this thread's shared-memory writes before the tensor cores' reads
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
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

__device__ __forceinline__ void copy_async(uint32_t dst, const void *src, bool valid) {
  const uint32_t size = valid ? 16 : 0;  // (nothing is read for 0: zeros)
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(size) : "memory");
}

// RUNS: a block's range may be longer than one accumulator takes.  (A kernel of its own: its registers cost shorter ranges 3 %.)
template <typename T, int DP, bool RUNS>
__global__ void __launch_bounds__(kWarps<T> * 32, 1) attend_many_kernel(const AttendArgs f) {
  const ClearAttentionArgs &a = f.a;
  using M = Many<DP>;
  constexpr bool SPLIT = kSplit<T>, FINE = kFine<T>;
  constexpr uint32_t SOFT_WARPS = kSoftWarps<T>, WARPS = kWarps<T>;
  constexpr uint32_t BLOCK_ROWS = SPLIT ? ROWS : 2 * ROWS;
  const auto tile_of = [](uint32_t j) { return RUNS ? j % RUN : j; };  // of a run
  extern __shared__ __align__(1024) unsigned char smem[];
  // USED: the values of tile j and the keys of tile j + 2; SFULL, PFULL: of each row tile, its two score tiles;
  // LAST, BEFORE: the products of the last tile's weights and of the one before it; FIRST: the scores of the first two
  // tiles; FREE: everything issued, after a wait that gave up
  enum : uint32_t {
    QFULL = 0,
    KFULL = 1,
    VFULL = KFULL + RING,
    USED = VFULL + RING,
    SFULL = USED + RING,
    PFULL = SFULL + 4,
    BEFORE = PFULL + 4,
    LAST = BEFORE + 2,
    FIRST = LAST + 2,
    FREE,
    BARS
  };
  __shared__ __align__(8) uint64_t bars[BARS];
  __shared__ uint32_t tmem_slot, s_fail;
  __shared__ uint32_t s_quit[TILE_WARPS];  // the meeting at which one of two softmax warps gave up
  // of the last eight tiles (the conversion is at most four ahead of a softmax), by groups of 16 positions: key
  // scales, pages out of range
  __shared__ float s_ks[8][POS / 16];
  __shared__ uint32_t s_skip[8][POS / 16];
  __shared__ float s_vr[8][POS / 16], s_above[8][POS / 16];  // value scales over sv, and what they add to scores in the running maximum
  __shared__ int32_t s_top[4];
  __shared__ float s_sv;
  // what the two threads of a row exchange; before the first tile, the power of two of each row's queries
  __shared__ float s_max[2][2 * ROWS];
  float *s_up = s_max[0];
  const uint32_t warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const uint32_t base = smem_addr(smem), bar0 = smem_addr(bars);
  const auto bar = [&](uint32_t i) { return bar0 + 8u * i; };

  // (the blocks with the most positions first)
  const uint32_t split = blockIdx.x % f.splits, own_head = blockIdx.x / f.splits % f.count, bh = f.first + own_head;
  const uint32_t kh = bh % a.heads, b = bh / a.heads, block = f.groups - 1 - blockIdx.x / f.splits / f.count;
  const uint32_t rows = a.tokens * a.group, row0 = block * BLOCK_ROWS;
  int64_t len = a.lengths[b];
  const int64_t most = static_cast<int64_t>(a.table_pitch) * a.page_tokens;
  if (len > most) {
    if (threadIdx.x == 0) atomicMax(a.err_flag, 1u);
    len = most;
  }
  // this block's range of the positions that its rows see
  const uint32_t all = group_end(a, len, min(row0 + BLOCK_ROWS, rows) - 1), share = split_share(f, all);
  const uint32_t start = split * share, end = min(all, start + share);
  const bool alone = all <= share;
  if (split > 0 && start >= all) return;
  const uint32_t n = (end - start + POS - 1) / POS;
  const uint32_t row_tiles = !SPLIT && rows - row0 > ROWS ? 2 : 1;
  const int32_t *table = a.page_table + static_cast<size_t>(b) * a.table_pitch;

  if (n == 0) {  // no row of the block has a position: zeros
    for (uint32_t i = warp; i < min(BLOCK_ROWS, rows - row0); i += WARPS) {
      const uint32_t row = row0 + i;
      T *out = static_cast<T *>(a.out) + static_cast<int64_t>(b) * a.out_strides[0] + static_cast<int64_t>(row / a.group) * a.out_strides[1] +
               static_cast<int64_t>(kh * a.group + row % a.group) * a.out_strides[2];
      for (uint32_t d = lane; d < a.dim; d += 32) out[d] = from_float<T>(0.0f);
    }
    return;
  }
  if (threadIdx.x == (WARPS - 1) * 32) {  // (of the MMA warp)
    s_fail = 0u;
    for (uint32_t i = 0; i < TILE_WARPS; ++i) s_quit[i] = 0u;
    mbar_init(bar(QFULL), SOFT_WARPS);
    for (uint32_t i = 0; i < RING; ++i) {
      mbar_init(bar(KFULL + i), 4);
      mbar_init(bar(VFULL + i), 4);
      mbar_init(bar(USED + i), 1);
    }
    for (uint32_t i = 0; i < 4; ++i) {
      mbar_init(bar(SFULL + i), 2);
      mbar_init(bar(PFULL + i), TILE_WARPS);
    }
    mbar_init(bar(FIRST), 1);
    mbar_init(bar(FREE), 1);
    for (uint32_t i = 0; i < 2; ++i) {
      mbar_init(bar(BEFORE + i), 1);
      mbar_init(bar(LAST + i), 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // What needs neither the barriers nor the tensor memory is begun before the block meets: loads of queries, copies of
  // the first tiles.
  uint32_t tmem = 0;
  const auto start_block = [&]() {
    fence_before();
    asm volatile("bar.sync 0, %0;" ::"n"(WARPS * 32) : "memory");
    fence_after();
    tmem = tmem_slot;
  };
  const auto give_up = [&]() {
    atomicExch(a.err_flag, 2u);
    atomicExch(&s_fail, 1u);
  };

  if (warp < SOFT_WARPS) {
    // row tile, half of the columns, row: two threads a row, in warps that share a quarter of tensor memory
    const uint32_t r = warp / 8, half = warp / 4 % 2, row_in = (warp % 4) * 32 + lane, row = row0 + r * ROWS + row_in;
    const uint32_t lanes = ((warp % 4) * 32u) << 16;
    // The two warps of a row meet at barrier 3 + pair.  A warp whose wait gave up meets the other once more and says
    // at which meeting, so that neither waits for one that has left.
    const uint32_t pair = r * 4 + warp % 4;
    uint32_t meetings = 0;
    const auto meet = [&](bool mine) {  // does either of the two say so?
      uint32_t any;
      asm volatile(
          "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
          : "=r"(any)
          : "r"(static_cast<uint32_t>(mine)), "r"(3 + pair)
          : "memory");
      ++meetings;
      return any != 0u;
    };
    const auto other_left = [&]() { return *const_cast<volatile uint32_t *>(&s_quit[pair]) == meetings; };
    const auto leave = [&]() {
      give_up();
      s_quit[pair] = meetings + 1;
      meet(false);
    };
    // ---- the warp's 16 queries, each brought to [1, 2) by a power of two, as f16: eight rows x four chunks of
    // eight dimensions at a time ----
    const uint32_t qr = lane % 8, qc = lane / 8;
    const bool wide_q = (reinterpret_cast<uintptr_t>(a.q) | static_cast<uintptr_t>((a.q_strides[0] | a.q_strides[1] | a.q_strides[2]) * sizeof(T))) % 16 == 0;
    if constexpr (SPLIT) {
      start_block();
#pragma unroll 1
      for (uint32_t g = 0; g < 2; ++g) {
        const uint32_t in_tile = warp * 16 + g * 8 + qr, rw = row0 + in_tile;
        const T *q = static_cast<const T *>(a.q) + static_cast<int64_t>(b) * a.q_strides[0] +
                     static_cast<int64_t>(rw / a.group) * a.q_strides[1] + static_cast<int64_t>(kh * a.group + rw % a.group) * a.q_strides[2];
        float x[DP / 32][8], top = 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < DP / 32; ++i) {
          const uint32_t d = (qc + 4 * i) * 8;
          const bool in = rw < rows && d < a.dim;  // (dim is a multiple of 16)
          float4 y[2] = {};
          if (in && wide_q) {
            y[0] = *reinterpret_cast<const float4 *>(q + d);
            y[1] = *reinterpret_cast<const float4 *>(q + d + 4);
          } else if (in) {
            y[0] = make_float4(to_float(q[d]), to_float(q[d + 1]), to_float(q[d + 2]), to_float(q[d + 3]));
            y[1] = make_float4(to_float(q[d + 4]), to_float(q[d + 5]), to_float(q[d + 6]), to_float(q[d + 7]));
          }
          x[i][0] = y[0].x, x[i][1] = y[0].y, x[i][2] = y[0].z, x[i][3] = y[0].w;
          x[i][4] = y[1].x, x[i][5] = y[1].y, x[i][6] = y[1].z, x[i][7] = y[1].w;
#pragma unroll
          for (uint32_t e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[i][e]));
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
        const int ex = min(max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -126), 126);
        const float down = copysignf(__int_as_float((127 - ex) << 23), a.softmax_scale);
        if (qc == 0) s_up[in_tile] = __int_as_float((127 + ex) << 23);
#pragma unroll
        for (uint32_t i = 0; i < DP / 32; ++i) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (uint32_t e = 0; e < 4; ++e) {
            const float u = x[i][2 * e] * down, v = x[i][2 * e + 1] * down;
            const __half2 h = __floats2half2_rn(u, v);
            hi[e] = half2_bits(h);
            lo[e] = half2_bits(__floats2half2_rn(u - __low2float(h), v - __high2float(h)));
          }
          unsigned char *dst = smem + (in_tile >> 3) * (DP * 16) + (qc + 4 * i) * 128 + qr * 16;
          *reinterpret_cast<uint4 *>(dst) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4 *>(dst + M::Q_TILE) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
      }
    } else {
      uint4 raw[2][DP / 32];
#pragma unroll
      for (uint32_t g = 0; g < 2; ++g) {
        const uint32_t rw = row0 + r * ROWS + (warp % 8) * 16 + g * 8 + qr;
        const T *q = static_cast<const T *>(a.q) + static_cast<int64_t>(b) * a.q_strides[0] +
                     static_cast<int64_t>(rw / a.group) * a.q_strides[1] + static_cast<int64_t>(kh * a.group + rw % a.group) * a.q_strides[2];
#pragma unroll
        for (uint32_t i = 0; i < DP / 32; ++i) {
          const uint32_t d = (qc + 4 * i) * 8;
          raw[g][i] = make_uint4(0u, 0u, 0u, 0u);
          if (rw >= rows || d >= a.dim) continue;  // (dim is a multiple of 16)
          if (wide_q) {
            raw[g][i] = *reinterpret_cast<const uint4 *>(q + d);
          } else {
            const auto two = [&](uint32_t e) {
              const T lo = q[d + e], hi = q[d + e + 1];
              return static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(&lo)) |
                     static_cast<uint32_t>(*reinterpret_cast<const uint16_t *>(&hi)) << 16;
            };
            raw[g][i] = make_uint4(two(0), two(2), two(4), two(6));
          }
        }
      }
      start_block();
#pragma unroll
      for (uint32_t g = 0; g < 2; ++g) {
        const uint32_t in_tile = (warp % 8) * 16 + g * 8 + qr;
        float x[DP / 32][8], top = 0.0f;
#pragma unroll
        for (uint32_t i = 0; i < DP / 32; ++i) {
          const T *el = reinterpret_cast<const T *>(&raw[g][i]);
#pragma unroll
          for (uint32_t e = 0; e < 8; ++e) {
            x[i][e] = to_float(el[e]);
            top = fmaxf(top, fabsf(x[i][e]));
          }
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
        const int ex = min(max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -126), 126);
        const float down = copysignf(__int_as_float((127 - ex) << 23), a.softmax_scale);
        if (qc == 0) s_up[r * ROWS + in_tile] = __int_as_float((127 + ex) << 23);
#pragma unroll
        for (uint32_t i = 0; i < DP / 32; ++i) {
          uint32_t w[4];
#pragma unroll
          for (uint32_t e = 0; e < 4; ++e) w[e] = half2_bits(__floats2half2_rn(x[i][2 * e] * down, x[i][2 * e + 1] * down));
          *reinterpret_cast<uint4 *>(smem + r * M::Q_TILE + (in_tile >> 3) * (DP * 16) + (qc + 4 * i) * 128 + qr * 16) =
              make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
    }
    fence_async();
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(QFULL));
    asm volatile("bar.sync %0, 256;" ::"r"(11 + r) : "memory");  // s_up of the row tile
    const float factor = s_up[r * ROWS + row_in] * (fabsf(a.softmax_scale) * kLog2e);
    const int32_t last = row < rows ? static_cast<int32_t>(len - a.tokens + row / a.group) : -1;
    const uint32_t o_col = tmem + lanes + M::O_COL + r * DP + half * (DP / 2);
    // (SPLIT: behind O the products of the weights' second halves, in the other row tile's place of the scores the sum of the
    // tiles up to the last fold)
    const uint32_t sum_col = tmem + lanes + 2 * POS + half * (DP / 2);
    const auto read_all = [&](uint32_t c, bool folded, float (&o)[16]) {
      float fine[16], before[16];
      tmem_ld16f(o_col + c, o);
      if constexpr (SPLIT) {
        tmem_ld16f(o_col + DP + c, fine);
        if (folded) tmem_ld16f(sum_col + c, before);
      }
      tmem_wait_ld();
      if constexpr (SPLIT) {
#pragma unroll
        for (uint32_t e = 0; e < 16; ++e) o[e] += folded ? fine[e] + before[e] : fine[e];
      }
    };
    constexpr uint32_t COLS = POS / 2;
    float m = neg_inf(), l = 0.0f;
    const size_t at = (static_cast<size_t>(own_head) * f.splits + split) * rows + row;
    // the runs before this one, as of the maximum then
    float run_m = neg_inf(), run_l = 0.0f;
    const auto run_fade = [&]() { return run_m == neg_inf() ? 0.0f : ex2(run_m - m); };
    const auto add_runs = [&](uint32_t c, float fade, float (&o)[16]) {
      const uint32_t d0 = half * (DP / 2) + c;
      if (row >= rows || d0 >= a.dim) return;  // (dim is a multiple of 16)
      const float4 *from = reinterpret_cast<const float4 *>(f.part + at * a.dim + d0);
#pragma unroll
      for (uint32_t e = 0; e < 16; e += 4) {
        const float4 x = from[e / 4];
        o[e] += fade * x.x, o[e + 1] += fade * x.y, o[e + 2] += fade * x.z, o[e + 3] += fade * x.w;
      }
    };
    if (r < row_tiles) {
      for (uint32_t j = 0; j < n; ++j) {
        const uint32_t buf = j % 8, two = r * 2 + j % 2, s_tile = tmem + lanes + two * POS;
        if (!__all_sync(0xffffffffu, wait_quick(bar(SFULL + two), (j / 2) & 1u))) {
          leave();
          goto done;
        }
        fence_after();
        float v[COLS];
        tmem_ld32(s_tile + half * COLS, v);
        // (the same for the warp)
        const uint32_t first = start + j * POS + half * COLS;  // this half's first position
        const bool part = __any_sync(0xffffffffu, (s_skip[buf][half * 2] | s_skip[buf][half * 2 + 1]) != 0 ||
                                                      static_cast<int32_t>(first + COLS - 1) > last);
        float kf[2] = {s_ks[buf][half * 2] * factor, s_ks[buf][half * 2 + 1] * factor};
        const float above[2] = {s_above[buf][half * 2], s_above[buf][half * 2 + 1]};
        tmem_wait_ld();
        float top = neg_inf();
        if (part) {
#pragma unroll
          for (uint32_t i = 0; i < 2; ++i) {
            const bool out = s_skip[buf][half * 2 + i] != 0;
            float t = neg_inf();
#pragma unroll
            for (uint32_t e = 0; e < 16; ++e) {
              const bool in = static_cast<int32_t>(first + i * 16 + e) <= last && !out;
              v[i * 16 + e] = in ? v[i * 16 + e] * kf[i] : neg_inf();
              t = fmaxf(t, v[i * 16 + e]);
            }
            top = fmaxf(top, t + above[i]);
            kf[i] = 1.0f;
          }
        } else {
#pragma unroll
          for (uint32_t i = 0; i < 2; ++i) {
            const float *x = v + i * 16;
            const float t = max3(max3(x[0], x[1], x[2]), max3(x[3], x[4], x[5]), max3(x[6], x[7], x[8]));
            top = fmaxf(top, fmaf(max3(t, max3(x[9], x[10], x[11]), max3(fmaxf(x[12], x[13]), x[14], x[15])), kf[i], above[i]));
          }
        }
        // the two warps agree to raise; both have read their scores by then, so that the weights may overwrite them
        const bool raise = meet(top > m + kRaise);
        if (other_left()) goto done;
        const bool fold = SPLIT && j > 0 && j % FOLD == 0, run = RUNS && j > 0 && j % RUN == 0;
        float keep = 1.0f;
        if (raise) {
          s_max[half][r * ROWS + row_in] = top;
          meet(false);
          if (other_left()) goto done;
          const float raised = fmaxf(fmaxf(m, top), s_max[half ^ 1u][r * ROWS + row_in]);
          keep = m == neg_inf() ? 0.0f : ex2(m - raised);
          m = raised;
          l *= keep;
        }
        const float off = kLift - (m == neg_inf() ? 0.0f : m);
        const uint64_t off2 = pair_of(off, off), kf2[2] = {pair_of(kf[0], kf[0]), pair_of(kf[1], kf[1])};
        uint64_t sum[2] = {};
        uint32_t w[16], rest[16];
#pragma unroll
        for (uint32_t e = 0; e < COLS; e += 2) {
          const float2 x = floats_of(fma2(pair_of(v[e], v[e + 1]), kf2[e / 16], off2));
          float p0 = ex2(x.x), p1 = ex2(x.y);
          sum[e / 2 % 2] = add2(sum[e / 2 % 2], pair_of(p0, p1));
          const float vr = s_vr[buf][half * 2 + e / 16];
          if constexpr (FINE) {  // (2 - 3 % faster than both in one instruction; 2 % slower for bfloat16)
            p0 *= vr;
            p1 *= vr;
          } else {
            const float2 p = floats_of(mul2(pair_of(p0, p1), pair_of(vr, vr)));
            p0 = p.x;
            p1 = p.y;
          }
          const __half2 h = __floats2half2_rn(p0, p1);
          w[e / 2] = half2_bits(h);
          if constexpr (FINE) rest[e / 2] = half2_bits(__floats2half2_rn(p0 - __low2float(h), p1 - __high2float(h)));
        }
        tmem_st16(s_tile + half * (COLS / 2), w);
        if constexpr (FINE) tmem_st16(s_tile + POS / 2 + half * (COLS / 2), rest);
        const float2 added = floats_of(add2(sum[0], sum[1]));
        l += added.x + added.y;
        if (j > 0 && (raise || fold || run)) {
          // O with the weights of tile j - 1: done before the scores of tile j + 1, where there is one
          const uint32_t next = r * 2 + (j + 1) % 2;
          if (!__all_sync(0xffffffffu, j + 1 < n ? wait_quick(bar(SFULL + next), ((j + 1) / 2) & 1u) : wait_quick(bar(BEFORE + r), 0))) {
            leave();
            goto done;
          }
          fence_after();
          const float fade = run ? run_fade() : 0.0f;
#pragma unroll 1
          for (uint32_t c = 0; c < DP / 2; c += 16) {
            float o[16];
            if (run) {  // (the next products begin anew)
              read_all(c, true, o);
#pragma unroll
              for (uint32_t e = 0; e < 16; ++e) o[e] *= keep;
              if (j > RUN) add_runs(c, fade, o);
              const uint32_t d0 = half * (DP / 2) + c;
              if (row < rows && d0 < a.dim) {
                float4 *to = reinterpret_cast<float4 *>(f.part + at * a.dim + d0);
#pragma unroll
                for (uint32_t e = 0; e < 16; e += 4) to[e / 4] = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
              }
              continue;
            }
            if (fold) {
              read_all(c, tile_of(j) > FOLD, o);
            } else {
              tmem_ld16f(o_col + c, o);
              tmem_wait_ld();
            }
#pragma unroll
            for (uint32_t e = 0; e < 16; ++e) o[e] *= keep;
            tmem_st16f((fold ? sum_col : o_col) + c, o);
            if (SPLIT && !fold) {
              tmem_ld16f(o_col + DP + c, o);
              tmem_wait_ld();
#pragma unroll
              for (uint32_t e = 0; e < 16; ++e) o[e] *= keep;
              tmem_st16f(o_col + DP + c, o);
              if (tile_of(j) > FOLD) {
                tmem_ld16f(sum_col + c, o);
                tmem_wait_ld();
#pragma unroll
                for (uint32_t e = 0; e < 16; ++e) o[e] *= keep;
                tmem_st16f(sum_col + c, o);
              }
            }
          }
        }
        tmem_wait_st();
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(PFULL + two));
        if (run) {
          // (l holds this tile's weights already: a tile more or less in a run's sum)
          run_l = run_l * run_fade() + l;
          run_m = m;
          l = 0.0f;
        }
      }
      if (!__all_sync(0xffffffffu, wait_quick(bar(LAST + r), 0))) {
        leave();
        goto done;
      }
      fence_after();
      const bool runs = RUNS && n > RUN;
      const float fade = runs ? run_fade() : 0.0f;
      if (runs) l += run_l * fade;
      s_max[half][r * ROWS + row_in] = l;
      meet(false);
      if (other_left()) goto done;
      l += s_max[half ^ 1u][r * ROWS + row_in];
      T *out = static_cast<T *>(a.out) + static_cast<int64_t>(b) * a.out_strides[0] + static_cast<int64_t>(row / a.group) * a.out_strides[1] +
               static_cast<int64_t>(kh * a.group + row % a.group) * a.out_strides[2];
      const bool wide = (reinterpret_cast<uintptr_t>(a.out) | static_cast<uintptr_t>((a.out_strides[0] | a.out_strides[1] | a.out_strides[2]) * sizeof(T))) % 16 == 0;
      // (O and l are both lifted; partial results are not)
      const float scale = alone ? 1.0f / l : 0.0078125f, sv = s_sv;  // (sv apart: a power of two that may be tiny)
      if (!alone && row < rows && half == 0) f.stats[at] = make_float2(l * 0.0078125f, m);
      // The warp's rows go out through shared memory (the queries' place: their products are done), so that a store writes
      // whole lines (16 bytes of 32 rows at a time: 5 % longer at 4 x 1024 queries, single precision 6 %).
      const auto write_rows = [&](auto type, decltype(type) *to) {  // (to: this thread's row)
        using E = decltype(type);
        constexpr uint32_t PASS = DP / sizeof(E), PIECE = 16 / sizeof(E), PIECES = DP / 16;  // (an eighth of a tile)
        const uint32_t key = PIECES == 8 ? lane % 8 : lane / 2 % 4;
        unsigned char *stage = smem + r * M::Q_TILE + warp % 8 * (M::Q_TILE / 8);
#pragma unroll 1
        for (uint32_t c = 0; c < DP / 2; c += PASS) {
#pragma unroll
          for (uint32_t h = 0; h < PASS; h += 16) {
            float o[16];
            read_all(c + h, tile_of(n - 1) >= FOLD, o);
            if (runs) add_runs(c + h, fade, o);
#pragma unroll
            for (uint32_t e = 0; e < 16; e += PIECE) {
              alignas(16) E x[PIECE];
#pragma unroll
              for (uint32_t i = 0; i < PIECE; ++i) x[i] = from_float<E>(l == 0.0f ? 0.0f : o[e + i] * scale * sv);
              *reinterpret_cast<uint4 *>(stage + lane * (PIECES * 16) + (((h + e) / PIECE) ^ key) * 16) = *reinterpret_cast<const uint4 *>(x);
            }
          }
          __syncwarp();
#pragma unroll
          for (uint32_t i = 0; i < PIECES; ++i) {
            const uint32_t of = (i * 32 + lane) / PIECES, piece = lane % PIECES, at_key = PIECES == 8 ? of % 8 : of / 2 % 4;
            const uint4 x = *reinterpret_cast<const uint4 *>(stage + of * (PIECES * 16) + (piece ^ at_key) * 16);
            E *dst = reinterpret_cast<E *>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(to), of));
            const uint32_t d = half * (DP / 2) + c + piece * PIECE;
            if (row - lane + of < rows && d < a.dim) *reinterpret_cast<uint4 *>(dst + d) = x;  // (dim is a multiple of 16)
          }
          __syncwarp();
        }
      };
      if (!alone) {
        write_rows(0.0f, f.part + at * a.dim);
      } else if (wide) {
        write_rows(T(), out);
      } else {
#pragma unroll 1
        for (uint32_t c = 0; c < DP / 2; c += 16) {
          float o[16];
          read_all(c, tile_of(n - 1) >= FOLD, o);
          if (runs) add_runs(c, fade, o);
          const uint32_t d0 = half * (DP / 2) + c;
          if (row >= rows || d0 >= a.dim) continue;
#pragma unroll
          for (uint32_t e = 0; e < 16; ++e) out[d0 + e] = from_float<T>(l == 0.0f ? 0.0f : o[e] * scale * sv);
        }
      }
    }
  } else if (warp < SOFT_WARPS + CONVERT_WARPS) {
    // ---- keys (four warps) and values (four) to f16: a warp 16 positions of each tile, in one page ----
    const uint32_t w = warp % 4;
    const bool keys = warp < SOFT_WARPS + 4;
    // the tiles to copy next: their pages, loaded a ring ahead; of the first, the page's slot in the list and the first row in it
    const uint32_t slots = POS / a.page_tokens, more = POS % a.page_tokens, slots_end = (end + a.page_tokens - 1) / a.page_tokens;
    uint32_t slot = (start + w * 16) / a.page_tokens, row = (start + w * 16) % a.page_tokens;
    uint32_t ahead_slot = slot, ahead_row = row;
    const auto next = [&](uint32_t &at_slot, uint32_t &at_row) {
      at_slot += slots;
      at_row += more;
      if (at_row >= a.page_tokens) {
        at_row -= a.page_tokens;
        ++at_slot;
      }
    };
    int32_t pages[STAGED];
#pragma unroll
    for (uint32_t i = 0; i < STAGED; ++i) {
      pages[i] = ahead_slot < slots_end ? table[ahead_slot] : -1;
      next(ahead_slot, ahead_row);
    }
    const int8_t *cache = (keys ? a.k_cache : a.v_cache) + static_cast<int64_t>(kh) * a.cache_strides[1];
    const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));  // 1152
    // of the tiles copied: scales, and whether the page is out of range
    float ks[STAGED] = {}, vs[STAGED] = {};
    bool skip[STAGED] = {};
    // a warp's share of a staged tile: keys [row of 8][chunk of 16 bytes] by the lane that reads them, values row by row
    const uint32_t raw_at = M::RAW_AT + (keys ? 0 : M::RAW) + w * (16 * DP);
    const uint32_t kr = lane % 8, kc = lane / 8;  // a key row of 8, a chunk of four
    const auto copy = [&](uint32_t st) {          // (st: a constant)
      const int32_t page = pages[st];
      const bool in = page >= 0 && static_cast<uint32_t>(page) < a.pages;
      skip[st] = slot < slots_end && !in;
      const size_t sc = in ? static_cast<size_t>(page) * a.heads + kh : 0;
      ks[st] = in && keys ? a.k_scale[sc] : 0.0f;
      vs[st] = in && keys ? a.v_scale[sc] : 0.0f;
      const int8_t *src = cache + (in ? page * a.cache_strides[0] + static_cast<int64_t>(row) * a.cache_strides[2] : 0);
      const uint32_t dst = base + raw_at + st * (2 * M::RAW) + lane * 16;
#pragma unroll
      for (uint32_t i = 0; i < DP / 32; ++i) {
        const uint32_t piece = i * 32 + lane;
        const uint32_t r = keys ? i / (DP / 64) * 8 + kr : piece / (DP / 16);
        const uint32_t d = keys ? (kc + 4 * (i % (DP / 64))) * 16 : piece % (DP / 16) * 16;
        const bool ok = in && d < a.dim;
        copy_async(dst + i * 512, ok ? src + r * a.cache_strides[2] + d : cache, ok);
      }
      next(slot, row);
      pages[st] = ahead_slot < slots_end ? table[ahead_slot] : -1;
      next(ahead_slot, ahead_row);
    };
#pragma unroll
    for (uint32_t i = 0; i + 1 < STAGED; ++i) {
      if (i < n) copy(i);
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    start_block();
    // the largest value scale of the pages in the range: by the values' warps, which are not the first to be waited for
    if (!keys) {
      int32_t most = kNoScale;
      for (uint32_t p = start / a.page_tokens + threadIdx.x % 128; p < slots_end; p += 128) {
        const int32_t id = table[p];
        if (id >= 0 && static_cast<uint32_t>(id) < a.pages)
          most = max(most, scale_exponent(a.v_scale[static_cast<size_t>(id) * a.heads + kh]));
        else
          atomicMax(a.err_flag, 1u);
      }
      most = __reduce_max_sync(0xffffffffu, most);
      if (lane == 0) s_top[w] = most;
      asm volatile("bar.arrive 1, 256;" ::: "memory");
    }
    int32_t unit = 0;  // of sv
    float per_sv = 1.0f;
    uint32_t buf = 0;
    if (keys) {
      for (uint32_t j0 = 0; j0 < n; j0 += STAGED) {
#pragma unroll
        for (uint32_t st = 0; st < STAGED; ++st) {
          const uint32_t j = j0 + st;
          if (j >= n) break;
          asm volatile("cp.async.wait_group %0;" ::"n"(STAGED - 2) : "memory");
          const unsigned char *src = smem + raw_at + st * (2 * M::RAW) + lane * 16;
          uint4 k[DP / 32];
#pragma unroll
          for (uint32_t i = 0; i < DP / 32; ++i) k[i] = *reinterpret_cast<const uint4 *>(src + i * 512);
          // the keys that lay here were tile j - 3's, used with tile j - 5's values, or among the first two
          if (j >= RING && !__all_sync(0xffffffffu, j >= 5 ? wait_quick(bar(USED + (j - 5) % RING), ((j - 5) / RING) & 1u)
                                                           : wait_quick(bar(FIRST), 0))) {
            give_up();
            goto done;
          }
          // 1024 + (k + 128) by byte permute, times the scale's sign, minus 1152 times it
          const __half2 sg = bits_half2(ks[st] < 0.0f ? 0xbc00bc00u : 0x3c003c00u), so = __hneg2(__hmul2(sg, off));
          unsigned char *kt = smem + M::K_AT + buf * M::K_TILE + w * 2 * (DP * 16) + kc * 256 + kr * 16;
#pragma unroll
          for (uint32_t i = 0; i < DP / 32; ++i) {
            const uint32_t x[4] = {k[i].x, k[i].y, k[i].z, k[i].w};
            uint32_t o[8];
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e) {
              const uint32_t u = x[e] ^ 0x80808080u;
              o[2 * e] = half2_bits(__hfma2(bits_half2(__byte_perm(u, 0x64646464u, 0x4140)), sg, so));
              o[2 * e + 1] = half2_bits(__hfma2(bits_half2(__byte_perm(u, 0x64646464u, 0x4342)), sg, so));
            }
            unsigned char *dst = kt + i / (DP / 64) * (DP * 16) + i % (DP / 64) * 1024;
            *reinterpret_cast<uint4 *>(dst) = make_uint4(o[0], o[1], o[2], o[3]);
            *reinterpret_cast<uint4 *>(dst + 128) = make_uint4(o[4], o[5], o[6], o[7]);
          }
          if (j == 0) {  // (the values' warps have seen the scales)
            asm volatile("bar.sync 1, 256;" ::: "memory");
            unit = scale_unit(max(max(s_top[0], s_top[1]), max(s_top[2], s_top[3])));
            per_sv = scalbnf(1.0f, -unit);
            if (w == 0 && lane == 0) s_sv = scalbnf(1.0f, unit);
          }
          if (lane == 0) {
            // (a value scale that is a NaN or an infinity: no number)
            const bool number = fabsf(vs[st]) < -neg_inf();
            s_ks[j % 8][w] = number ? fabsf(ks[st]) : __int_as_float(0x7fc00000);
            s_skip[j % 8][w] = skip[st];
            s_vr[j % 8][w] = number ? vs[st] * per_sv : 0.0f;
            s_above[j % 8][w] = number ? scale_above(vs[st], unit) : 0.0f;
          }
          fence_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(KFULL + buf));
          if (++buf == RING) buf = 0;
          // into the place read in the round before this one
          if (j + STAGED - 1 < n) copy((st + STAGED - 1) % STAGED);
          asm volatile("cp.async.commit_group;" ::: "memory");
        }
      }
    } else {
      constexpr uint32_t VG = DP == 128 ? 2 : 1;  // groups of 8 positions that a lane takes in turn
      const uint32_t quad = lane % (DP / 4), vsub = DP == 128 ? 0 : lane / 16;
      // A lane transposes four dimensions of eight positions, rotated by its place so that the eight lanes of a store
      // phase write the eight rows of a core matrix: dimension (e + turn) % 4 of its four in round e.
      const uint32_t turn = lane / 2 % 4;
      const uint32_t sel_a = turn == 0 ? 0x5140u : turn == 1 ? 0x6251u : turn == 2 ? 0x7362u : 0x4073u;
      const uint32_t sel_b = turn == 0 ? 0x7362u : turn == 1 ? 0x4073u : turn == 2 ? 0x5140u : 0x6251u;
      for (uint32_t j0 = 0; j0 < n; j0 += STAGED) {
#pragma unroll
        for (uint32_t st = 0; st < STAGED; ++st) {
          const uint32_t j = j0 + st;
          if (j >= n) break;
          asm volatile("cp.async.wait_group %0;" ::"n"(STAGED - 2) : "memory");
          __syncwarp();
          const unsigned char *src = smem + raw_at + st * (2 * M::RAW) + quad * 4;
          uint32_t x[VG][8];
#pragma unroll
          for (uint32_t g = 0; g < VG; ++g)
#pragma unroll
            for (uint32_t p = 0; p < 8; ++p) x[g][p] = *reinterpret_cast<const uint32_t *>(src + ((g + vsub) * 8 + p) * DP) ^ 0x80808080u;
          if (j >= RING && !__all_sync(0xffffffffu, wait_quick(bar(USED + buf), ((j - RING) / RING) & 1u))) {
            give_up();
            goto done;
          }
          unsigned char *vt = smem + M::V_AT + buf * M::V_TILE + (quad >> 1) * V_GROUP + (w * 2 + vsub) * 128 + (quad & 1u) * 64;
#pragma unroll
          for (uint32_t g = 0; g < VG; ++g) {
            uint32_t o[4][4];  // [round][pair of positions]
#pragma unroll
            for (uint32_t p = 0; p < 4; ++p) {
              const uint32_t t0 = __byte_perm(x[g][2 * p], x[g][2 * p + 1], sel_a), t1 = __byte_perm(x[g][2 * p], x[g][2 * p + 1], sel_b);
#pragma unroll
              for (uint32_t e = 0; e < 4; ++e) {
                const __half2 v = __hsub2(bits_half2(__byte_perm(e < 2 ? t0 : t1, 0x64646464u, e % 2 ? 0x4342 : 0x4140)), off);
                o[e][p] = half2_bits(v);
              }
            }
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e)
              *reinterpret_cast<uint4 *>(vt + g * 128 + (e + turn) % 4 * 16) = make_uint4(o[e][0], o[e][1], o[e][2], o[e][3]);
          }
          fence_async();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(VFULL + buf));
          if (++buf == RING) buf = 0;
          // into the place read in the round before this one (all lanes have passed a barrier since)
          if (j + STAGED - 1 < n) copy((st + STAGED - 1) % STAGED);
          asm volatile("cp.async.commit_group;" ::: "memory");
        }
      }
    }
  } else {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    start_block();
    // ---- products ----
    const uint32_t elect = elected();
    const auto ready = [&](uint32_t i, uint32_t parity) { return __all_sync(0xffffffffu, wait_quick(bar(i), parity)); };
    const auto scores = [&](uint32_t r, uint32_t j, uint32_t kbuf) {
      const uint32_t two = r * 2 + j % 2;
      const uint64_t qd = desc_of(base + r * M::Q_TILE, DP * 16), kd = desc_of(base + M::K_AT + kbuf * M::K_TILE, DP * 16);
      if constexpr (SPLIT) {  // (the small products first: less is cut off)
        const uint64_t rest = desc_of(base + M::Q_TILE, DP * 16);
#pragma unroll
        for (uint32_t k = 0; k < DP / 16; ++k) mma_ss(tmem + two * POS, rest + k * 16u, kd + k * 16u, idesc(POS), k != 0, elect);
      }
#pragma unroll
      for (uint32_t k = 0; k < DP / 16; ++k)  // 256 bytes on: 16 in the descriptor's units
        mma_ss(tmem + two * POS, qd + k * 16u, kd + k * 16u, idesc(POS), SPLIT || k != 0, elect);
      if (elect) mbar_arrive(bar(SFULL + two));  // (also passes on the page scales that came with the keys)
      commit(bar(SFULL + two), elect);
    };
    if (!ready(QFULL, 0)) {
      give_up();
      goto done;
    }
    for (uint32_t j = 0; j < 2 && j < n; ++j) {
      if (!ready(KFULL + j, 0)) {
        give_up();
        goto done;
      }
      fence_after();
      for (uint32_t r = 0; r < row_tiles; ++r) scores(r, j, j);
    }
    commit(bar(FIRST), elect);
    uint32_t vbuf = 0, kbuf = 2, vpar = 0, kpar = 0;
    for (uint32_t j = 0; j < n; ++j) {
      if (!ready(VFULL + vbuf, vpar) || (j + 2 < n && !ready(KFULL + kbuf, kpar))) {
        give_up();
        goto done;
      }
      const uint64_t vd = desc_of(base + M::V_AT + vbuf * M::V_TILE, V_GROUP);
#pragma unroll
      for (uint32_t r = 0; r < 2; ++r) {
        if (r >= row_tiles) break;
        const uint32_t two = r * 2 + j % 2;
        if (!ready(PFULL + two, (j / 2) & 1u)) {
          give_up();
          goto done;
        }
        fence_after();
#pragma unroll
        for (uint32_t k = 0; k < POS / 16; ++k)
          mma_ts(tmem + M::O_COL + r * DP, tmem + two * POS + k * 8u, vd + k * 16u, idesc(DP), ((SPLIT ? j % FOLD : tile_of(j)) | k) != 0, elect);
        if constexpr (FINE) {
#pragma unroll
          for (uint32_t k = 0; k < POS / 16; ++k)
            mma_ts(tmem + M::O_COL + (SPLIT ? DP : r * DP), tmem + two * POS + POS / 2 + k * 8u, vd + k * 16u, idesc(DP), !SPLIT || (j % FOLD | k) != 0,
                     elect);
        }
        if (j + 2 < n)
          scores(r, j + 2, kbuf);
        else
          commit(bar((j + 1 == n ? LAST : BEFORE) + r), elect);
      }
      commit(bar(USED + vbuf), elect);
      if (++vbuf == RING) {
        vbuf = 0;
        vpar ^= 1u;
      }
      if (++kbuf == RING) {
        kbuf = 0;
        kpar ^= 1u;
      }
    }
    // no commit arrives after the block's end: each barrier's last one (the softmax waits for SFULL)
    bool ok = ready(FIRST, 0);
    for (uint32_t j = n > RING ? n - RING : 0; j < n; ++j) ok = ready(USED + j % RING, (j / RING) & 1u) && ok;
    for (uint32_t r = 0; r < row_tiles; ++r) ok = ready(LAST + r, 0) && (n == 1 || ready(BEFORE + r, 0)) && ok;
    if (!ok) give_up();
  }
done:
  __syncwarp();
  // (also of warps that gave up: copies into shared memory and stores to tensor memory end before either is released)
  asm volatile("cp.async.wait_all;" ::: "memory");
  tmem_wait_st();
  fence_before();
  __syncthreads();
  if (s_fail != 0u) {
    // what was issued ends by itself: the tensor memory is freed after it (a block that kept it would end in an error of
    // the whole context), and only where this wait too gives up it stays allocated
    if (warp == SOFT_WARPS + CONVERT_WARPS) {
      commit(bar(FREE), elected());
      if (!__all_sync(0xffffffffu, mbar_wait(bar(FREE), 0)) && lane == 0) atomicExch(&s_fail, 2u);
    }
    __syncthreads();
  }
  if (warp == SOFT_WARPS + CONVERT_WARPS && s_fail != 2u)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
}

uint32_t block_rows_of(int type) { return type == kOutF32 ? ROWS : 2 * ROWS; }

// Splits where the blocks do not fill the SMs: as many as do, of 512 positions at least.  float16 and single precision under lists
// too long for one accumulator are also split where that fills the last round of blocks better (2 x 2048 queries at 65536
// positions, float16 4.8 ms with two against 5.5), but no further: splits that turn out empty cost a third of a short context
// (1 x 1024 at 1024 positions under lists for 131072, bfloat16 46 us with four against 29; 8 x 2048 at 2048, float16 0.97 ms against
// 0.45).
AttendArgs many_args(const ClearAttentionArgs &a, int type, void *work, uint32_t sms) {
  AttendArgs f{a, nullptr, nullptr, 0, 0, 1, 1, 512, false};
  const uint32_t block = block_rows_of(type);
  f.groups = (a.tokens * a.group + block - 1) / block;
  const uint64_t blocks = static_cast<uint64_t>(a.batch) * a.heads * f.groups, most = static_cast<uint64_t>(a.table_pitch) * a.page_tokens;
  const uint64_t want = sms / blocks, longest = (most + 511) / 512;
  f.splits = static_cast<uint32_t>(want < longest ? want : longest);
  if (f.splits < 1) f.splits = 1;
  if (type != kOutBf16) {
    const auto rounds = [&](uint64_t splits) { return (blocks * splits + sms - 1) / sms; };
    const uint64_t long_lists = (most + kMostPositions - 1) / kMostPositions, room = 8ull * sms / blocks;
    for (uint32_t n = f.splits + 1; n <= long_lists && n <= room; ++n)
      if (rounds(n) * f.splits * 10 < rounds(f.splits) * n * 9) f.splits = n;
  }
  f.runs = most > static_cast<uint64_t>(f.splits) * kMostPositions;
  attend_place(&f, work);
  return f;
}

template <typename T, int DP>
cudaError_t launch(const AttendArgs &f, cudaStream_t s) {
  auto kern = f.runs ? attend_many_kernel<T, DP, true> : attend_many_kernel<T, DP, false>;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(Many<DP>::SMEM));
  if (e != cudaSuccess) return e;
  kern<<<f.count * f.groups * f.splits, kWarps<T> * 32, Many<DP>::SMEM, s>>>(f);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch(const AttendArgs &f, cudaStream_t s) {
  return f.a.dim <= 64 ? launch<T, 64>(f, s) : launch<T, 128>(f, s);
}

}  // namespace

// From 48 rows a cached head on: the other kernel takes 16 at a time (0.65 us an SM for 64 positions), this one 256 in 1.4 us
// (128 of single precision).
bool attend_many_takes(const ClearAttentionArgs &a) {
  return a.dim <= 128 && static_cast<uint64_t>(a.tokens) * a.group >= 48 && attend_few_takes(a);
}

size_t attend_many_bytes(const ClearAttentionArgs &a, int type, uint32_t sms) { return attend_part_bytes(many_args(a, type, nullptr, sms)); }

cudaError_t launch_clear_attention_many(const ClearAttentionArgs &a, int type, void *work, uint32_t sms, cudaStream_t s) {
  return attend_each(many_args(a, type, work, sms), [&](const AttendArgs &f) {
    const cudaError_t e = type == kOutF32 ? launch<float>(f, s) : type == kOutF16 ? launch<__half>(f, s) : launch<__nv_bfloat16>(f, s);
    return e != cudaSuccess || f.splits == 1 ? e : launch_attend_join(f, type, block_rows_of(type), s);
  });
}

}  // namespace rosetta
