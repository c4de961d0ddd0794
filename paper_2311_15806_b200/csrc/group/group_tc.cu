// Products of a 4-bit layer with group scales with many rows, on the tensor cores (pipe_group_linear, pipe_expert_linear).
//
// The weights are the A operand: a tile is 128 output channels per CTA (256 over a pair of SMs, cta_group::2) by TN rows of
// activations.  A thread owns one output channel, reads the 128 codes of a stage (four runs of 16 bytes), subtracts the zero point
// exactly and multiplies by the scale -- one rounding to the layer's type, the type that the MMA takes its operands in; it costs a
// product what the rounding of the activations costs it.  Where the widened weights go depends on the tile's width:
//   TN = 256 (a pair's) has 1024 cycles of products per stage, and its two accumulators take all of tensor memory; the weights go to
//     shared memory, 128-byte swizzled, by two groups of four warps
//   TN <= 128 has half of that or less, and its 112 KB of shared-memory traffic a stage would be the bound; there the weights go to
//     tensor memory, which tcgen05.mma takes A from as well: four slots of 64 columns behind the two accumulators, one to each of four
//     groups of warps
// Activations come by tensor copies in the 128-byte swizzle, a stage's codes by one more, each on a ring.  Rows that are gathered come by
// 16-byte asynchronous copies of two warps (a tensor copy that gathers four rows takes some 75 cycles of an SM, 64 of them a stage).
// The fence that makes ordinary writes visible to the tensor core waits for everything the thread has in flight, so gathered rows
// are fenced by the warp that issues the MMAs, the pair's second CTA's by the same warp there, which has nothing to issue.  Scales
// and zero points are read by the threads that use them, a stage of theirs ahead.
// A scale that the type has may stand for weights that it has not (fp16: from 4368 on).  Such a weight's product is infinite or NaN, though
// the sum that it belongs to need not be: the wideners report that there is such a scale, and the outputs of its channels are then
// computed as for few rows, by the threads that store them.
// Sums are binary32 in tensor memory, in two accumulators, so that the drain of a tile overlaps the next one's products.
//   warp 0  activations (gathered: and warp 3)   warp 1  MMA issue, tensor memory   warp 2  codes
//   warps 4-7   drain accumulators (bias, sigma, rounding, a turn in shared memory to rows of y)
//   warps 8-    groups that widen weights, stages in turn
// Few tiles: the CTAs of a cluster share a tile's reduction axis and add their sums through distributed shared memory, in order.
// Measured (bf16, groups of 128): 4096 -> 11008 on 4096 rows 247 us alone in a graph, 1.50 PFLOP/s, tensor pipe 83 % active; with SiLU,
// among other passes, at the power cap 296; 8 experts of it, 8192 gathered rows, 567 alone, 640 to 670 among others (tensor pipe 70 %).
// 1024 rows 71, 512 50 (tensor pipe 59 %), 128 19.6 (41 %), 17 17.4 (11 %): there a stage takes its fixed time, whatever its width, and 86
// tiles leave 62 SMs idle.
#include "group_common.cuh"
#include "pipe_tc_common.cuh"

namespace pipe {
namespace grp {

using namespace tcc;

template <bool TA>
constexpr int kTWideners = widener_groups(TA);
template <bool TA>
constexpr int kTThreads = 256 + 128 * kTWideners<TA>;
constexpr uint32_t kTAcol = 256;         // their columns
struct TcArgs : TcPlan {
  Call c;
  int wide_y;      // rows of y are 16-byte aligned
};

__device__ __forceinline__ void tma_pair_2d(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar)
      : "memory");
}
// 16 bytes from global to shared memory, past L1; `real` of them (16 or 0), zeros behind.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, int real) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(real) : "memory");
}
// An arrival on the barrier once this thread's copies so far have landed (one of the arrivals that the barrier is set to).
__device__ __forceinline__ void arrive_behind_copies(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
template <int V>
struct Int {
  static constexpr int value = V;
};
__device__ __forceinline__ void copies_done() { asm volatile("cp.async.wait_all;" ::: "memory"); }
template <int CG, bool TA>   // a: columns of tensor memory (TA) or a descriptor
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  if constexpr (CG == 2 && TA)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(static_cast<uint32_t>(a)), "l"(b), "r"(idesc), "r"(accumulate ? 1u : 0u)
        : "memory");
  else if constexpr (CG == 2)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate ? 1u : 0u)
        : "memory");
  else   // (one CTA alone always has them in tensor memory)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(static_cast<uint32_t>(a)), "l"(b), "r"(idesc), "r"(accumulate ? 1u : 0u)
        : "memory");
}
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"(static_cast<uint16_t>(3))
                 : "memory");
  else
    mma_commit(bar);
}
// Arrival on a barrier of the pair's first CTA (an address of the cluster's window).  Release at CTA scope is enough: what it
// reports is read by this SM's own tensor core, to which the fences before the arrival have made it visible.  (At cluster scope the
// arrival waits some 2000 cycles for everything that the thread has written.)
__device__ __forceinline__ void arrive_lead(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&v)[4][4]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
      "r"(v[0][0]), "r"(v[0][1]), "r"(v[0][2]), "r"(v[0][3]), "r"(v[1][0]), "r"(v[1][1]), "r"(v[1][2]), "r"(v[1][3]),
      "r"(v[2][0]), "r"(v[2][1]), "r"(v[2][2]), "r"(v[2][3]), "r"(v[3][0]), "r"(v[3][1]), "r"(v[3][2]), "r"(v[3][3])
      : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float (&v)[16]) {
  uint32_t u[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]),
        "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
      : "r"(addr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(u[i]);
}
// 16 lanes by 32 columns: register 4 j + 2 h + i is lane (of the 16) l/4 + 8 h, column 8 j + 2 (l % 4) + i.
__device__ __forceinline__ void tmem_ld_16x32(uint32_t addr, float (&v)[16]) {
  uint32_t u[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]),
        "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
      : "r"(addr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(u[i]);
}
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
// Four 8 x 8 blocks of pairs, turned: lane l names the 16 bytes that take column l % 8 of block l / 8.
__device__ __forceinline__ void turn_store(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// One lane of a converged warp, in the form that the compiler knows as one thread of a uniform warp: asked by its lane number
// instead, the thread that issues the MMAs took 1150 cycles for a stage of any width.
__device__ __forceinline__ bool elect_one() {
  uint32_t pred;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(pred));
  return pred != 0;
}
// A bounded wait by a whole warp: false when the CTA is aborting.  Its lanes may see a wait that gives up end differently (the barrier may
// complete between two polls), and what follows is done by whole warps: they go on together or leave together.
template <int SLEEP_NS = 0>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, int* status) {
  return __all_sync(0xffffffffu, mbar_wait<false, SLEEP_NS>(bar, parity, abort_flag, status)) != 0;
}
__device__ __forceinline__ void drain_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
// Whether all four warps of the drain may go on: behind it they meet at barriers without a limit, so that one that has given up must
// not leave the others waiting.
__device__ __forceinline__ bool drain_agrees(bool ok) {
  uint32_t all;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
      "bar.red.and.pred q, 1, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(all)
      : "r"(ok ? 1u : 0u)
      : "memory");
  return all != 0;
}

// Eight neighbouring outputs of a row of y, `room` of them inside the layer.
__device__ __forceinline__ void store_y8(uint16_t* y, const uint4& w, int wide, int room) {
  if (wide && room >= 8) {
    *reinterpret_cast<uint4*>(y) = w;
  } else {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < room) y[k] = static_cast<uint16_t>(u[k >> 1] >> (16 * (k & 1)));
  }
}

// Scales whose weights may be beyond the type's range (an infinite or NaN scale has no finite outputs to save).
template <class H>
__device__ __forceinline__ bool over_range(uint32_t scale) {
  const uint32_t m = scale & 0x7FFFu;
  return m >= H::kOver && m < H::kInf;
}
// The outputs of those among the eight channels from o on that have such a scale, in rows slot, slot + 8, .. below `end`: a group's sum of
// exact products in binary32, times its scale.  (Seldom run: kept small, and inline, for a call would cost the kernel spills.)
template <class H>
__device__ __forceinline__ void store_by_groups(const Call& c, int e, int o, int slot, int end) {
  const int groups = c.I / c.g, runs = c.g / 32;
  uint32_t which = 0;
  for (int k = 0; k < 8 && o + k < c.O; ++k)
#pragma unroll 4
    for (int f = 0; f < groups; ++f)
      if (over_range<H>(__ldcg(static_cast<const uint16_t*>(c.scales) + (static_cast<int64_t>(e) * groups + f) * c.O + o + k))) which |= 1u << k;
  for (; slot < end; slot += 8) {
    for (uint32_t left = which; left; left &= left - 1) {
      const int ch = o + __ffs(left) - 1;
      const int64_t r = c.rows ? __ldcg(c.rows + slot) : slot;
      const bool real = r >= 0 && r < c.T;
      float v[1] = {0.f};
#pragma unroll 1
      for (int f = 0; real && f < groups; ++f) {
        const int64_t meta = (static_cast<int64_t>(e) * groups + f) * c.O + ch;
        const uint32_t zero = zero_pair<H>(c.zeros ? __ldcg(c.zeros + meta) : 8u);
        float sum = 0.f;
#pragma unroll 1
        for (int b = f * runs; b < (f + 1) * runs; ++b) {
          const uint4 q = __ldcg(reinterpret_cast<const uint4*>(c.codes + ((static_cast<int64_t>(e) * c.KB + b) * c.O + ch) * 16));
          const uint4* x = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(c.x) + r * c.ldx + 32 * b);
          const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  #pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4 a = __ldcg(x + i);
            const uint32_t u[4] = {a.x, a.y, a.z, a.w};
  #pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t n = H::add2(code_pair<H>(w[i], k), zero);
              sum = fmaf(H::to_float(static_cast<uint16_t>(u[k])), H::to_float(static_cast<uint16_t>(n)), sum);
              sum = fmaf(H::to_float(static_cast<uint16_t>(u[k] >> 16)), H::to_float(static_cast<uint16_t>(n >> 16)), sum);
            }
          }
        }
        v[0] = fmaf(H::to_float(__ldcg(static_cast<const uint16_t*>(c.scales) + meta)), sum, v[0]);
      }
      if (c.bias) v[0] += H::to_float(__ldcg(static_cast<const uint16_t*>(c.bias) + static_cast<int64_t>(e) * c.O + ch));
      quick_activation(v, c.act);
      static_cast<uint16_t*>(c.y)[static_cast<int64_t>(slot) * c.ldy + ch] = H::from_float(v[0]);
    }
  }
}

// Tile t of the launch: a unit's rows, 128 CG channels from m on.
struct Tile : Unit {
  int m;
  int n;   // columns of its MMAs: the rows rounded up to 32
};
__device__ __forceinline__ Tile tile_of(const TcArgs& p, const int32_t* table, int t) {
  Tile r;
  static_cast<Unit&>(r) = unit_at(table, p.c.E, p.TN, t / p.mtiles);
  r.m = t % p.mtiles;
  r.n = (r.hi - r.lo + 31) & ~31;
  return r;
}

// KPG: runs of 32 codes per group.
template <class H, int CG, int KPG, bool TA>
__global__ void __launch_bounds__(kTThreads<TA>, 1) group_tc_kernel(const __grid_constant__ TcArgs p, const __grid_constant__ CUtensorMap xmap,
                                                                     const __grid_constant__ CUtensorMap cmap) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bars[4 * kTMaxRing + 2 * kTMaxCodes + 4];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_s;
  __shared__ int over_s;   // a scale has been met whose weights may be beyond the type's range
  const Call& c = p.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  int32_t* table = reinterpret_cast<int32_t*>(gen + p.off_table);
  const uint32_t bar0 = smem_u32(bars);
  const uint32_t x_full = bar0, a_full = bar0 + 8 * kTMaxRing, done = bar0 + 16 * kTMaxRing, d_full = bar0 + 24 * kTMaxRing, d_empty = d_full + 16,
                 c_full = d_empty + 16, c_empty = c_full + 8 * kTMaxCodes, x_peer = c_empty + 8 * kTMaxCodes;
  volatile int* abort_flag = &abort_s;
  volatile int* over_flag = &over_s;
  const int crank = cluster_rank();
  const int rank = CG == 2 ? crank : 0;                 // within the pair
  const int part = CG == 1 && p.split > 1 ? crank : 0;  // of the reduction axis
  const int team = blockIdx.x / (CG * p.split), teams = gridDim.x / (CG * p.split);
  const int st0 = static_cast<int>(static_cast<int64_t>(p.stages) * part / p.split), st1 = static_cast<int>(static_cast<int64_t>(p.stages) * (part + 1) / p.split);
  const int own_rows = p.TN / CG;                       // activation rows in this CTA's shared memory
  const uint32_t x_bytes = static_cast<uint32_t>(own_rows) * 256u;
  const uint32_t ring = p.ring;

  if (threadIdx.x == 0) {
    abort_s = 0;
    over_s = 0;
    for (int s = 0; s < kTMaxRing; ++s) {
      mbar_init(x_full + 8 * s, c.rows ? 64 : 1);
      mbar_init(x_peer + 8 * s, 1);
      mbar_init(a_full + 8 * s, 4 * CG);
      mbar_init(done + 8 * s, 1);
    }
    for (int s = 0; s < kTMaxCodes; ++s) {
      mbar_init(c_full + 8 * s, 1);
      mbar_init(c_empty + 8 * s, 4);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(d_full + 8 * b, 1);
      mbar_init(d_empty + 8 * b, 4 * CG);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {   // (two CTAs of this kernel never meet on an SM: with 129 KB or more each they do not fit)
    if (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(512) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  grid_wait();
  grid_release();
  build_units<kTThreads<TA>>(c, p.TN, table);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2 || p.split > 1) cluster_sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  const int tiles = table[c.E] * p.mtiles;   // (below 2^31: the host has looked; of a cluster that shares the axis one at most)

  if (warp == 0 && !c.rows) {
    // ---- activations
    RingPos rp{0, 0};
    uint32_t it = 0;
    const uint32_t lead = CG == 2 ? cluster_address(bars, 0) : bar0;   // the first CTA's barriers
    bool ok = true;
    for (int64_t t = team; ok && t < tiles; t += teams) {
      const Tile tl = tile_of(p, table, static_cast<int>(t));
      const int row0 = tl.lo + rank * (tl.n / CG);
      for (int st = st0; st < st1; ++st, ++it, rp.advance(1, ring)) {
        if (!warp_wait(done + 8 * rp.slot, rp.phase ^ 1, abort_flag, c.status)) { ok = false; break; }
        if (elect_one()) {
          if (rank == 0) mbar_expect_tx(x_full + 8 * rp.slot, CG * x_bytes);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t dst = base + rp.slot * x_bytes + h * (x_bytes / 2);
            const int col = st * kTStage + 64 * h;
            if (CG == 2) tma_pair_2d(dst, &xmap, col, row0, lead + 8 * rp.slot);
            else tma_load_2d(dst, &xmap, col, row0, lead + 8 * rp.slot);
          }
        }
        __syncwarp();
      }
    }
    if (rank == 0 && *abort_flag) drain_ring(x_full, it, p.ring, 20000000ll);
  } else if ((warp == 0 || warp == 3) && c.rows) {
    // ---- activations, gathered: this warp's half of the rows, four rows by 128 bytes per copy instruction
    constexpr int kMost = 128 / 2 / 4;
    RingPos rp{0, 0};
    bool ok = true;
    for (int64_t t = team; ok && t < tiles; t += teams) {
      const Tile tl = tile_of(p, table, static_cast<int>(t));
      const int half = tl.n / CG / 2, mine = half / 4;   // copies of this warp per 64 columns (half: a multiple of 8)
      const int first = (warp ? half : 0) + (lane >> 3);
      const uint32_t place = static_cast<uint32_t>(first * 128 + (((lane & 7) ^ (first & 7)) * 16));   // (+ 4 rows: the other half of the atom)
      const uint16_t* src[kMost];   // rows behind the tile's: its last one, whose sums are not stored
      uint32_t none = 0;            // rows whose index lies outside: zeros
#pragma unroll
      for (int i = 0; i < kMost; ++i) {
        const int at = tl.lo + rank * (tl.n / CG) + first + 4 * i;
        int64_t r = __ldcg(c.rows + (at < tl.hi ? at : tl.hi - 1));
        if (r < 0 || r >= c.T) {
          none |= 1u << i;
          r = 0;
        }
        src[i] = static_cast<const uint16_t*>(c.x) + r * c.ldx + 8 * (lane & 7) + st0 * kTStage;
      }
      const bool plain = !__any_sync(0xffffffffu, none != 0);
      // a stage whose 128 columns from src + 128 * AHEAD on are all there, of FULL copies (0: `mine`) per 64 columns
      auto whole_stage = [&](auto ahead, auto full) {
        constexpr int AHEAD = decltype(ahead)::value, FULL = decltype(full)::value;
        const uint32_t even = base + rp.slot * x_bytes + place, odd = even ^ 64u;
#pragma unroll
        for (int i = 0; i < kMost; ++i)
          if (FULL ? i < FULL : i < mine) {
            copy16((i & 1 ? odd : even) + i * 512, src[i] + AHEAD * kTStage, 16);
            copy16((i & 1 ? odd : even) + x_bytes / 2 + i * 512, src[i] + AHEAD * kTStage + 64, 16);
          }
      };
      auto free_slot = [&]() { return warp_wait(done + 8 * rp.slot, rp.phase ^ 1, abort_flag, c.status); };
      auto hand_on = [&]() {
        arrive_behind_copies(x_full + 8 * rp.slot);
        rp.advance(1, ring);
      };
      int st = st0;
      const int whole = plain ? (st1 * kTStage <= c.I ? st1 : st1 - 1) : st0;   // stages before this one have nothing to leave out
      for (; ok && st + 2 <= whole; st += 2) {   // (two at a time: the rows' addresses are advanced once)
        ok = free_slot();
        if (!ok) break;
        if (mine == kMost) whole_stage(Int<0>{}, Int<kMost>{});
        else whole_stage(Int<0>{}, Int<0>{});
        hand_on();
        ok = free_slot();
        if (!ok) break;
        if (mine == kMost) whole_stage(Int<1>{}, Int<kMost>{});
        else whole_stage(Int<1>{}, Int<0>{});
        hand_on();
#pragma unroll
        for (int i = 0; i < kMost; ++i) src[i] += 2 * kTStage;
      }
      for (; ok && st < st1; ++st) {
        ok = free_slot();
        if (!ok) break;
        const uint32_t even = base + rp.slot * x_bytes + place, odd = even ^ 64u;
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          const bool inside = st * kTStage + 64 * h + 8 * (lane & 7) < c.I;
#pragma unroll
          for (int i = 0; i < kMost; ++i)
            if (i < mine) {
              const bool real = inside && !((none >> i) & 1);
              copy16((i & 1 ? odd : even) + h * (x_bytes / 2) + i * 512, real ? src[i] + 64 * h : static_cast<const uint16_t*>(c.x), real ? 16 : 0);
            }
        }
        hand_on();
#pragma unroll
        for (int i = 0; i < kMost; ++i) src[i] += kTStage;
      }
    }
    copies_done();
  } else if (warp == 2) {
    // ---- codes
    RingPos rp{0, 0};
    uint32_t it = 0;
    bool ok = true;
    for (int64_t t = team; ok && t < tiles; t += teams) {
      const Tile tl = tile_of(p, table, static_cast<int>(t));
      const int o0 = (tl.m * CG + rank) * 128;
      // scales and zero points on their way into L2: this lane's piece of a stage's scales (lanes 0-19, five to a group) or zero points
      // (lanes 20-31, three to a group)
      const int rows = c.O - o0 < 128 ? c.O - o0 : 128;
      const bool is_zero = lane >= 20;
      const int piece_group = is_zero ? (lane - 20) / 3 : lane / 5, piece_byte = 64 * (is_zero ? (lane - 20) % 3 : lane % 5);
      const int run_bytes = is_zero ? rows : 2 * rows, groups = c.KB / KPG;
      const bool mine = rows > 0 && piece_group < 4 / KPG && (!is_zero || c.zeros);
      const int64_t meta0 = (static_cast<int64_t>(tl.e) * groups + piece_group) * c.O + o0;
      const uint8_t* meta = (is_zero ? c.zeros + meta0 : static_cast<const uint8_t*>(c.scales) + 2 * meta0) + (piece_byte < run_bytes ? piece_byte : run_bytes - 1);
      for (int st = st0; st < st1; ++st, ++it, rp.advance(1, p.code_depth)) {
        if (!warp_wait(c_empty + 8 * rp.slot, rp.phase ^ 1, abort_flag, c.status)) { ok = false; break; }
        if (elect_one()) {
          mbar_expect_tx(c_full + 8 * rp.slot, kTCodeBytes);
          tma_load_2d(base + p.off_codes + rp.slot * kTCodeBytes, &cmap, 2 * o0, tl.e * c.KB + 4 * st, c_full + 8 * rp.slot);
        }
        if (mine && st * (4 / KPG) + piece_group < groups) prefetch_l2(meta + static_cast<int64_t>(st) * (4 / KPG) * c.O * (is_zero ? 1 : 2));
        __syncwarp();
      }
    }
    if (*abort_flag) drain_ring(c_full, it, p.code_depth, 20000000ll);
  } else if (warp == 1) {
    // ---- MMA.  With weights in tensor memory one elected lane waits and issues; otherwise the whole warp waits, one lane elected every stage
    // issues, and the waits' verdict is voted on behind it.  (4096 -> 11008, 17 to 512 rows: the first 17.9 to 49.5 us, the second 19.1 to
    // 54; 8 gathered experts, 4096 tokens: 670 and 658.)  Of a descriptor only the low word changes (its address field, in 16-byte units,
    // never carries out of it).
    if (rank == 0 && (!TA || elect_one())) {
      const uint32_t type = H::kBase == Bf16::kBase ? 1u : 0u;
      const uint32_t idesc0 = (1u << 4) | (type << 7) | (type << 10) | (static_cast<uint32_t>(128 * CG >> 4) << 24);
      const uint64_t xdesc = smem_desc_sw128(base), adesc = smem_desc_sw128(base + p.off_a);
      const uint32_t x_lo = static_cast<uint32_t>(xdesc), x_hi = static_cast<uint32_t>(xdesc >> 32);
      const uint32_t a_lo = TA ? tmem + kTAcol : static_cast<uint32_t>(adesc), a_hi = TA ? 0u : static_cast<uint32_t>(adesc >> 32);
      const uint32_t x_stage = x_bytes >> 4, x_half = x_bytes >> 5;
      RingPos rp{0, 0}, wp{0, 0};
      uint32_t n = 0, issued = 0;
      bool ok = true;
      for (int64_t t = team; ok && t < tiles; t += teams, ++n) {
        const uint32_t buf = n & 1, use = n >> 1;
        const uint32_t idesc = idesc0 | (static_cast<uint32_t>(tile_of(p, table, static_cast<int>(t)).n >> 3) << 17);
        ok = TA ? mbar_wait(d_empty + 8 * buf, (use & 1) ^ 1, abort_flag, c.status) : warp_wait(d_empty + 8 * buf, (use & 1) ^ 1, abort_flag, c.status);
        if (!ok) break;
        const uint32_t d = tmem + buf * p.TN;
        for (int st = st0; st < st1; ++st, rp.advance(1, ring), wp.advance(1, kTWideners<TA>)) {
          ok = mbar_wait(x_full + 8 * rp.slot, rp.phase, abort_flag, c.status) &&
               (CG == 1 || !c.rows || mbar_wait(x_peer + 8 * rp.slot, rp.phase, abort_flag, c.status)) && mbar_wait(a_full + 8 * rp.slot, rp.phase, abort_flag, c.status);
          if (c.rows) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t xl = x_lo + rp.slot * x_stage, al = a_lo + wp.slot * (TA ? 64u : kTSlotBytes >> 4);
          if ((TA || elect_one()) && ok) {   // (what did not come is not handed on)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const uint32_t ak = TA ? al + 8u * k : al + (k >> 2) * (kTSlotBytes >> 5) + 2u * (k & 3);
              const uint32_t xk = xl + (k >> 2) * x_half + 2u * (k & 3);
              mma_f16<CG, TA>(d, (static_cast<uint64_t>(a_hi) << 32) | ak, (static_cast<uint64_t>(x_hi) << 32) | xk, idesc, k > 0 || st > st0);
            }
            commit<CG>(done + 8 * rp.slot);
          }
          ++issued;
          if (!TA) ok = __all_sync(0xffffffffu, ok) != 0;
          if (!ok) break;
        }
        if (ok && (TA || elect_one())) commit<CG>(d_full + 8 * buf);
        if (!TA) __syncwarp();
      }
      if (!ok) drain_ring(done, issued, p.ring, 20000000ll);   // no products in flight when tensor memory goes
    } else if (rank != 0 && c.rows) {
      // the pair's second CTA: its gathered rows, made visible to the tensor core, are reported to the first
      const uint32_t lead = cluster_address(bars, 0) + (x_peer - bar0);
      RingPos rp{0, 0};
      bool ok = true;
      for (int64_t t = team; ok && t < tiles; t += teams)
        for (int st = st0; st < st1; ++st, rp.advance(1, ring)) {
          if (!warp_wait(x_full + 8 * rp.slot, rp.phase, abort_flag, c.status)) { ok = false; break; }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) arrive_lead(lead + 8 * rp.slot);
        }
    }
    __syncwarp();   // (one thread may have been alone)
  } else if (warp >= 8) {
    // ---- weights: a thread's channel is a row of the tile
    constexpr uint32_t W = kTWideners<TA>;
    const uint32_t wg = (warp - 8) >> 2;
    const int row = (warp & 3) * 32 + lane;
    const uint32_t lead_a = cluster_address(bars, CG == 2 ? 0 : crank) + 8 * kTMaxRing;
    const uint32_t total = team < tiles ? static_cast<uint32_t>((tiles - team + teams - 1) / teams) * (st1 - st0) : 0;
    // the stage whose scales and zero points are fetched next
    const int groups = c.KB / KPG, nst = st1 - st0;
    int64_t t = team;
    int st = st0 + static_cast<int>(wg);
    int64_t meta = 0;   // of this channel in the first group of the tile's expert
    bool here = false;
    auto open_tile = [&]() {   // (a channel beyond the layer: the last one's, not used)
      const Tile tl = tile_of(p, table, static_cast<int>(t));
      const int o = (tl.m * CG + rank) * 128 + row;
      here = o < c.O;
      meta = static_cast<int64_t>(tl.e) * groups * c.O + (here ? o : c.O - 1);
    };
    uint32_t s2[4 / KPG], z2[4 / KPG], sc[4 / KPG], zp[4 / KPG];
    auto fetch = [&]() {
#pragma unroll
      for (int f = 0; f < 4 / KPG; ++f) {
        const int group = st * (4 / KPG) + f;   // (one beyond the axis: the last one's, which meet activations of zero; made zero themselves below)
        const int64_t at = meta + static_cast<int64_t>(group < groups ? group : groups - 1) * c.O;
        sc[f] = __ldcg(static_cast<const uint16_t*>(c.scales) + at);
        if (c.zeros) zp[f] = __ldcg(c.zeros + at);
      }
    };
    auto settle = [&]() {   // a stage number beyond the tile's is one of a later tile's
      if (st >= st1) {
        do {
          st -= nst;
          t += teams;
        } while (st >= st1);
        if (t < tiles) open_tile();
      }
    };
    if (wg < total) {
      settle();
      if (t == team) open_tile();
      fetch();
    }
    // positions of stage it in the rings of activations (whose barriers are used) and codes; past: of the stage that had its slot
    // before, W stages ago.  A group's slot is its number.
    RingPos rp{0, 0}, cp{0, 0}, past{0, 0};
    rp.advance(wg, ring);
    cp.advance(wg, p.code_depth);
    past.advance(wg, ring);
    bool ok = true;   // (a lane that gives up goes on without waiting: the warp stays whole, and what did not come is not handed on)
    for (uint32_t it = wg; it < total; it += W) {
      // (zero where there is no such channel or group: what is widened there is zero, whatever its codes)
#pragma unroll
      for (int f = 0; f < 4 / KPG; ++f) {
        s2[f] = here && st * (4 / KPG) + f < groups ? sc[f] * 0x10001u : 0u;
        z2[f] = zero_pair<H>(c.zeros ? zp[f] : 8u);
      }
      if (it + W < total) {
        st += W;
        settle();
        fetch();
      }
      ok = ok && mbar_wait(c_full + 8 * cp.slot, cp.phase, abort_flag, c.status);
      const uint8_t* at = gen + p.off_codes + cp.slot * kTCodeBytes;
      uint4 q[4];
#pragma unroll
      for (int b = 0; b < 4; ++b) q[b] = reinterpret_cast<const uint4*>(at)[b * 128 + row];
      uint32_t largest = s2[0];   // (while the codes are on their way)
#pragma unroll
      for (int f = 1; f < 4 / KPG; ++f) largest = H::max_abs2(largest, s2[f]);
      if ((largest & 0x7FFFu) >= H::kOver) *over_flag = 1;
      auto widen = [&](int b, uint32_t (&v)[4][4]) {   // the 32 codes of run b
        const uint32_t w[4] = {q[b].x, q[b].y, q[b].z, q[b].w};
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i >> 2][i & 3] = H::mul2(H::add2(code_pair<H>(w[i >> 2], i & 3), z2[b / KPG]), s2[b / KPG]);
      };
      auto slot_free = [&]() {   // the products of the slot's last stage are done
        if (it < W) return;
        ok = ok && mbar_wait(done + 8 * past.slot, past.phase, abort_flag, c.status);
        past.advance(W, ring);
      };
      if constexpr (TA) {
        slot_free();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t to = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + kTAcol + wg * 64;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          uint32_t v[4][4];
          widen(b, v);
          tmem_st16(to + b * 16, v);
        }
        __syncwarp();
        if (lane == 0 && ok) mbar_arrive(c_empty + 8 * cp.slot);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      } else {
        uint32_t v[4][4][4];   // all of it, before the slot is free: what follows the products of the slot's last stage is the store alone
#pragma unroll
        for (int b = 0; b < 4; ++b) widen(b, v[b]);
        __syncwarp();
        if (lane == 0 && ok) mbar_arrive(c_empty + 8 * cp.slot);
        slot_free();
        uint8_t* to = gen + p.off_a + wg * kTSlotBytes + row * 128;
#pragma unroll
        for (int b = 0; b < 4; ++b)
#pragma unroll
          for (int word = 0; word < 4; ++word) {
            const int piece = (4 * (b & 1) + word) ^ (row & 7);
            *reinterpret_cast<uint4*>(to + (b >> 1) * (kTSlotBytes / 2) + piece * 16) = make_uint4(v[b][word][0], v[b][word][1], v[b][word][2], v[b][word][3]);
          }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // visible to the tensor core
      }
      __syncwarp();
      if (lane == 0 && ok) arrive_lead(lead_a + 8 * rp.slot);
      rp.advance(W, ring);
      cp.advance(W, p.code_depth);
    }
  } else if (warp >= 4 && p.split == 1) {
    // ---- drain
    const int q = warp & 3, tid = threadIdx.x - 128;
    const uint32_t from = tmem + (static_cast<uint32_t>(q * 32) << 16);
    const uint32_t lead_e = cluster_address(bars, CG == 2 ? 0 : crank) + (d_empty - bar0);
    uint8_t* turn = gen + p.off_turn;
    const int piece = tid & 15, r0 = tid >> 4;
    uint32_t n = 0, chunk = 0;
    for (int64_t t = team; t < tiles; t += teams, ++n) {
      const Tile tl = tile_of(p, table, static_cast<int>(t));
      const int o0 = (tl.m * CG + rank) * 128;
      const uint32_t buf = n & 1, use = n >> 1;
      float bias[4];   // of channels 32 q + lane / 4 + 8 h
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int o = o0 + 32 * q + 8 * h + (lane >> 2);
        bias[h] = c.bias && o < c.O ? H::to_float(__ldcg(static_cast<const uint16_t*>(c.bias) + static_cast<int64_t>(tl.e) * c.O + o)) : 0.f;
      }
      const int col = o0 + 8 * piece;
      uint16_t* y = static_cast<uint16_t*>(c.y) + (static_cast<int64_t>(tl.lo) + r0) * c.ldy + col;
      if (!drain_agrees(warp_wait<64>(d_full + 8 * buf, use & 1, abort_flag, c.status))) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const int count = tl.hi - tl.lo;   // rows of y, 32 at a time
      for (int n0 = 0; n0 < count; n0 += 32, ++chunk) {
        uint8_t* to = turn + (chunk & 1) * kTTurnBytes;
#pragma unroll
        for (int g = 0; g < 2; ++g) {   // 16 channels each
          float v[16];
          tmem_ld_16x32(from + (static_cast<uint32_t>(16 * g) << 16) + buf * p.TN + n0, v);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          if (g == 1 && n0 + 32 >= count) {   // the accumulator is read
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (lane == 0) arrive_lead(lead_e + 8 * buf);
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {   // 8 channels: four blocks of 8 rows; a row's 16-byte pieces lie permuted by its number
            float u[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = v[4 * (i >> 1) + 2 * h + (i & 1)] + bias[2 * g + h];
            quick_activation(u, c.act);
            const int at = (4 * q + 2 * g + h) ^ (lane & 7);
            turn_store(smem_u32(to) + lane * 256 + at * 16, H::pack(u[0], u[1]), H::pack(u[2], u[3]), H::pack(u[4], u[5]), H::pack(u[6], u[7]));
          }
        }
        drain_sync();
        uint4 w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const uint4*>(to + (r0 + 8 * i) * 256 + ((piece ^ (r0 & 7)) * 16));
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n0 + r0 + 8 * i < count && col < c.O) store_y8(y + static_cast<int64_t>(8 * i) * c.ldy, w[i], p.wide_y, c.O - col);
        y += 32 * c.ldy;
      }
      // (set ahead of the arrivals that this tile's products waited for; a later tile's scale may have set it too)
      if (*over_flag) store_by_groups<H>(c, tl.e, col, tl.lo + r0, tl.hi);
    }
  }
  if (CG == 1 && p.split > 1) {
    // ---- a cluster's one tile: every CTA leaves its sums in shared memory (behind the last product nothing else lives there),
    // then finishes a share of the outputs, adding the CTAs' sums in ascending order
    float* sums = reinterpret_cast<float*>(gen);   // [TN][128]
    const bool work = team < tiles;
    const Tile tl = work ? tile_of(p, table, team) : Tile{};
    bool ok = work;
    if (work && warp >= 4 && warp < 8) {
      const int row = (warp & 3) * 32 + lane;
      ok = warp_wait<64>(d_full, 0, abort_flag, c.status);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      if (ok)
        for (int n0 = 0; n0 < p.TN; n0 += 16) {
          float v[16];
          tmem_ld16(tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16) + n0, v);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
          for (int i = 0; i < 16; ++i) sums[(n0 + i) * 128 + row] = v[i];
        }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    cluster_sync();
    if (work) {
      const int o0 = tl.m * 128;
      const int over = lane < p.split ? cluster_load(&over_s, lane) : 0;   // (each CTA has met its own share of the scales)
      for (int i = crank * kTThreads<TA> + threadIdx.x; i < p.TN * 16; i += p.split * kTThreads<TA>) {
        const int r = i >> 4, col = (i & 15) * 8;
        const int64_t at = static_cast<int64_t>(tl.lo + r);
        if (at >= tl.hi || o0 + col >= c.O) continue;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 0.f;
        // (loads of four CTAs in flight: one after the other, each some 1000 cycles, eight CTAs' took 10 us)
        for (int q0 = 0; q0 < p.split; q0 += 4) {
          float w[4][8];
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (q0 + q < p.split) {
              const uint32_t a = cluster_address(sums + r * 128 + col, q0 + q);
#pragma unroll
              for (int k = 0; k < 8; k += 4)
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(w[q][k]), "=f"(w[q][k + 1]), "=f"(w[q][k + 2]), "=f"(w[q][k + 3])
                             : "r"(a + 4 * k)
                             : "memory");
            }
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (q0 + q < p.split) {
#pragma unroll
              for (int k = 0; k < 8; ++k) v[k] += w[q][k];
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int o = o0 + col + k;
          if (c.bias && o < c.O) v[k] += H::to_float(__ldcg(static_cast<const uint16_t*>(c.bias) + static_cast<int64_t>(tl.e) * c.O + o));
        }
        quick_activation(v, c.act);
        store_y8(static_cast<uint16_t*>(c.y) + at * c.ldy + o0 + col,
                 make_uint4(H::pack(v[0], v[1]), H::pack(v[2], v[3]), H::pack(v[4], v[5]), H::pack(v[6], v[7])), p.wide_y, c.O - o0 - col);
      }
      if (__any_sync(0xffffffffu, over))
        for (int i = crank * kTThreads<TA> + threadIdx.x; i < p.TN * 16; i += p.split * kTThreads<TA>) {
          const int row = tl.lo + (i >> 4);
          if (row < tl.hi) store_by_groups<H>(c, tl.e, o0 + (i & 15) * 8, row, row + 1);
        }
    }
    cluster_sync();   // no CTA leaves while another reads its sums
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2) cluster_sync();   // nothing of the pair is in flight when its tensor memory goes
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

template <class H, int CG, bool TA>
static auto tc_kernel(int g) {
  return g == 32 ? group_tc_kernel<H, CG, 1, TA> : (g == 64 ? group_tc_kernel<H, CG, 2, TA> : group_tc_kernel<H, CG, 4, TA>);
}
template <class H>
static auto tc_kernel(int cg, bool ta, int g) {
  return cg == 1 ? tc_kernel<H, 1, true>(g) : (ta ? tc_kernel<H, 2, true>(g) : tc_kernel<H, 2, false>(g));
}

static bool encode_2d(CUtensorMap* map, CUtensorMapDataType type, const void* base, uint64_t cols, uint64_t rows, uint64_t pitch_bytes, int box_cols,
                      int box_rows, CUtensorMapSwizzle swizzle) {
  EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {cols, rows}, strides[1] = {pitch_bytes};
  const cuuint32_t box[2] = {static_cast<cuuint32_t>(box_cols), static_cast<cuuint32_t>(box_rows)}, estr[2] = {1, 1};
  return fn(map, type, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

pipe_status linear_tc(const Call& c, bool bf16, cudaStream_t stream) {
  TcArgs p;
  p.c = c;
  // (no tensor to copy from, or no plan: the other kernel)
  if (c.T == 0 || !plan_tc(TcShape{c.E, c.O, c.I, c.offsets != nullptr, c.N}, &p)) return PIPE_ERR_UNSUPPORTED;
  static_assert(kChipSMs == kPlanSMs, "one chip");
  p.wide_y = !(reinterpret_cast<uintptr_t>(c.y) & 15) && c.ldy % 8 == 0;
  const int cg = p.cg;
  const bool ta = p.ta;
  // activations: boxes of 64 columns; codes: rows of O runs of 16 bytes, taken as 8-byte elements, a stage's four runs of 128 channels in
  // one box (behind the layer's channels zeros; behind an expert's last run the next one's, which meet scales of zero)
  CUtensorMap xmap, cmap;
  if (!encode_2d(&xmap, CU_TENSOR_MAP_DATA_TYPE_UINT16, c.x, c.I, c.T, static_cast<uint64_t>(c.ldx) * 2, 64, p.TN / cg, CU_TENSOR_MAP_SWIZZLE_128B) ||
      !encode_2d(&cmap, CU_TENSOR_MAP_DATA_TYPE_FLOAT64, c.codes, static_cast<uint64_t>(c.O) * 2, static_cast<uint64_t>(c.E) * c.KB,
                 static_cast<uint64_t>(c.O) * 16, 256, 4, CU_TENSOR_MAP_SWIZZLE_NONE))
    return runtime_failed();
  void (*k)(TcArgs, CUtensorMap, CUtensorMap) = bf16 ? tc_kernel<Bf16>(cg, ta, c.g) : tc_kernel<Fp16>(cg, ta, c.g);
  if (!allow_dynamic_smem(reinterpret_cast<const void*>(k), kTMaxSmem)) return runtime_failed();
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cg * p.split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(static_cast<unsigned>(p.teams * cg * p.split));
  cfg.blockDim = dim3(ta ? kTThreads<true> : kTThreads<false>);
  cfg.dynamicSmemBytes = p.smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (cudaLaunchKernelEx(&cfg, k, p, xmap, cmap) != cudaSuccess) return runtime_failed();
  count_launch(1);
  return launch_status();
}

}  // namespace grp
}  // namespace pipe
