// Products of a 4-bit layer with group scales with many rows, on the tensor cores (pipe_group_linear, pipe_expert_linear).
//
// The weights are the A operand: a tile is 128 output channels per CTA (256 over a pair of SMs, cta_group::2) by TN rows of
// activations.  tcgen05.mma takes A from tensor memory, so the widened weights never pass through shared memory, whose bandwidth
// the activations need: a thread owns one output channel, reads the 128 codes of a stage (four runs of 16 bytes), subtracts the
// zero point exactly, multiplies by the scale -- one rounding to the layer's type, the type that the MMA takes its operands in;
// it costs a product what the rounding of the activations costs it -- and stores 64 columns of tensor memory.  Activations come
// by tensor copies (rows that are gathered: four rows per copy) in the 128-byte swizzle, codes by bulk copies, each on a ring.
// Sums are binary32 in tensor memory.  Tiles of 256 rows have one accumulator, narrower ones two, so that the drain of a tile
// overlaps the next one's products.
//   warp 0  activations   warp 1  MMA issue, tensor memory   warp 2  codes   warp 3  idle
//   warps 4-11  two groups that drain accumulators (bias, sigma, rounding, a turn in shared memory to rows of y)
//   warps 12-19 two groups that widen weights, every other stage each
// Few tiles: the CTAs of a cluster share a tile's reduction axis and add their sums through distributed shared memory, in order.
#include "group_common.cuh"
#include "pipe_tc_common.cuh"

namespace pipe {
namespace grp {

using namespace tcc;

constexpr int kTThreads = 640;
constexpr int kTStage = 128;         // reduction length of a stage
constexpr int kTRing = 4;            // stages of activations and of widened weights (64 columns of tensor memory each)
constexpr int kTMaxCodes = 12;       // most stages of codes
constexpr int kTCodeBytes = 128 * kTStage / 2;
constexpr int kTTurnBytes = 32 * 128 * 2;   // 32 rows of y by 128 channels
constexpr uint32_t kTAcols = 256;    // tensor memory: accumulators in columns 0-255, widened weights in 256-511

struct TcArgs {
  Call c;
  int TN;          // rows of a tile
  int mtiles;      // ceil(O / (128 CG))
  int stages;      // ceil(I / 128)
  int split;       // CTAs that share a tile's reduction axis
  int code_depth;
  int wide_y;      // rows of y are 16-byte aligned
  uint32_t off_codes, off_turn, off_table;   // shared memory behind the activations
};

__device__ __forceinline__ void tma_pair_2d(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar)
      : "memory");
}
template <int CG>
__device__ __forceinline__ void tma_gather4(uint32_t dst, const CUtensorMap* map, int c0, int4 r, uint32_t bar) {
  if constexpr (CG == 2)
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(r.x), "r"(r.y), "r"(r.z), "r"(r.w), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(r.x), "r"(r.y), "r"(r.z), "r"(r.w), "r"(bar)
        : "memory");
}
template <int CG>
__device__ __forceinline__ void mma_f16_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  if constexpr (CG == 2)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate ? 1u : 0u)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate ? 1u : 0u)
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
// Arrival on a barrier of the pair's first CTA (an address of the cluster's window).
__device__ __forceinline__ void arrive_lead(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
      "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
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
__device__ __forceinline__ void group_sync(int id) { asm volatile("bar.sync %0, 128;" ::"r"(id) : "memory"); }

// Tile t of the launch: its expert, its rows, its first channel.
struct Tile {
  int e, m;
  int lo, hi;   // rows of y (N < 2^31)
};
// first[e]: units before expert e, first[E] all of them; begin[e], end[e]: its rows.
__device__ __forceinline__ Tile tile_of(const TcArgs& p, const int32_t* first, int t) {
  Tile r;
  r.m = t % p.mtiles;
  const int u = t / p.mtiles;
  int lo = 0, hi = p.c.E;   // the last e with first[e] <= u
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= u) lo = mid;
    else hi = mid;
  }
  r.e = lo;
  const int32_t *begin = first + p.c.E + 1, *end = begin + p.c.E;
  r.lo = begin[lo] + (u - first[lo]) * p.TN;
  r.hi = end[lo] - r.lo < p.TN ? end[lo] : r.lo + p.TN;
  return r;
}

template <class H, int CG>
__global__ void __launch_bounds__(kTThreads, 1) group_tc_kernel(const __grid_constant__ TcArgs p, const __grid_constant__ CUtensorMap xmap) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bars[3 * kTRing + 2 * kTMaxCodes + 4];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_s;
  const Call& c = p.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  int32_t* table = reinterpret_cast<int32_t*>(gen + p.off_table);
  const uint32_t bar0 = smem_u32(bars);
  const uint32_t x_full = bar0, a_full = bar0 + 8 * kTRing, done = bar0 + 16 * kTRing, d_full = bar0 + 24 * kTRing, d_empty = d_full + 16,
                 c_full = d_empty + 16, c_empty = c_full + 8 * kTMaxCodes;
  volatile int* abort_flag = &abort_s;
  const int crank = cluster_rank();
  const int rank = CG == 2 ? crank : 0;                 // within the pair
  const int part = CG == 1 && p.split > 1 ? crank : 0;  // of the reduction axis
  const int team = blockIdx.x / (CG * p.split), teams = gridDim.x / (CG * p.split);
  const int st0 = static_cast<int>(static_cast<int64_t>(p.stages) * part / p.split), st1 = static_cast<int>(static_cast<int64_t>(p.stages) * (part + 1) / p.split);
  const int own_rows = p.TN / CG;                       // activation rows in this CTA's shared memory
  const uint32_t x_bytes = static_cast<uint32_t>(own_rows) * 256u;
  const int bufs = p.TN <= 128 ? 2 : 1;

  if (threadIdx.x == 0) {
    abort_s = 0;
    for (int s = 0; s < kTRing; ++s) {
      mbar_init(x_full + 8 * s, 1);
      mbar_init(a_full + 8 * s, 4 * CG);
      mbar_init(done + 8 * s, 1);
    }
    for (int s = 0; s < kTMaxCodes; ++s) {
      mbar_init(c_full + 8 * s, 1);
      mbar_init(c_empty + 8 * s, 4);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(d_full + 8 * b, 1);
      mbar_init(d_empty + 8 * b, 8 * CG);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
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
  // the units of every expert: rows (clamped as find_unit does), tiles, then a prefix over the experts
  for (int e = threadIdx.x; e < c.E; e += kTThreads) {
    int64_t lo = 0, hi = c.N;
    if (c.offsets) {
      lo = __ldcg(c.offsets + e);
      hi = __ldcg(c.offsets + e + 1);
      lo = lo < 0 ? 0 : (lo > c.N ? c.N : lo);
      hi = hi < lo ? lo : (hi > c.N ? c.N : hi);
    }
    table[c.E + 1 + e] = static_cast<int32_t>(lo);
    table[2 * c.E + 1 + e] = static_cast<int32_t>(hi);
  }
  __syncthreads();
  if (warp == 0) {
    int before = 0;
    for (int e0 = 0; e0 < c.E; e0 += 32) {
      const int e = e0 + lane;
      const int mine = e < c.E ? (table[2 * c.E + 1 + e] - table[c.E + 1 + e] + p.TN - 1) / p.TN : 0;
      int upto = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += v;
      }
      if (e < c.E) table[e] = before + upto - mine;
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) table[c.E] = before;
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2 || p.split > 1) cluster_sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  // (offsets out of order can make more units than the host's bound: the rest is not computed, and a tile number stays below 2^31)
  const int64_t all = static_cast<int64_t>(table[c.E]) * p.mtiles;
  const int most = p.split > 1 ? teams : 0x7fffffff;   // (a cluster that shares the axis does one tile)
  const int tiles = static_cast<int>(all < most ? all : most);

  if (warp == 0) {
    // ---- activations
    uint32_t it = 0;
    const uint32_t lead = CG == 2 ? cluster_address(bars, 0) : bar0;   // the first CTA's barriers
    bool ok = true;
    for (int64_t t = team; ok && t < tiles; t += teams) {
      const Tile tl = tile_of(p, table, static_cast<int>(t));
      const int row0 = tl.lo + rank * own_rows;
      for (int st = st0; st < st1; ++st, ++it) {
        const uint32_t s = it % kTRing, use = it / kTRing;
        if (!mbar_wait(done + 8 * s, (use & 1) ^ 1, abort_flag, c.status)) { ok = false; break; }
        const uint32_t full = lead + 8 * s, dst = base + s * x_bytes;
        if (lane == 0 && rank == 0) mbar_expect_tx(x_full + 8 * s, CG * x_bytes);
        __syncwarp();
        if (!c.rows) {
          if (lane < 2) {
            const int col = st * kTStage + 64 * lane;
            if (CG == 2) tma_pair_2d(dst + lane * (x_bytes / 2), &xmap, col, row0, full);
            else tma_load_2d(dst + lane * (x_bytes / 2), &xmap, col, row0, full);
          }
        } else {
          for (int q = lane; q < own_rows / 4; q += 32) {
            int r[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int at = row0 + 4 * q + i;
              r[i] = at < tl.hi ? __ldcg(c.rows + at) : 0;
              if (r[i] < 0 || r[i] >= c.T) r[i] = static_cast<int>(c.T);   // outside: zeros
            }
            const int4 rr = make_int4(r[0], r[1], r[2], r[3]);
            tma_gather4<CG>(dst + q * 512, &xmap, st * kTStage, rr, full);
            tma_gather4<CG>(dst + x_bytes / 2 + q * 512, &xmap, st * kTStage + 64, rr, full);
          }
        }
        __syncwarp();
      }
    }
    if (rank == 0 && *abort_flag) drain_ring(x_full, it, kTRing, 20000000ll);
  } else if (warp == 2) {
    // ---- codes
    uint32_t it = 0;
    bool ok = true;
    for (int64_t t = team; ok && t < tiles; t += teams) {
      const Tile tl = tile_of(p, table, static_cast<int>(t));
      const int o0 = (tl.m * CG + rank) * 128;
      const int rows = c.O - o0 < 128 ? (c.O > o0 ? c.O - o0 : 0) : 128;
      const uint8_t* src = c.codes + (static_cast<int64_t>(tl.e) * c.KB * c.O + o0) * 16;
      for (int st = st0; st < st1; ++st, ++it) {
        const uint32_t s = it % p.code_depth, use = it / p.code_depth;
        if (!mbar_wait(c_empty + 8 * s, (use & 1) ^ 1, abort_flag, c.status)) { ok = false; break; }
        const int runs = c.KB - 4 * st < 4 ? c.KB - 4 * st : 4;
        if (lane == 0) mbar_expect_tx(c_full + 8 * s, static_cast<uint32_t>(runs * rows * 16));
        __syncwarp();
        if (lane < runs && rows > 0) {
          const uint32_t dst = base + p.off_codes + s * kTCodeBytes + lane * 2048;
          asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                       "l"(src + static_cast<int64_t>(4 * st + lane) * c.O * 16), "r"(rows * 16), "r"(c_full + 8 * s)
                       : "memory");
        }
        __syncwarp();
      }
    }
    if (*abort_flag) drain_ring(c_full, it, p.code_depth, 20000000ll);
  } else if (warp == 1) {
    // ---- MMA
    if (rank == 0) {
      const uint32_t type = H::kBase == Bf16::kBase ? 1u : 0u;
      const uint32_t idesc = (1u << 4) | (type << 7) | (type << 10) | (static_cast<uint32_t>(p.TN >> 3) << 17) | (static_cast<uint32_t>(128 * CG >> 4) << 24);
      uint32_t it = 0, n = 0;
      bool ok = true;
      for (int64_t t = team; ok && t < tiles; t += teams, ++n) {
        const uint32_t buf = n % bufs, use = n / bufs;
        if (!mbar_wait<true>(d_empty + 8 * buf, (use & 1) ^ 1, abort_flag, c.status)) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem + buf * 128;
        for (int st = st0; st < st1; ++st, ++it) {
          const uint32_t s = it % kTRing, ph = (it / kTRing) & 1;
          if (!mbar_wait<CG == 2>(x_full + 8 * s, ph, abort_flag, c.status) || !mbar_wait<true>(a_full + 8 * s, ph, abort_flag, c.status)) { ok = false; break; }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          if (lane == 0) {
            const uint32_t a = tmem + kTAcols + s * 64;
            const uint32_t x = base + s * x_bytes;
#pragma unroll
            for (int k = 0; k < 8; ++k)
              mma_f16_ta<CG>(d, a + 8 * k, smem_desc_sw128(x + (k >> 2) * (x_bytes / 2) + (k & 3) * 32), idesc, st > st0 || k > 0);
            commit<CG>(done + 8 * s);
          }
          __syncwarp();
        }
        if (ok && lane == 0) commit<CG>(d_full + 8 * buf);
        __syncwarp();
      }
    }
  } else if (warp >= 12) {
    // ---- weights: a thread's channel is its lane of tensor memory
    const int wg = (warp - 12) >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t lead_a = cluster_address(bars, CG == 2 ? 0 : crank) + 8 * kTRing;
    const int kpg = c.g >> 5, groups = c.KB / kpg;
    uint32_t it = 0;
    bool ok = true;
    for (int64_t t = team; ok && t < tiles; t += teams) {
      const Tile tl = tile_of(p, table, static_cast<int>(t));
      const int o = (tl.m * CG + rank) * 128 + row;
      const bool here = o < c.O;
      const int64_t at0 = static_cast<int64_t>(tl.e) * groups * c.O + (here ? o : 0);
      const uint16_t* scales = static_cast<const uint16_t*>(c.scales) + at0;
      const uint8_t* zeros = c.zeros ? c.zeros + at0 : nullptr;
      // scales and zero points of the four runs of a stage (read one of this group's stages ahead)
      uint32_t sc[4], zp[4];
      auto fetch = [&](int st) {
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int kb = 4 * st + b;
          if (b % kpg == 0) {
            sc[b] = 0;
            zp[b] = 8;
            if (here && st < st1 && kb < c.KB) {
              const int64_t at = static_cast<int64_t>(kb / kpg) * c.O;
              sc[b] = __ldcg(scales + at);
              if (zeros) zp[b] = __ldcg(zeros + at);
            }
          } else {
            sc[b] = sc[b - 1];
            zp[b] = zp[b - 1];
          }
        }
      };
      int st = st0 + static_cast<int>((it ^ static_cast<uint32_t>(wg)) & 1);
      it += st - st0;
      fetch(st);
      for (; st < st1; st += 2, it += 2) {
        const uint32_t cs = it % p.code_depth, s = it % kTRing, use = it / kTRing;
        uint32_t s2[4], z2[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          s2[b] = sc[b] | (sc[b] << 16);
          z2[b] = zero_pair<H>(zp[b]);
        }
        fetch(st + 2);
        if (!mbar_wait(c_full + 8 * cs, (it / p.code_depth) & 1, abort_flag, c.status)) { ok = false; break; }
        const uint4* src = reinterpret_cast<const uint4*>(gen + p.off_codes + cs * kTCodeBytes) + row;
        uint4 q[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) q[b] = src[b * 128];
        if (!mbar_wait(done + 8 * s, (use & 1) ^ 1, abort_flag, c.status)) { ok = false; break; }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          uint32_t v[16];
          const uint32_t w[4] = {q[b].x, q[b].y, q[b].z, q[b].w};
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] = H::mul2(H::sub2(code_pair<H>(w[i >> 2], i & 3), z2[b]), s2[b]);
          if (4 * st + b >= c.KB) {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = 0;
          }
          tmem_st16(tmem + lane_base + kTAcols + s * 64 + b * 16, v);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(c_empty + 8 * cs);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) arrive_lead(lead_a + 8 * s);
      }
      it -= st - st1;   // the stage count at the tile's end
    }
  } else if (warp >= 4 && p.split == 1) {
    // ---- drain
    const int wg = (warp - 4) >> 2, row = (warp & 3) * 32 + lane, tid = threadIdx.x - 128 - 128 * wg;
    const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t lead_e = cluster_address(bars, CG == 2 ? 0 : crank) + (d_empty - bar0);
    uint8_t* turn = gen + p.off_turn + wg * 2 * kTTurnBytes;
    uint32_t n = 0, chunk = 0;
    for (int64_t t = team; t < tiles; t += teams, ++n) {
      const Tile tl = tile_of(p, table, static_cast<int>(t));
      const int o0 = (tl.m * CG + rank) * 128, o = o0 + row;
      const uint32_t buf = n % bufs, use = n / bufs;
      const float bias = c.bias && o < c.O ? H::to_float(__ldcg(static_cast<const uint16_t*>(c.bias) + static_cast<int64_t>(tl.e) * c.O + o)) : 0.f;
      if (!mbar_wait<false, 64>(d_full + 8 * buf, use & 1, abort_flag, c.status)) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      for (int n0 = 32 * wg; n0 < p.TN; n0 += 64, ++chunk) {
        if (tl.lo + n0 >= tl.hi) break;   // (the same for all warps of the group)
        uint8_t* to = turn + (chunk & 1) * kTTurnBytes;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float v[16];
          tmem_ld16(tmem + lane_base + buf * 128 + n0 + 16 * h, v);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
          for (int i = 0; i < 16; ++i)
            *reinterpret_cast<uint16_t*>(to + (16 * h + i) * 256 + row * 2) = H::from_float(apply_activation(v[i] + bias, c.act));
        }
        group_sync(1 + wg);
        const int col = (tid & 15) * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = (tid >> 4) + 8 * i;
          const int64_t at = static_cast<int64_t>(tl.lo + n0 + r);
          if (at < tl.hi && o0 + col < c.O) {
            const uint4 q = *reinterpret_cast<const uint4*>(to + r * 256 + col * 2);
            uint16_t* y = static_cast<uint16_t*>(c.y) + at * c.ldy + o0 + col;
            if (p.wide_y && o0 + col + 8 <= c.O) {
              *reinterpret_cast<uint4*>(y) = q;
            } else {
              const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
              for (int k = 0; k < 8; ++k)
                if (o0 + col + k < c.O) y[k] = static_cast<uint16_t>(u[k >> 1] >> (16 * (k & 1)));
            }
          }
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) arrive_lead(lead_e + 8 * buf);
    }
  }
  if (CG == 1 && p.split > 1) {
    // ---- a cluster's one tile: every CTA leaves its sums in shared memory (behind the last product nothing else lives there),
    // then finishes a share of the outputs, adding the CTAs' sums in ascending order
    float* sums = reinterpret_cast<float*>(gen);   // [TN][128]
    const bool work = team < tiles;
    const Tile tl = work ? tile_of(p, table, team) : Tile{};
    bool ok = work;
    if (work && warp >= 4 && warp < 12) {
      const int wg = (warp - 4) >> 2, row = (warp & 3) * 32 + lane;
      ok = mbar_wait<false, 64>(d_full, 0, abort_flag, c.status);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      if (ok)
        for (int n0 = 16 * wg; n0 < p.TN; n0 += 32) {
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
      for (int i = crank * kTThreads + threadIdx.x; i < p.TN * 16; i += p.split * kTThreads) {
        const int r = i >> 4, col = (i & 15) * 8;
        const int64_t at = static_cast<int64_t>(tl.lo + r);
        if (at >= tl.hi || o0 + col >= c.O) continue;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = 0.f;
        for (int q = 0; q < p.split; ++q) {
          const uint32_t a = cluster_address(sums + r * 128 + col, q);
#pragma unroll
          for (int k = 0; k < 8; k += 4) {
            float w[4];
            asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(w[0]), "=f"(w[1]), "=f"(w[2]), "=f"(w[3]) : "r"(a + 4 * k) : "memory");
#pragma unroll
            for (int j = 0; j < 4; ++j) v[k + j] += w[j];
          }
        }
        uint32_t u[4];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int o = o0 + col + k;
          if (c.bias && o < c.O) v[k] += H::to_float(__ldcg(static_cast<const uint16_t*>(c.bias) + static_cast<int64_t>(tl.e) * c.O + o));
          const uint32_t h = H::from_float(apply_activation(v[k], c.act));
          u[k >> 1] = k & 1 ? u[k >> 1] | (h << 16) : h;
        }
        uint16_t* y = static_cast<uint16_t*>(c.y) + at * c.ldy + o0 + col;
        if (p.wide_y && o0 + col + 8 <= c.O) {
          *reinterpret_cast<uint4*>(y) = make_uint4(u[0], u[1], u[2], u[3]);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (o0 + col + k < c.O) y[k] = static_cast<uint16_t>(u[k >> 1] >> (16 * (k & 1)));
        }
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

static bool make_x_map(CUtensorMap* map, const Call& c, int box_rows) {
  EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(c.I), static_cast<cuuint64_t>(c.T > 0 ? c.T : 1)};
  const cuuint64_t strides[1] = {static_cast<cuuint64_t>(c.ldx) * 2};
  const cuuint32_t box[2] = {64, static_cast<cuuint32_t>(box_rows)};
  const cuuint32_t estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, const_cast<void*>(c.x), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

pipe_status linear_tc(const Call& c, bool bf16, cudaStream_t stream) {
  if (c.T == 0) return PIPE_ERR_UNSUPPORTED;   // (no tensor to copy from; the other kernel reads none)
  TcArgs p;
  p.c = c;
  const int64_t rows = c.offsets ? ceil_div<int64_t>(c.N, c.E) : c.N;
  // 256 rows are a pair's tile: one CTA alone has no room for four stages of them
  const int cg = rows > 128 && c.O > 128 ? 2 : 1;
  p.TN = rows <= 32 ? 32 : (rows <= 64 ? 64 : (cg == 1 ? 128 : 256));
  p.stages = ceil_div(c.I, kTStage);
  const int64_t units = most_units(c, p.TN);
  p.mtiles = ceil_div(c.O, 128 * cg);
  const int64_t tiles = units * p.mtiles;
  p.split = 1;
  if (cg == 1)
    while (p.split < 8 && tiles * p.split * 2 <= kPlanSMs && p.stages >= 4 * p.split) p.split *= 2;
  int64_t teams = p.split > 1 ? tiles : kPlanSMs / cg;
  if (teams > tiles) teams = tiles;
  p.wide_y = !(reinterpret_cast<uintptr_t>(c.y) & 15) && c.ldy % 8 == 0;
  const int x_bytes = kTRing * (p.TN / cg) * 256;
  const int table = (3 * c.E + 1) * 4;
  p.off_codes = x_bytes;
  const int turn = p.split > 1 ? 0 : 4 * kTTurnBytes;
  const int room = 220 * 1024 - 1024 - x_bytes - turn - table;
  p.code_depth = room / kTCodeBytes < kTMaxCodes ? room / kTCodeBytes : kTMaxCodes;
  if (p.code_depth < 2) return PIPE_ERR_UNSUPPORTED;
  p.off_turn = p.off_codes + p.code_depth * kTCodeBytes;
  p.off_table = p.off_turn + turn;
  const int smem = 1024 + static_cast<int>(p.off_table) + table;
  CUtensorMap map;
  if (!make_x_map(&map, c, c.rows ? 1 : p.TN / cg)) return PIPE_ERR_CUDA;
  void (*k)(TcArgs, CUtensorMap) = bf16 ? (cg == 2 ? group_tc_kernel<Bf16, 2> : group_tc_kernel<Bf16, 1>) : (cg == 2 ? group_tc_kernel<Fp16, 2> : group_tc_kernel<Fp16, 1>);
  if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return PIPE_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cg * p.split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(static_cast<unsigned>(teams * cg * p.split));
  cfg.blockDim = dim3(kTThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (cudaLaunchKernelEx(&cfg, k, p, map) != cudaSuccess) return PIPE_ERR_CUDA;
  count_launch(1);
  return launch_status();
}

}  // namespace grp
}  // namespace pipe
