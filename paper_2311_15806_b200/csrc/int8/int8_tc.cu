// Products of the 8-bit integer layers on the tensor cores (pipe_int8_linear, pipe_int8_expert_linear): tcgen05 kind::i8.
//
// The weights are the M operand, the tokens the N operand: a tile is TM output channels per CTA, 32 to 128 of the MMA's 128 (over a pair of SMs,
// cta_group::2, twice that) by up to TN rows, so that one token costs an MMA of 16 columns and a prompt one of 256.  Both operands lie K-major as they are in memory:
// tensor copies of 128 codes by the tile's rows in the 128-byte swizzle, on one ring, what lies behind the rows or the reduction axis
// read as zeros.  Sums are int32 in tensor memory, exact, in two accumulators, so that the drain of a tile overlaps the next one's
// products.  The drain applies the channel's scale, the token's, bias and sigma; 16-bit outputs are turned in shared memory to rows of
// y, 32-bit ones are stored as they come, 32 neighbouring channels at a time.
//   warp 0 copies   warp 1 MMAs, tensor memory   warps 2 .. drain, two or four for every 32 lanes of tensor memory, which take 32 rows in turn
// Few tiles: the CTAs of a cluster share a tile's reduction axis and add their sums through distributed shared memory (integers: in any
// order the same).  Such a CTA gives its tensor memory back before it waits for the others: one that held it could wait for a CTA
// that waits for tensor memory on another SM.
// A call's weights are asked into L2 before the wait for the launch before it: that reads nothing early, what is read comes behind the
// wait.
// Bound by HBM on few rows (4096 -> 11008 on one row: 10.2 us among launches that overlap, 4.4 TB/s; the start and the last drain are the
// rest), by the tensor pipe on many (4096 rows: 119 us, 3.1 POP/s, pipe 87 % busy; under the power cap of a long run 141), by the drain, 3.7 us
// of a tile of 256 x 256 with eight warps, on many rows of fewer than some 1000 values (11008 <- 256 on 4096 rows: 35 us with sixteen).
#include "int8_common.cuh"
#include "int8_plan.h"
#include "pipe_tc_common.cuh"

namespace pipe {
namespace i8 {

using namespace tcc;
using grp::cluster_address;
using grp::cluster_rank;
using grp::cluster_sync;
using grp::Unit;

constexpr int kThreads = 64 + 32 * kMoreDrainWarps, kFewThreads = 64 + 32 * kDrainWarps;   // the most, and those that every launch has
struct TcArgs : TcPlan {
  Call call;
  int wide_y;      // rows of y are 16-byte aligned
};

__device__ __forceinline__ void tma_pair_2d(uint32_t dst, const CUtensorMap* map, int c0, int c1, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void ask_l2(const CUtensorMap* map, int c0, int c1) {
  asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" ::"l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1) : "memory");
}
template <int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate) {
  if constexpr (CG == 2)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate ? 1u : 0u)
        : "memory");
  else
    mma_i8(d, a, b, idesc, accumulate);
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
// Arrival on a barrier of the pair's first CTA (an address of the cluster's window); what it reports has been read by then.
__device__ __forceinline__ void arrive_lead(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, int (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
        "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(addr)
      : "memory");
}
// 16 lanes by 32 columns: register 4 j + 2 h + i is lane (of the 16) l/4 + 8 h, column 8 j + 2 (l % 4) + i.
__device__ __forceinline__ void tmem_ld_16x32(uint32_t addr, int (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
        "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(addr)
      : "memory");
}
// Four 8 x 8 blocks of pairs, turned: lane l names the 16 bytes that take column l % 8 of block l / 8.
__device__ __forceinline__ void turn_store(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ bool elect_one() {
  uint32_t pred;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(pred));
  return pred != 0;
}
// Eight neighbouring outputs of a row of y, `room` of them inside the layer.
template <class H>
__device__ __forceinline__ void store_y8(void* y, int64_t at, const float (&v)[8], int wide, int room) {
  if (wide && room >= 8) {
    if constexpr (H::kBytes == 4) {
      float4* p = reinterpret_cast<float4*>(static_cast<float*>(y) + at);
      p[0] = make_float4(v[0], v[1], v[2], v[3]);
      p[1] = make_float4(v[4], v[5], v[6], v[7]);
    } else {
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(y) + at) = make_uint4(H::pack(v[0], v[1]), H::pack(v[2], v[3]), H::pack(v[4], v[5]), H::pack(v[6], v[7]));
    }
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < room) H::store(y, at + k, v[k]);
  }
}

// Tile t of the launch: a unit's rows, TM channels of every CTA.
struct Tile : Unit {
  int o0;  // this CTA's first channel
  int n;   // columns of its MMAs: the rows rounded up to what the MMA takes
};
template <int CG>
__device__ __forceinline__ Tile tile_of(const TcArgs& p, const int32_t* table, int t, int rank) {
  Tile r;
  const int u = t / p.mtiles;
  if (p.call.c.offsets) {
    static_cast<Unit&>(r) = grp::unit_at(table, p.call.c.E, p.TN, u);
  } else {   // (N and the tile's end are below 2^31)
    r.e = 0;
    r.lo = u * p.TN;
    r.hi = min(r.lo + p.TN, static_cast<int>(p.call.c.N));
  }
  r.o0 = (t % p.mtiles * CG + rank) * p.TM;
  constexpr int kStep = CG == 2 ? 32 : 16;
  r.n = (r.hi - r.lo + kStep - 1) & ~(kStep - 1);
  return r;
}

template <class H, int CG>
__global__ void __launch_bounds__(kThreads) int8_tc_kernel(const __grid_constant__ TcArgs p, const __grid_constant__ CUtensorMap wmap,
                                                            const __grid_constant__ CUtensorMap xmap) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ uint64_t bars[2 * kMaxRing + 4];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_s;
  const grp::Call& c = p.call.c;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* gen = smem_raw + (base - smem_u32(smem_raw));
  int32_t* table = reinterpret_cast<int32_t*>(gen + p.off_table);
  const uint32_t bar0 = smem_u32(bars);
  const uint32_t full = bar0, done = bar0 + 8 * kMaxRing, d_full = bar0 + 16 * kMaxRing, d_empty = d_full + 16;
  volatile int* abort_flag = &abort_s;
  const int crank = cluster_rank();
  const int rank = CG == 2 ? crank : 0;                 // within the pair
  const int part = CG == 1 && p.split > 1 ? crank : 0;  // of the reduction axis
  const int team = blockIdx.x / (CG * p.split), teams = gridDim.x / (CG * p.split);
  const int st0 = p.stages * part / p.split, st1 = p.stages * (part + 1) / p.split;   // (stages <= 1024)
  const uint32_t w_block = static_cast<uint32_t>(p.TM) * kBlock, x_block = static_cast<uint32_t>(p.TN / CG) * kBlock;
  const uint32_t stage_bytes = p.KS * (w_block + x_block);
  const uint32_t ring = p.ring;
  const int acc_pitch = accumulator_columns(p.TN);

  if (threadIdx.x == 0) {
    abort_s = 0;
    for (int s = 0; s < kMaxRing; ++s) {
      mbar_init(full + 8 * s, 1);
      mbar_init(done + 8 * s, 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(d_full + 8 * b, 1);
      mbar_init(d_empty + 8 * b, p.drain * CG);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&wmap)) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&xmap)) : "memory");
    if (!c.offsets && team < p.tiles) {
      const int o0 = (team % p.mtiles * CG + rank) * p.TM;
      for (int b = st0 * p.KS; b < st1 * p.KS && b < st0 * p.KS + p.ahead; ++b) ask_l2(&wmap, b * kBlock, o0);
    }
  }
  if (warp == 1) {
    if (CG == 2) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(p.columns) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(p.columns) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  grid_wait();
  grid_release();
  if (c.offsets) grp::build_units<kFewThreads>(c, p.TN, table);   // (one expert needs no table: 0.7 us)
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2) cluster_sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = tmem_slot;
  const int tiles = c.offsets ? table[c.E] * p.mtiles : static_cast<int>(p.tiles);   // (below 2^31: the host has looked; of a cluster that shares the axis one at most)

  if (warp == 0) {
    // ---- copies: one thread
    if (elect_one()) {
      RingPos rp{0, 0};
      uint32_t it = 0;
      const uint32_t lead = CG == 2 ? cluster_address(bars, 0) : bar0;   // the first CTA's barriers
      bool ok = true;
      for (int64_t t = team; ok && t < tiles; t += teams) {
        const Tile tl = tile_of<CG>(p, table, static_cast<int>(t), rank);
        const int row0 = tl.lo + rank * (tl.n / CG), w0 = tl.e * c.O + tl.o0;
        for (int st = st0; st < st1; ++st, ++it, rp.advance(1, ring)) {
          if (!mbar_wait(done + 8 * rp.slot, rp.phase ^ 1, abort_flag, c.status)) { ok = false; break; }
          if (rank == 0) mbar_expect_tx(full + 8 * rp.slot, CG * stage_bytes);
          const uint32_t w = base + rp.slot * stage_bytes, x = w + p.KS * w_block;
          for (int b = 0; b < p.KS; ++b) {
            const int k = (st * p.KS + b) * kBlock;
            if (CG == 2) {
              tma_pair_2d(w + b * w_block, &wmap, k, w0, lead + 8 * rp.slot);
              tma_pair_2d(x + b * x_block, &xmap, k, row0, lead + 8 * rp.slot);
            } else {
              tma_load_2d(w + b * w_block, &wmap, k, w0, full + 8 * rp.slot);
              tma_load_2d(x + b * x_block, &xmap, k, row0, full + 8 * rp.slot);
            }
          }
        }
      }
      if (rank == 0 && *abort_flag) drain_ring(full, it, p.ring, 20000000ll);
    }
    __syncwarp();
  } else if (warp == 1) {
    // ---- MMAs: one thread of the pair's first CTA.  Of a descriptor only the low word changes (its address field, in 16-byte units,
    // never carries out of it).
    if (rank == 0 && elect_one()) {
      const uint64_t desc0 = smem_desc_sw128(base);
      const uint32_t lo = static_cast<uint32_t>(desc0);
      const uint64_t hi = desc0 & 0xFFFFFFFF00000000ull;
      RingPos rp{0, 0};
      uint32_t n = 0, issued = 0;
      bool ok = true;
      for (int64_t t = team; ok && t < tiles; t += teams, ++n) {
        const uint32_t buf = n & 1, use = n >> 1;
        const uint32_t idesc = idesc_i8(128 * CG, tile_of<CG>(p, table, static_cast<int>(t), rank).n);
        ok = CG == 2 ? mbar_wait<true>(d_empty + 8 * buf, (use & 1) ^ 1, abort_flag, c.status) : mbar_wait(d_empty + 8 * buf, (use & 1) ^ 1, abort_flag, c.status);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t d = tmem + buf * acc_pitch;
        for (int st = st0; st < st1; ++st, rp.advance(1, ring)) {
          ok = mbar_wait(full + 8 * rp.slot, rp.phase, abort_flag, c.status);
          if (!ok) break;
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t al = lo + rp.slot * (stage_bytes >> 4), xl = al + p.KS * (w_block >> 4);
          for (int b = 0; b < p.KS; ++b) {
#pragma unroll
            for (int k = 0; k < 4; ++k) mma<CG>(d, hi | (al + b * (w_block >> 4) + 2u * k), hi | (xl + b * (x_block >> 4) + 2u * k), idesc, k > 0 || b > 0 || st > st0);
          }
          commit<CG>(done + 8 * rp.slot);
          ++issued;
        }
        if (ok) commit<CG>(d_full + 8 * buf);
      }
      if (!ok) drain_ring(done, issued, p.ring, 20000000ll);   // no products in flight when tensor memory goes
    }
    __syncwarp();   // (one thread may have been alone)
  } else if (p.split == 1) {
    // ---- drain
    const int q = warp & 3, part = (warp - 2) >> 2;   // this warp's 32 lanes of tensor memory, and its turn
    const uint32_t from = tmem + (static_cast<uint32_t>(q * 32) << 16);
    const uint32_t lead_e = (CG == 2 ? cluster_address(bars, 0) : bar0) + (d_empty - bar0);
    float* sx = reinterpret_cast<float*>(gen + p.off_sx) + q * acc_pitch;   // the rows' scales: a warp copies those of its rows
    uint8_t* turn = gen + p.off_turn + (4 * part + q) * kTurnBytes;
    const int step = 8 * p.drain;   // four warps take 32 rows
    uint32_t n = 0;
    for (int64_t t = team; t < tiles; t += teams, ++n) {
      const Tile tl = tile_of<CG>(p, table, static_cast<int>(t), rank);
      const int o0 = tl.o0, end = min(c.O, o0 + p.TM), count = tl.hi - tl.lo;
      const int64_t ch0 = static_cast<int64_t>(tl.e) * c.O, row0 = tl.lo;
      const uint32_t buf = n & 1, use = n >> 1;
      constexpr int kMine = H::kBytes == 4 ? 1 : 4;   // this thread's channels: 32 q + lane, or 32 q + lane / 4 + 8 h
      float sw[kMine], bias[kMine];
#pragma unroll
      for (int h = 0; h < kMine; ++h) {
        const int o = o0 + 32 * q + (kMine == 1 ? lane : 8 * h + (lane >> 2));
        sw[h] = o < end ? __ldcg(p.call.sw + ch0 + o) : 0.f;
        bias[h] = c.bias && o < end ? H::load(c.bias, ch0 + o) : 0.f;
      }
      for (int i = 32 * part + lane; i < acc_pitch; i += step) sx[i] = i < count ? __ldcg(p.call.sx + tl.lo + i) : 0.f;
      __syncwarp();
      if (!__all_sync(0xffffffffu, mbar_wait<CG == 2, 64>(d_full + 8 * buf, use & 1, abort_flag, c.status))) break;
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const uint32_t acc = from + buf * acc_pitch;
      for (int n0 = 32 * part; n0 < count; n0 += step) {   // rows of y, 32 at a time
        int v[2][16];
        if constexpr (H::kBytes == 4) {
          const int o = o0 + 32 * q + lane;
          float* y = static_cast<float*>(c.y) + (row0 + n0) * c.ldy + o;
          tmem_ld16(acc + n0, v[0]);   // 16 rows each
          tmem_ld16(acc + n0 + 16, v[1]);
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          float u[2][16];
#pragma unroll
          for (int g = 0; g < 2; ++g) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              const float4 s = *reinterpret_cast<const float4*>(sx + n0 + 16 * g + i);
              u[g][i] = scaled(v[g][i], sw[0], s.x, bias[0]);
              u[g][i + 1] = scaled(v[g][i + 1], sw[0], s.y, bias[0]);
              u[g][i + 2] = scaled(v[g][i + 2], sw[0], s.z, bias[0]);
              u[g][i + 3] = scaled(v[g][i + 3], sw[0], s.w, bias[0]);
            }
          }
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            activate<H>(u[g], c.act);
            if (o < end) {
#pragma unroll
              for (int i = 0; i < 16; ++i, y += c.ldy)
                if (n0 + 16 * g + i < count) *y = u[g][i];
            }
          }
        } else if (!p.wide_y) {
          // rows that begin anywhere: a channel a lane as well, 16 rows at a time (2095 rows of 4798 channels: 15 us; turned and stored
          // a row at a time 29, eight neighbouring channels a lane 56)
          const int o = o0 + 32 * q + lane;
          const float scale = o < end ? __ldcg(p.call.sw + ch0 + o) : 0.f, add = c.bias && o < end ? H::load(c.bias, ch0 + o) : 0.f;
          uint16_t* y = static_cast<uint16_t*>(c.y) + (row0 + n0) * c.ldy + o;
#pragma unroll 1
          for (int i0 = 0; i0 < 32; i0 += 16) {
            tmem_ld16(acc + n0 + i0, v[0]);
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
            float u[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) u[i] = scaled(v[0][i], scale, sx[n0 + i0 + i], add);
            activate<H>(u, c.act);
            if (o < end) {
#pragma unroll
              for (int i = 0; i < 16; ++i, y += c.ldy)
                if (n0 + i0 + i < count) H::store(y, 0, u[i]);
            }
          }
        } else {
          tmem_ld_16x32(acc + n0, v[0]);   // 16 channels each
          tmem_ld_16x32(acc + (16u << 16) + n0, v[1]);
          float sc[8];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 two = *reinterpret_cast<const float2*>(sx + n0 + 8 * j + 2 * (lane & 3));
            sc[2 * j] = two.x;
            sc[2 * j + 1] = two.y;
          }
          __syncwarp();   // the turn of the rows before has been read
          asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
          // 8 channels at a time: four blocks of 8 rows; a row is 64 bytes, its 16-byte pieces permuted by its number
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            float u[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) u[i] = scaled(v[h >> 1][4 * (i >> 1) + 2 * (h & 1) + (i & 1)], sw[h], sc[i], bias[h]);
            activate<H>(u, c.act);
            turn_store(smem_u32(turn) + lane * 64 + ((h ^ ((lane >> 1) & 3)) * 16), H::pack(u[0], u[1]), H::pack(u[2], u[3]), H::pack(u[4], u[5]), H::pack(u[6], u[7]));
          }
          __syncwarp();
          uint16_t* y = static_cast<uint16_t*>(c.y) + (row0 + n0) * c.ldy + o0 + 32 * q;
          const int room = end - o0 - 32 * q;   // channels of y from there on
          const int piece = lane & 3, r0 = lane >> 2;
          uint16_t* at = y + r0 * c.ldy + 8 * piece;
          uint4 w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const uint4*>(turn + (r0 + 8 * i) * 64 + ((piece ^ ((r0 >> 1) & 3)) * 16));
#pragma unroll
          for (int i = 0; i < 4; ++i, at += 8 * c.ldy)
            if (n0 + r0 + 8 * i < count) {
              if (room - 8 * piece >= 8) {
                *reinterpret_cast<uint4*>(at) = w[i];
              } else {
                const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
                for (int k = 0; k < 8; ++k)
                  if (k < room - 8 * piece) at[k] = static_cast<uint16_t>(u[k >> 1] >> (16 * (k & 1)));
              }
            }
        }
      }
      // the accumulator is read
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) arrive_lead(lead_e + 8 * buf);
    }
  } else if (warp < 6 && team < tiles) {
    // ---- a split's sums go to shared memory (behind the last product nothing else lives there)
    const int q = warp & 3, row = 32 * q + lane;
    int32_t* sums = reinterpret_cast<int32_t*>(gen);   // [TN][128]
    const Tile tl = tile_of<CG>(p, table, team, rank);
    const bool ok = __all_sync(0xffffffffu, mbar_wait<false, 64>(d_full, 0, abort_flag, c.status)) != 0;
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (ok)
      for (int n0 = 0; n0 < tl.n; n0 += 16) {
        int v[16];
        tmem_ld16(tmem + (static_cast<uint32_t>(q * 32) << 16) + n0, v);
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[(n0 + i) * 128 + row] = v[i];
      }
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (CG == 2) cluster_sync();   // nothing of the pair is in flight when its tensor memory goes
  if (warp == 1) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(p.columns) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(p.columns) : "memory");
  }
  if (CG == 1 && p.split > 1) {
    // ---- every CTA finishes a share of the tile's outputs from the CTAs' sums
    cluster_sync();
    if (team < tiles) {
      const int32_t* sums = reinterpret_cast<const int32_t*>(gen);
      const Tile tl = tile_of<CG>(p, table, team, rank);
      const int64_t ch0 = static_cast<int64_t>(tl.e) * c.O;
      for (int i = crank * kFewThreads + threadIdx.x; i < (tl.hi - tl.lo) * 16; i += p.split * kFewThreads) {
        const int r = i >> 4, col = tl.o0 + (i & 15) * 8;
        if (col >= min(c.O, tl.o0 + p.TM)) continue;
        int acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int q = 0; q < 8; ++q)   // (all loads in flight at once)
          if (q < p.split) {
            const uint32_t a = cluster_address(sums + r * 128 + (i & 15) * 8, q);
            int w[8];
#pragma unroll
            for (int k = 0; k < 8; k += 4)
              asm volatile("ld.shared::cluster.v4.s32 {%0, %1, %2, %3}, [%4];"
                           : "=r"(w[k]), "=r"(w[k + 1]), "=r"(w[k + 2]), "=r"(w[k + 3])
                           : "r"(a + 4 * k)
                           : "memory");
#pragma unroll
            for (int k = 0; k < 8; ++k) acc[k] += w[k];
          }
        const float sx = __ldcg(p.call.sx + tl.lo + r);
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const bool real = col + k < c.O;
          v[k] = scaled(acc[k], real ? __ldcg(p.call.sw + ch0 + col + k) : 0.f, sx, real && c.bias ? H::load(c.bias, ch0 + col + k) : 0.f);
        }
        activate<H>(v, c.act);
        store_y8<H>(c.y, (static_cast<int64_t>(tl.lo) + r) * c.ldy + col, v, p.wide_y, c.O - col);
      }
    }
    cluster_sync();   // no CTA leaves while another reads its sums
  }
}

template <class H>
static auto tc_kernel(int cg) {
  return cg == 1 ? int8_tc_kernel<H, 1> : int8_tc_kernel<H, 2>;
}

static bool encode(CUtensorMap* map, const void* base, int64_t rows, int cols, int64_t pitch, int box_rows) {
  EncodeFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)}, strides[1] = {static_cast<cuuint64_t>(pitch)};
  const cuuint32_t box[2] = {kBlock, static_cast<cuuint32_t>(box_rows)}, estr[2] = {1, 1};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The plan, gone over once for a shape (some 2 us) as long as this thread has no other one in its place.
static bool plan_for(const TcShape& c, TcPlan* p) {
  struct Known {
    TcShape shape;
    TcPlan plan;
    bool good;
  };
  static thread_local Known known[16] = {};
  Known& k = known[(static_cast<uint64_t>(c.N) * 7 + c.O * 3u + c.I) % 16];
  if (k.shape.E != c.E || k.shape.O != c.O || k.shape.I != c.I || k.shape.ragged != c.ragged || k.shape.N != c.N) {   // (E is 0 in an empty place)
    k.good = plan_tc(c, &k.plan);
    k.shape = c;
  }
  *p = k.plan;
  return k.good;
}

pipe_status linear_tc(const Call& call, cudaStream_t stream) {
  const grp::Call& c = call.c;
  TcArgs p;
  if (!plan_for(TcShape{c.E, c.O, c.I, c.offsets != nullptr, c.N}, &p)) return PIPE_ERR_UNSUPPORTED;
  p.call = call;
  p.wide_y = !(reinterpret_cast<uintptr_t>(c.y) & 15) && c.ldy % (call.dtype == PIPE_DTYPE_FP32 ? 4 : 8) == 0;
  CUtensorMap wmap, xmap;
  if (!encode(&wmap, call.w, static_cast<int64_t>(c.E) * c.O, c.I, call.ldw, p.TM) || !encode(&xmap, c.x, c.N, c.I, c.ldx, p.TN / p.cg)) return grp::runtime_failed();
  void (*k)(TcArgs, CUtensorMap, CUtensorMap) =
      call.dtype == PIPE_DTYPE_FP32 ? tc_kernel<Fp32>(p.cg) : (call.dtype == PIPE_DTYPE_BF16 ? tc_kernel<Bf16>(p.cg) : tc_kernel<Fp16>(p.cg));
  if (!grp::allow_dynamic_smem(reinterpret_cast<const void*>(k), kMaxSmem)) return grp::runtime_failed();
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = p.cg * p.split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(static_cast<unsigned>(p.teams * p.cg * p.split));
  cfg.blockDim = dim3(64 + 32 * p.drain);
  cfg.dynamicSmemBytes = p.smem;
  cfg.stream = stream;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (cudaLaunchKernelEx(&cfg, k, p, wmap, xmap) != cudaSuccess) return grp::runtime_failed();
  count_launch(1);
  return launch_status();
}

}  // namespace i8
}  // namespace pipe
