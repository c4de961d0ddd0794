// Products of a 4-bit layer with group scales with a few rows (pipe_group_linear, pipe_expert_linear).
//
// With a few rows the product is bound by reading the codes once, and by the instructions that widen them.  The warp-level MMA
// m16n8k16 takes the weights as its 16-row and the activations as its 8-column operand: the codes minus their zero point are small
// integers, exact in bf16 and fp16, so a group's sum is formed in binary32 from exact operands and the scale enters once per group
// and output, in binary32 too.  A run of 32 codes of a row is 16 bytes, 4 per lane of a quad: the lane's 8 codes are its operands
// of two MMAs, and the activations that meet them are 8 neighbouring values of the row, 16 bytes.
// A CTA takes one tile of 16 * MT channels and one unit of rows; its four warps, and the CTAs of a cluster where there are few tiles,
// share the reduction axis in steps of 128 codes.  A warp's activations are asked into L1, which the CTAs of an SM share, at once;
// codes, scales and zero points of its next steps are in flight in registers (copies through shared memory cost more instructions
// than the arithmetic).  Sums are added in a fixed order.
// Measured, back to back in a graph (weights then in L2): 4096 -> 11008 on one row 8.5 us (23.3 MB), on 8 rows 10.3, on 16 rows 13.3; 64
// experts 2048 -> 1408, 48 rows on 31 of them, 18.4 (46 MB), 22.5 among other calls, where the weights come from HBM.  Bound by the
// latency of a CTA's chain (unit, addresses, first codes, sums): issue slots are 20 to 36 % busy.
#include "group_common.cuh"

namespace pipe {
namespace grp {

constexpr int kSWarps = 4;
constexpr int kSThreads = 32 * kSWarps;

struct SmallArgs {
  Call c;
  int steps;      // steps of 128 codes: ceil(I / 128); 0 where there are no activations at all
  int units;      // the most there can be
};

// Unit u of the rows cut into units of at most `per` rows of one expert: every lane of the calling warp gets the answer; false: there
// are fewer units.  Offsets are taken as clamped to [0, N] and ascending, whatever they hold.
__device__ __forceinline__ bool find_unit(const Call& c, int u, int per, Unit& out) {
  if (!c.offsets) {
    out.e = 0;
    out.lo = u * per;
    out.hi = out.lo + per < c.N ? out.lo + per : static_cast<int>(c.N);
    return out.lo < c.N;
  }
  const int lane = threadIdx.x & 31, N = static_cast<int>(c.N);
  int before = 0, top = 0;
  for (int e0 = 0; e0 < c.E; e0 += 32) {
    const int e = e0 + lane;
    int lo = 0, hi = 0;
    if (e < c.E) {
      lo = min(max(__ldcg(c.offsets + e), 0), N);
      hi = min(max(__ldcg(c.offsets + e + 1), 0), N);
    }
    make_ascending(lo, hi, top, e < c.E, min(31, c.E - 1 - e0));
    const int mine = (hi - lo + per - 1) / per;
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += v;
    }
    const int total = __shfl_sync(0xffffffffu, upto, 31);
    if (u < before + total) {
      const int src = __ffs(__ballot_sync(0xffffffffu, upto > u - before)) - 1;
      const int tile = u - before - __shfl_sync(0xffffffffu, upto - mine, src);
      out.e = e0 + src;
      out.lo = __shfl_sync(0xffffffffu, lo, src) + tile * per;
      out.hi = min(out.lo + per, __shfl_sync(0xffffffffu, hi, src));
      return true;
    }
    before += total;
  }
  return false;
}

// NT: 8-column tiles (rows of a unit: 8 NT); KPG: runs of 32 codes per group.
// TAIL: I is no multiple of 128, the last step has fewer runs.
template <class H, int MT, int NT, int KPG, bool ASYM, bool TAIL>
__global__ void __launch_bounds__(kSThreads, MT == 1 ? 5 : (MT * NT == 2 ? 4 : 3)) group_small_kernel(SmallArgs p) {
  constexpr int kM = 16 * MT, kN = 8 * NT, kP = kM + 4;   // kP: pitch of a row of sums (its writers then meet different banks)
  constexpr int kGroups = 4 / KPG;                         // groups of a step
  constexpr int kAhead = MT == 1 ? 4 : 2;                  // steps of codes in registers
  constexpr int kMeta = 2;                                 // steps of scales and zero points
  __shared__ float part[kSWarps * kN * kP];
  const Call& c = p.c;
  const int ctas = cluster_ctas(), rank = cluster_rank();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
  const uint32_t tile = ctas == 1 ? blockIdx.x : blockIdx.x / static_cast<uint32_t>(ctas);
  const int o0 = static_cast<int>(tile) * kM;
  const int slices = ctas * kSWarps, slice = rank * kSWarps + warp;
  const int step0 = static_cast<int>(static_cast<uint32_t>(p.steps) * slice / slices);   // (steps < 2^26, slices <= 32)
  const int step1 = static_cast<int>(static_cast<uint32_t>(p.steps) * (slice + 1) / slices);
  const int groups = c.KB / KPG;
  const int64_t run_bytes = static_cast<int64_t>(c.O) * 16;

  if (!c.offsets) {
    // this warp's codes on their way into L2 before the wait (asking for a line that is still being written does no harm)
    const int n = (step1 - step0) * 4 * 2 * MT;
    for (int i = lane; i < n; i += 32) {
      const int kb = 4 * step0 + i / (2 * MT), o = o0 + 8 * (i % (2 * MT));
      if (kb < c.KB && o < c.O) asm volatile("prefetch.global.L2 [%0];" ::"l"(c.codes + kb * run_bytes + o * int64_t{16}));
    }
  }
  grid_wait();
  grid_release();
  for (int un = blockIdx.y; un < p.units; un += gridDim.y) {
    Unit u;
    if (!find_unit(c, un, kN, u)) break;   // (the same answer in every CTA of the cluster)
    const int count = u.hi - u.lo;
    // This lane's rows of the MMA operands: channels o0 + gid + 8 m.  Of channels beyond the layer nothing is read: their sums, of
    // whatever the registers hold, are not stored.  Rows of activations: behind the unit's last row it, not stored; in the place of one
    // whose index lies outside some row, its sums made zero below.
    bool real[2 * MT];
#pragma unroll
    for (int m = 0; m < 2 * MT; ++m) real[m] = o0 + 8 * m + gid < c.O;
    const uint8_t* code[4];   // the four runs of the next step to be asked for
#pragma unroll
    for (int b = 0; b < 4; ++b) code[b] = c.codes + (static_cast<int64_t>(u.e) * c.KB + 4 * step0 + b) * run_bytes + (o0 + gid) * int64_t{16} + 4 * tig;
    const int64_t meta0 = (static_cast<int64_t>(u.e) * groups + step0 * kGroups) * c.O + o0 + gid;
    const uint16_t* scales = static_cast<const uint16_t*>(c.scales) + meta0;
    const uint8_t* zeros = ASYM ? c.zeros + meta0 : nullptr;
    const uint16_t* x[NT];
    uint32_t inside[NT];   // bit 4 n: row n of the column tile exists
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int s = u.lo + min(8 * n + gid, count - 1);
      int64_t r = c.rows ? __ldcg(c.rows + s) : s;
      const bool ok = r >= 0 && r < c.T;
      inside[n] = __ballot_sync(0xffffffffu, ok);
      if (!ok) r = 0;
      x[n] = static_cast<const uint16_t*>(c.x) + r * c.ldx + 128 * step0 + 8 * tig;
    }
    uint32_t w[kAhead][4][2 * MT] = {};
    auto load = [&](int step, uint32_t (&d)[4][2 * MT]) {
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        if (!TAIL || 4 * step + b < c.KB) {
#pragma unroll
          for (int m = 0; m < 2 * MT; ++m)
            if (real[m]) d[b][m] = __ldcg(reinterpret_cast<const uint32_t*>(code[b] + 128 * m));
        }
        code[b] += 4 * run_bytes;
      }
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (step0 + i < step1) load(step0 + i, w[i]);
    {   // this warp's share of the rows on their way into L1: four lanes have each row's address, eight of a row's lines are asked for at a time
      const int lines = (min(c.I, 128 * step1) - 128 * step0 + 63) / 64;   // of 128 bytes
#pragma unroll
      for (int n = 0; n < NT; ++n)
        if (8 * n + gid < count)
          for (int i = tig; i < lines; i += 4) asm volatile("prefetch.global.L1 [%0];" ::"l"(x[n] - 8 * tig + 64 * i));
    }

    float acc[MT][NT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m][n][i] = 0.f;

    uint32_t sc[kMeta][kGroups][2 * MT] = {}, zp[kMeta][kGroups][2 * MT] = {};
    auto fetch = [&](int step, uint32_t (&s)[kGroups][2 * MT], uint32_t (&z)[kGroups][2 * MT]) {
#pragma unroll
      for (int f = 0; f < kGroups; ++f) {
        if (!TAIL || step * kGroups + f < groups) {
#pragma unroll
          for (int m = 0; m < 2 * MT; ++m)
            if (real[m]) {
              s[f][m] = __ldcg(scales + 8 * m);
              if (ASYM) z[f][m] = __ldcg(zeros + 8 * m);
            }
        }
        scales += c.O;
        if (ASYM) zeros += c.O;
      }
    };
    auto compute = [&](int step, const uint32_t (&d)[4][2 * MT], const uint32_t (&s)[kGroups][2 * MT], const uint32_t (&z)[kGroups][2 * MT]) {
      const int runs = c.KB - 4 * step;   // fewer than 4: the last step of a layer whose I is no multiple of 128
#pragma unroll
      for (int f = 0; f < kGroups; ++f) {
        if (TAIL && f * KPG >= runs) break;
        float sum[MT][NT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[m][n][k] = 0.f;
#pragma unroll
        for (int b = f * KPG; b < (f + 1) * KPG; ++b) {
          uint4 xv[NT];
#pragma unroll
          for (int n = 0; n < NT; ++n) xv[n] = *reinterpret_cast<const uint4*>(x[n] + 32 * b);
#pragma unroll
          for (int m = 0; m < MT; ++m) {
            uint32_t a[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const uint32_t zz = zero_pair<H>(ASYM ? z[f][2 * m + h] : 8u);
#pragma unroll
              for (int k = 0; k < 4; ++k) a[h][k] = H::add2(code_pair<H>(d[b][2 * m + h], k), zz);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              H::mma(sum[m][n], a[0][0], a[1][0], a[0][1], a[1][1], xv[n].x, xv[n].y);
              H::mma(sum[m][n], a[0][2], a[1][2], a[0][3], a[1][3], xv[n].z, xv[n].w);
            }
          }
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              acc[m][n][k] = fmaf(H::to_float(static_cast<uint16_t>(s[f][2 * m + (k >> 1)])), sum[m][n][k], acc[m][n][k]);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) x[n] += 128;
    };
#pragma unroll
    for (int i = 0; i < kMeta; ++i)
      if (step0 + i < step1) fetch(step0 + i, sc[i], zp[i]);
    int step = step0;
    for (; step + 2 * kAhead <= step1; step += kAhead) {   // (what is asked for is all inside this warp's share)
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        compute(step + i, w[i], sc[i % kMeta], zp[i % kMeta]);
        fetch(step + i + kMeta, sc[i % kMeta], zp[i % kMeta]);
        load(step + i + kAhead, w[i]);
      }
    }
    for (; step < step1; step += kAhead) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (step + i < step1) {
          compute(step + i, w[i], sc[i % kMeta], zp[i % kMeta]);
          if (step + i + kMeta < step1) fetch(step + i + kMeta, sc[i % kMeta], zp[i % kMeta]);
          if (step + i + kAhead < step1) load(step + i + kAhead, w[i]);
        }
    }

    // sums of the warps, then of the CTAs, in ascending order of the axis
    float* to = part + warp * kN * kP;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 8 * n + 2 * tig + (i & 1);
          if (r < count) to[r * kP + 16 * m + gid + 8 * (i >> 1)] = (inside[n] >> (4 * (r & 7))) & 1 ? acc[m][n][i] : 0.f;
        }
    __syncthreads();
    if (ctas > 1) {
      for (int i = threadIdx.x; i < kM * count; i += kSThreads) {
        const int n = i / kM, m = i % kM;
        float v = part[n * kP + m];
#pragma unroll
        for (int k = 1; k < kSWarps; ++k) v += part[(k * kN + n) * kP + m];
        part[n * kP + m] = v;   // (no other thread reads this place)
      }
      cluster_sync();
    }
    for (int i = threadIdx.x + kSThreads * rank; i < kM * count; i += kSThreads * ctas) {   // every CTA finishes a share of the outputs
      const int n = i / kM, m = i % kM, o = o0 + m;
      float v[1] = {0.f};
      if (ctas > 1) {
        for (int k = 0; k < ctas; ++k) v[0] += cluster_load(part + n * kP + m, k);
      } else {
        v[0] = part[n * kP + m];
#pragma unroll
        for (int k = 1; k < kSWarps; ++k) v[0] += part[(k * kN + n) * kP + m];
      }
      if (o < c.O) {
        if (c.bias) v[0] += H::to_float(__ldcg(static_cast<const uint16_t*>(c.bias) + static_cast<int64_t>(u.e) * c.O + o));
        quick_activation(v, c.act);
        static_cast<uint16_t*>(c.y)[static_cast<int64_t>(u.lo + n) * c.ldy + o] = H::from_float(v[0]);
      }
    }
    // no CTA leaves, and none takes another unit, while its sums are being read
    if (ctas > 1) cluster_sync();
    else __syncthreads();
  }
}

using SmallKernel = void (*)(SmallArgs);
template <class H, int MT, int NT, int KPG>
static SmallKernel small_kernel(bool asym, bool tail) {
  if constexpr (KPG == 4) return asym ? group_small_kernel<H, MT, NT, 4, true, false> : group_small_kernel<H, MT, NT, 4, false, false>;
  else if (tail) return asym ? group_small_kernel<H, MT, NT, KPG, true, true> : group_small_kernel<H, MT, NT, KPG, false, true>;
  else return asym ? group_small_kernel<H, MT, NT, KPG, true, false> : group_small_kernel<H, MT, NT, KPG, false, false>;
}
template <class H, int MT, int NT>
static SmallKernel small_kernel(int g, bool asym, bool tail) {
  return g == 32 ? small_kernel<H, MT, NT, 1>(asym, tail) : (g == 64 ? small_kernel<H, MT, NT, 2>(asym, tail) : small_kernel<H, MT, NT, 4>(asym, tail));
}
template <class H>
static SmallKernel small_kernel(int mt, int nt, int g, bool asym, bool tail) {
  return nt == 2 ? small_kernel<H, 2, 2>(g, asym, tail) : (mt == 4 ? small_kernel<H, 4, 1>(g, asym, tail) : (mt == 2 ? small_kernel<H, 2, 1>(g, asym, tail) : small_kernel<H, 1, 1>(g, asym, tail)));
}

pipe_status linear_small(const Call& c, bool bf16, cudaStream_t stream) {
  SmallArgs p;
  p.c = c;
  p.steps = c.T > 0 ? ceil_div(c.KB, 4) : 0;
  const int64_t rows = c.offsets ? ceil_div<int64_t>(c.N, c.E) : c.N;
  const int nt = rows <= 8 ? 1 : 2;
  // Channels of a tile (16 mt) and CTAs that share an axis: a round of CTAs costs some 3 us before its first product (launch, addresses,
  // first loads), and each step of a warp's share 0.3, 0.46 or 0.85 us (mt = 1, 2, 4; two column tiles 0.75).  These are weights that
  // order the choices below, no times: 11008 -> 4096 on 13 rows comes to 11.8 us by them and takes 19.5 to 22.  Measured against them
  // (one token): 4096 -> 11008 mt = 1 alone 8.2 us, with two CTAs to a tile 12.0, mt = 2 alone 9.4; 11008 -> 4096 mt = 2 with four 8.5,
  // with two 10.0, mt = 1 with two 10.7, with four 14.7; 54 units of 2048 -> 1408 mt = 4 18, mt = 2 20, mt = 1 32.
  p.units = static_cast<int>(most_units(c, 8 * nt));
  int mt = 0, ctas = 0;
  int64_t best = 0;
  for (int m = nt; m <= (nt == 2 ? 2 : 4); m *= 2)
    for (int k = 1; k == 1 || (k <= 8 && p.steps >= k * kSWarps); k *= 2) {
      const int per_sm = nt == 2 || m == 4 ? 3 : (m == 2 ? 4 : 5);   // CTAs that an SM holds (by registers)
      const int64_t blocks = p.units * ceil_div<int64_t>(c.O, 16 * m) * k;
      const int64_t step_cost = nt == 2 ? 75 : (m == 1 ? 30 : (m == 2 ? 46 : 85));
      const int64_t cost = ceil_div<int64_t>(blocks, per_sm * kPlanSMs) * (300 + (k > 1 ? 50 : 0) + step_cost * ceil_div(p.steps, k * kSWarps));
      if (!mt || cost < best) {
        best = cost;
        mt = m;
        ctas = k;
      }
    }
  const int64_t tiles = ceil_div(c.O, 16 * mt);
  if (tiles * ctas >= (int64_t{1} << 31)) return PIPE_ERR_UNSUPPORTED;
  const SmallKernel k = bf16 ? small_kernel<Bf16>(mt, nt, c.g, c.zeros != nullptr, c.KB % 4 != 0) : small_kernel<Fp16>(mt, nt, c.g, c.zeros != nullptr, c.KB % 4 != 0);
  const dim3 grid(static_cast<unsigned>(tiles * ctas), static_cast<unsigned>(p.units < 65535 ? p.units : 65535));
  if (launch_overlapped(k, grid, kSThreads, ctas, true, stream, p) != cudaSuccess) return runtime_failed();
  count_launch(1);
  return launch_status();
}

}  // namespace grp
}  // namespace pipe
