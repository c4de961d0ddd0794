// Products of a 4-bit layer with group scales with a few rows (pipe_group_linear, pipe_expert_linear).
//
// With a few rows the product is bound by reading the codes once.  The warp-level MMA m16n8k16 takes the weights as its 16-row and
// the activations as its 8-column operand: the codes minus their zero point are small integers, exact in bf16 and fp16, so a
// group's sum is formed in binary32 from exact operands and the scale enters once per group and output, in binary32 too.  A run of
// 32 codes of a row is 16 bytes, 4 per lane of a quad: the lane's 8 codes are its operands of two MMAs, and the activations that
// meet them are 8 neighbouring values of the row, 16 bytes.  A warp takes 16 * MT output channels and every step of 128 codes of
// its share of the reduction axis; the warps of a CTA and the CTAs of a cluster share the axis and add their sums in a fixed
// order, in shared memory and across it.
#include "group_common.cuh"

namespace pipe {
namespace grp {

constexpr int kSWarps = 8;

struct SmallArgs {
  Call c;
  int tiles;    // row tiles of the layer: ceil(O / (16 MT))
  int steps;    // steps of 128 codes: ceil(I / 128)
};

// NT: 8-column tiles (tokens of a unit: 8 NT); KPG: runs of 32 codes per group.
template <class H, int MT, int NT, int KPG, bool ASYM>
__global__ void __launch_bounds__(32 * kSWarps) group_small_kernel(SmallArgs p) {
  constexpr int kM = 16 * MT, kN = 8 * NT;
  constexpr int kFlush = 4 / KPG;            // groups of a step
  __shared__ float part[kSWarps][kN][kM + 1];
  const Call& c = p.c;
  const int ctas = cluster_ctas(), rank = cluster_rank();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, gid = lane >> 2, tig = lane & 3;
  const int64_t block = blockIdx.x / ctas;
  const int tile = static_cast<int>(block % p.tiles);
  const int o0 = tile * kM;
  const int slices = ctas * kSWarps, slice = rank * kSWarps + warp;
  const int step0 = static_cast<int>(static_cast<int64_t>(p.steps) * slice / slices), step1 = static_cast<int>(static_cast<int64_t>(p.steps) * (slice + 1) / slices);

  grid_wait();
  grid_release();
  Unit u;
  if (!find_unit(c, block / p.tiles, kN, u)) return;   // (the same answer in every CTA of the cluster)

  // rows of this lane's MMA operands; one beyond the layer reads the last one instead and is not stored
  uint32_t row[2 * MT];
#pragma unroll
  for (int m = 0; m < 2 * MT; ++m) {
    const int o = o0 + 16 * (m >> 1) + 8 * (m & 1) + gid;
    row[m] = static_cast<uint32_t>(o < c.O ? o : c.O - 1);
  }
  const uint8_t* codes = c.codes + static_cast<int64_t>(u.e) * c.KB * c.O * 16 + 4 * tig;
  const int groups = c.KB / KPG;
  const uint16_t* scales = static_cast<const uint16_t*>(c.scales) + static_cast<int64_t>(u.e) * groups * c.O;
  const uint8_t* zeros = ASYM ? c.zeros + static_cast<int64_t>(u.e) * groups * c.O : nullptr;
  const uint16_t* x[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int64_t s = u.lo + 8 * n + gid;
    x[n] = nullptr;
    if (s < u.hi) {
      const int64_t r = c.rows ? __ldcg(c.rows + s) : s;
      if (r >= 0 && r < c.T) x[n] = static_cast<const uint16_t*>(c.x) + r * c.ldx + 8 * tig;
    }
  }

  float acc[MT][NT][4];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[m][n][i] = 0.f;

  uint32_t w[2][4][2 * MT];
  auto load = [&](int step, uint32_t (&d)[4][2 * MT]) {
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int kb = 4 * step + b;
      if (kb < c.KB) {
        const uint8_t* run = codes + static_cast<int64_t>(kb) * c.O * 16;
#pragma unroll
        for (int m = 0; m < 2 * MT; ++m) d[b][m] = __ldcg(reinterpret_cast<const uint32_t*>(run + static_cast<uint64_t>(row[m]) * 16));
      } else {
#pragma unroll
        for (int m = 0; m < 2 * MT; ++m) d[b][m] = 0;
      }
    }
  };
  auto compute = [&](int step, const uint32_t (&d)[4][2 * MT]) {
#pragma unroll
    for (int f = 0; f < kFlush; ++f) {
      if (4 * step + f * KPG >= c.KB) break;   // (the last step of a layer whose I is no multiple of 128)
      const int64_t at = static_cast<int64_t>((4 * step + f * KPG) / KPG) * c.O;
      float s[2 * MT];
      uint32_t z[2 * MT];
#pragma unroll
      for (int m = 0; m < 2 * MT; ++m) {
        s[m] = H::to_float(__ldcg(scales + at + row[m]));
        z[m] = zero_pair<H>(ASYM ? __ldcg(zeros + at + row[m]) : 8u);
      }
      float sum[MT][NT][4];
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[m][n][i] = 0.f;
#pragma unroll
      for (int b = 0; b < KPG; ++b) {
        uint4 xv[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          xv[n] = make_uint4(0, 0, 0, 0);
          if (x[n]) xv[n] = *reinterpret_cast<const uint4*>(x[n] + (4 * step + f * KPG + b) * 32);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          uint32_t a[2][4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            a[0][i] = H::sub2(code_pair<H>(d[f * KPG + b][2 * m], i), z[2 * m]);
            a[1][i] = H::sub2(code_pair<H>(d[f * KPG + b][2 * m + 1], i), z[2 * m + 1]);
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
          for (int i = 0; i < 4; ++i) acc[m][n][i] = fmaf(s[2 * m + (i >> 1)], sum[m][n][i], acc[m][n][i]);
    }
  };
  if (step0 < step1) load(step0, w[0]);
  for (int step = step0; step < step1; step += 2) {
    if (step + 1 < step1) load(step + 1, w[1]);
    compute(step, w[0]);
    if (step + 1 < step1) {
      if (step + 2 < step1) load(step + 2, w[0]);
      compute(step + 1, w[1]);
    }
  }

  // sums of the warps, then of the CTAs, in ascending order of the axis
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) part[warp][8 * n + 2 * tig + (i & 1)][16 * m + gid + 8 * (i >> 1)] = acc[m][n][i];
  __syncthreads();
  for (int i = threadIdx.x; i < kM * kN; i += 32 * kSWarps) {
    const int n = i / kM, m = i % kM;
    float v = part[0][n][m];
#pragma unroll
    for (int k = 1; k < kSWarps; ++k) v += part[k][n][m];
    part[0][n][m] = v;   // (no other thread reads this place)
  }
  if (ctas > 1) cluster_sync();
  else __syncthreads();
  // every CTA finishes a share of the outputs
  for (int i = threadIdx.x + 32 * kSWarps * rank; i < kM * kN; i += 32 * kSWarps * ctas) {
    const int n = i / kM, m = i % kM, o = o0 + m;
    const int64_t s = u.lo + n;
    float v = 0.f;
    for (int k = 0; k < ctas; ++k) v += cluster_load(&part[0][n][m], k);
    if (s < u.hi && o < c.O) {
      if (c.bias) v += H::to_float(__ldcg(static_cast<const uint16_t*>(c.bias) + static_cast<int64_t>(u.e) * c.O + o));
      static_cast<uint16_t*>(c.y)[s * c.ldy + o] = H::from_float(apply_activation(v, c.act));
    }
  }
  if (ctas > 1) cluster_sync();   // no CTA leaves while another reads its sums
}

template <class H, int MT, int NT, int KPG>
static void (*small_kernel(bool asym))(SmallArgs) {
  return asym ? group_small_kernel<H, MT, NT, KPG, true> : group_small_kernel<H, MT, NT, KPG, false>;
}
template <class H, int MT, int NT>
static void (*small_kernel(int g, bool asym))(SmallArgs) {
  return g == 32 ? small_kernel<H, MT, NT, 1>(asym) : (g == 64 ? small_kernel<H, MT, NT, 2>(asym) : small_kernel<H, MT, NT, 4>(asym));
}

pipe_status linear_small(const Call& c, bool bf16, cudaStream_t stream) {
  SmallArgs p;
  p.c = c;
  p.steps = ceil_div(c.KB, 4);
  const bool asym = c.zeros != nullptr;
  const int64_t rows = c.offsets ? ceil_div<int64_t>(c.N, c.E) : c.N;
  const int nt = rows <= 8 ? 1 : 2;
  const int mt = nt;
  p.tiles = ceil_div(c.O, 16 * mt);
  const int64_t blocks = most_units(c, 8 * nt) * p.tiles;
  int ctas = 1;
  while (ctas < 8 && blocks * ctas < 2 * kPlanSMs && p.steps >= 2 * ctas * kSWarps) ctas *= 2;
  if (blocks * ctas >= (int64_t{1} << 31)) return PIPE_ERR_UNSUPPORTED;
  void (*k)(SmallArgs) = bf16 ? (nt == 1 ? small_kernel<Bf16, 1, 1>(c.g, asym) : small_kernel<Bf16, 2, 2>(c.g, asym))
                              : (nt == 1 ? small_kernel<Fp16, 1, 1>(c.g, asym) : small_kernel<Fp16, 2, 2>(c.g, asym));
  if (launch_overlapped(k, dim3(static_cast<unsigned>(blocks * ctas)), 32 * kSWarps, ctas, true, stream, p) != cudaSuccess) return PIPE_ERR_CUDA;
  count_launch(1);
  return launch_status();
}

}  // namespace grp
}  // namespace pipe
