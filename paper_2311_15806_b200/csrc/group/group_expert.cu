// The router's choice dealt to the experts, and the experts' outputs joined (definitions: pipe_expert_rows, pipe_expert_combine
// in include/pipe.h).
#include "group_common.cuh"

namespace pipe {
namespace grp {

// ---- rows by expert: a stable counting sort in one launch.  Every warp owns a run of the choice and counts its experts in a row
// of shared memory of its own; the counts become first slots by a prefix over the warps, the CTAs of the cluster (distributed
// shared memory) and the experts; then every warp walks its run again, 32 places at a time, equal experts among them ranked by a
// match.  Integer counts only, so no order of atomics shows.  Bound by latency: two walks and three barriers.
constexpr int kRWarps = 32;
constexpr int kRCtas = 8;

struct RowsArgs {
  const int32_t* choice;
  int n, k, E;           // n = T * k places
  int per;               // places of a warp, a multiple of 32
  int32_t *offsets, *rows, *slots;
};

__global__ void __launch_bounds__(32 * kRWarps) expert_rows_kernel(RowsArgs a) {
  extern __shared__ int32_t smem[];   // count[kRWarps][E], total[E], first[E]
  const int rank = cluster_rank(), ctas = cluster_ctas();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int32_t *count = smem + warp * a.E, *total = smem + kRWarps * a.E, *first = total + a.E;
  __shared__ int32_t sums[kRWarps];
  grid_wait();
  grid_release();
  for (int e = lane; e < a.E; e += 32) count[e] = 0;
  __syncwarp();
  const int64_t begin = static_cast<int64_t>(rank * kRWarps + warp) * a.per;
  const int64_t end = begin + a.per < a.n ? begin + a.per : a.n;
  for (int64_t i = begin + lane; i < end; i += 32) {
    const int e = __ldcg(a.choice + i);
    if (e >= 0 && e < a.E) atomicAdd(count + e, 1);
  }
  __syncthreads();
  for (int e = tid; e < a.E; e += 32 * kRWarps) {
    int run = 0;
    for (int w = 0; w < kRWarps; ++w) {
      const int v = smem[w * a.E + e];
      smem[w * a.E + e] = run;
      run += v;
    }
    total[e] = run;
  }
  cluster_sync();
  // E <= PIPE_MAX_EXPERTS = the block's threads: one expert per thread
  int before = 0, all = 0;
  if (tid < a.E)
    for (int r = 0; r < ctas; ++r) {
      const int v = cluster_load(total + tid, r);
      before += r < rank ? v : 0;
      all += v;
    }
  int upto = all;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += v;
  }
  if (lane == 31) sums[warp] = upto;
  __syncthreads();
  int base = 0;
  for (int w = 0; w < warp; ++w) base += sums[w];
  if (tid < a.E) {
    first[tid] = base + upto - all + before;
    if (rank == 0) {
      a.offsets[tid] = base + upto - all;
      if (tid == a.E - 1) a.offsets[a.E] = base + upto;
    }
  }
  cluster_sync();   // (also: no CTA leaves while another reads its totals)
  for (int64_t i0 = begin; i0 < end; i0 += 32) {
    const int64_t i = i0 + lane;
    int e = i < end ? __ldcg(a.choice + i) : -1;
    if (e < 0 || e >= a.E) e = -1;
    const uint32_t same = __match_any_sync(0xffffffffu, e);
    const int at = e >= 0 ? first[e] + count[e] + __popc(same & ((1u << lane) - 1)) : -1;
    __syncwarp();
    if (e >= 0 && lane == __ffs(same) - 1) count[e] += __popc(same);
    __syncwarp();
    if (i < end) {
      a.slots[i] = at;
      if (at >= 0) a.rows[at] = static_cast<int32_t>(i) / a.k;
    }
  }
}

// ---- a token's experts joined: every output is k products in binary32; bound by reading the k rows.
struct CombineArgs {
  const uint16_t* y;
  int64_t N, ldy;
  const int32_t* slots;
  const float* weights;
  int64_t T;
  int k, O, per_row;   // per_row: threads of a token
  uint16_t* out;
  int64_t ldo;
};
constexpr int kCThreads = 256;

template <class H, int V>   // V outputs per thread: 8 (16-byte rows) or 1
__global__ void __launch_bounds__(kCThreads) expert_combine_kernel(CombineArgs a) {
  grid_wait();
  grid_release();
  const int64_t id = static_cast<int64_t>(blockIdx.x) * kCThreads + threadIdx.x;
  const int64_t t = id / a.per_row;
  if (t >= a.T) return;
  const int o = static_cast<int>(id - t * a.per_row) * V;
  float v[V];
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = 0.f;
#pragma unroll 4
  for (int j = 0; j < a.k; ++j) {
    const int s = __ldcg(a.slots + t * a.k + j);
    const float w = __ldcg(a.weights + t * a.k + j);
    if (s < 0 || s >= a.N) continue;
    const uint16_t* p = a.y + s * a.ldy + o;
    if (V == 8) {
      const uint4 q = __ldcg(reinterpret_cast<const uint4*>(p));
      const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < V; ++i) v[i] = fmaf(w, H::to_float(static_cast<uint16_t>(u[i / 2] >> (16 * (i & 1)))), v[i]);
    } else {
      v[0] = fmaf(w, H::to_float(__ldcg(p)), v[0]);
    }
  }
  uint16_t* p = a.out + t * a.ldo + o;
  if (V == 8) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = H::from_float(v[(2 * i) % V]) | (static_cast<uint32_t>(H::from_float(v[(2 * i + 1) % V])) << 16);
    *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
  } else {
    *p = H::from_float(v[0]);
  }
}

}  // namespace grp
}  // namespace pipe

using namespace pipe;

extern "C" pipe_status pipe_expert_rows(const int32_t* d_choice, int64_t T, int32_t k, int32_t experts, int32_t* d_offsets, int32_t* d_rows,
                                        int32_t* d_slots, void* stream) {
  if (T < 0 || k < 1 || experts < 1 || experts > PIPE_MAX_EXPERTS) return PIPE_ERR_INVALID_ARG;
  if (T > (int64_t{0x7fffffff} - 1) / k) return PIPE_ERR_UNSUPPORTED;
  if (!d_offsets || (T > 0 && (!d_choice || !d_rows || !d_slots))) return PIPE_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(d_choice) | reinterpret_cast<uintptr_t>(d_offsets) | reinterpret_cast<uintptr_t>(d_rows) |
       reinterpret_cast<uintptr_t>(d_slots)) & 3)
    return PIPE_ERR_ALIGNMENT;
  grp::RowsArgs a;
  a.choice = d_choice;
  a.n = static_cast<int>(T * k);
  a.k = k;
  a.E = experts;
  a.offsets = d_offsets;
  a.rows = d_rows;
  a.slots = d_slots;
  // one CTA while its warps have few steps of 32 places each: a cluster costs two barriers across SMs
  const int ctas = a.n <= 8 * 32 * grp::kRWarps ? 1 : grp::kRCtas;
  a.per = static_cast<int>(round_up<int64_t>(ceil_div<int64_t>(a.n, ctas * grp::kRWarps), 32));
  const size_t smem = static_cast<size_t>(grp::kRWarps + 2) * experts * 4;
  if (smem > 48 * 1024 &&
      cudaFuncSetAttribute(grp::expert_rows_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess)
    return PIPE_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(32 * grp::kRWarps);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  if (cudaLaunchKernelEx(&cfg, grp::expert_rows_kernel, a) != cudaSuccess) return PIPE_ERR_CUDA;
  count_launch(1);
  take_expansion_mark(cfg.stream);
  return launch_status();
}

extern "C" pipe_status pipe_expert_combine(const void* d_y, int64_t N, int64_t ldy, const int32_t* d_slots, const float* d_weights, int64_t T,
                                           int32_t k, int32_t O, int32_t dtype, void* d_out, int64_t ldo, void* stream) {
  if (T < 0 || N < 0 || k < 1 || O < 1 || (dtype != PIPE_DTYPE_BF16 && dtype != PIPE_DTYPE_FP16)) return PIPE_ERR_INVALID_ARG;
  if (T >= (int64_t{1} << 31) || N >= (int64_t{1} << 31)) return PIPE_ERR_INVALID_ARG;
  if (ldy < O || ldo < O) return PIPE_ERR_INVALID_ARG;
  if (T == 0) return PIPE_OK;
  if ((N > 0 && !d_y) || !d_slots || !d_weights || !d_out) return PIPE_ERR_INVALID_ARG;
  if ((reinterpret_cast<uintptr_t>(d_y) & 1) || (reinterpret_cast<uintptr_t>(d_out) & 1) || (reinterpret_cast<uintptr_t>(d_slots) & 3) ||
      (reinterpret_cast<uintptr_t>(d_weights) & 3))
    return PIPE_ERR_ALIGNMENT;
  grp::CombineArgs a;
  a.y = static_cast<const uint16_t*>(d_y);
  a.N = N;
  a.ldy = ldy;
  a.slots = d_slots;
  a.weights = d_weights;
  a.T = T;
  a.k = k;
  a.O = O;
  a.out = static_cast<uint16_t*>(d_out);
  a.ldo = ldo;
  const bool wide = !(reinterpret_cast<uintptr_t>(d_y) & 15) && !(reinterpret_cast<uintptr_t>(d_out) & 15) && ldy % 8 == 0 && ldo % 8 == 0 && O % 8 == 0;
  a.per_row = wide ? O / 8 : O;
  const int64_t blocks = ceil_div<int64_t>(T * a.per_row, grp::kCThreads);
  if (blocks >= (int64_t{1} << 31)) return PIPE_ERR_UNSUPPORTED;
  const bool bf16 = dtype == PIPE_DTYPE_BF16;
  void (*kern)(grp::CombineArgs) = wide ? (bf16 ? grp::expert_combine_kernel<grp::Bf16, 8> : grp::expert_combine_kernel<grp::Fp16, 8>)
                                        : (bf16 ? grp::expert_combine_kernel<grp::Bf16, 1> : grp::expert_combine_kernel<grp::Fp16, 1>);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (launch_overlapped(kern, dim3(static_cast<unsigned>(blocks)), grp::kCThreads, 1, true, s, a) != cudaSuccess) return PIPE_ERR_CUDA;
  count_launch(1);
  take_expansion_mark(s);
  return launch_status();
}
