// The router's choice dealt to the experts, and the experts' outputs joined (definitions: pipe_expert_rows, pipe_expert_combine
// in include/pipe.h).
#include "group_common.cuh"

namespace pipe {
namespace grp {

// ---- rows by expert: a stable counting sort.  Every warp owns a run of the choice and counts its experts in a row of shared memory
// of its own; the counts become first slots by a prefix over the warps and the experts; then every warp walks its run again, 32 places
// at a time, equal experts among them ranked by a match.  Integer counts only, so no order of atomics shows.  Bound by latency: up to
// kROne places one CTA does all of it.  Beyond that the walks are the blocks' of a grid, between them one CTA's prefix over the blocks
// (262144 places on 256 experts: one cluster of eight CTAs 41 us).  What the three launches hand on, the counts and then the first
// slots of every block, lies in that block's own part of d_slots, which it overwrites at last.
constexpr int kROne = 8192;       // most places of the one-launch form
constexpr int kRBlock = 2048;     // places of a block (the last one: up to twice that), at least PIPE_MAX_EXPERTS
static_assert(kRBlock >= PIPE_MAX_EXPERTS, "a block's part of d_slots holds a count per expert");

struct RowsArgs {
  const int32_t* choice;
  int n, k, E;           // n = T * k places
  int blocks;
  int32_t *offsets, *rows, *slots;
};

// Counts of this warp's run, one per expert.
__device__ __forceinline__ void count_run(const RowsArgs& a, int begin, int end, int32_t* count) {
  const int lane = threadIdx.x & 31;
  for (int e = lane; e < a.E; e += 32) count[e] = 0;
  __syncwarp();
#pragma unroll 4
  for (int i = begin + lane; i < end; i += 32) {
    const int e = __ldcg(a.choice + i);
    if (e >= 0 && e < a.E) atomicAdd(count + e, 1);
  }
}
// Places this warp's run; next[e]: the slot of the run's next place of expert e.
__device__ __forceinline__ void place_run(const RowsArgs& a, int begin, int end, int32_t* next) {
  const int lane = threadIdx.x & 31;
  int coming = begin + lane < end ? __ldcg(a.choice + begin + lane) : -1;
  for (int i0 = begin; i0 < end; i0 += 32) {
    const int i = i0 + lane;
    int e = coming;
    coming = i + 32 < end ? __ldcg(a.choice + i + 32) : -1;
    if (e < 0 || e >= a.E) e = -1;
    const uint32_t same = __match_any_sync(0xffffffffu, e);
    const int at = e >= 0 ? next[e] + __popc(same & ((1u << lane) - 1)) : -1;
    __syncwarp();
    if (e >= 0 && lane == 31 - __clz(same)) next[e] = at + 1;
    __syncwarp();
    if (i < end) {
      a.slots[i] = at;
      if (at >= 0) a.rows[at] = i / a.k;
    }
  }
}
// smem[w * E + e]: counts of WARPS warps -> the counts of the warps before; their sum is returned.
template <int WARPS>
__device__ __forceinline__ int prefix_warps(int32_t* smem, int E, int e) {
  int v[WARPS], run = 0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) v[w] = smem[w * E + e];
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    smem[w * E + e] = run;
    run += v[w];
  }
  return run;
}
// Exclusive prefix of one value per thread over 1024 threads; `all`: their sum.
__device__ __forceinline__ int prefix_block(int v, int32_t* sums, int& all) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int upto = v;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, upto, d);
    if (lane >= d) upto += u;
  }
  if (lane == 31) sums[warp] = upto;
  __syncthreads();
  int before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < 32; ++w) {
    before += w < warp ? sums[w] : 0;
    all += sums[w];
  }
  return before + upto - v;
}

__global__ void __launch_bounds__(1024) expert_rows_kernel(RowsArgs a) {
  extern __shared__ int32_t smem[];   // [32][E]
  __shared__ int32_t sums[32];
  const int tid = threadIdx.x, warp = tid >> 5;
  const int per = (a.n + 1023) / 1024 * 32;
  const int begin = min(warp * per, a.n), end = min(begin + per, a.n);
  grid_wait();
  grid_release();
  count_run(a, begin, end, smem + warp * a.E);
  __syncthreads();
  const int mine = tid < a.E ? prefix_warps<32>(smem, a.E, tid) : 0;   // E <= 1024: one expert per thread
  int all;
  const int first = prefix_block(mine, sums, all);
  if (tid < a.E) {
    a.offsets[tid] = first;
    if (tid == a.E - 1) a.offsets[a.E] = all;
#pragma unroll
    for (int w = 0; w < 32; ++w) smem[w * a.E + tid] += first;
  }
  __syncthreads();
  place_run(a, begin, end, smem + warp * a.E);
}

__device__ __forceinline__ int block_places(const RowsArgs& a) { return blockIdx.x == a.blocks - 1 ? a.n - static_cast<int>(blockIdx.x) * kRBlock : kRBlock; }

__global__ void __launch_bounds__(256) expert_count_kernel(RowsArgs a) {
  extern __shared__ int32_t smem[];   // [E]
  grid_wait();
  grid_release();
  const int begin = static_cast<int>(blockIdx.x) * kRBlock, end = begin + block_places(a);
  for (int e = threadIdx.x; e < a.E; e += 256) smem[e] = 0;
  __syncthreads();
#pragma unroll 8
  for (int i = begin + threadIdx.x; i < end; i += 256) {
    const int e = __ldcg(a.choice + i);
    if (e >= 0 && e < a.E) atomicAdd(smem + e, 1);
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += 256) a.slots[begin + e] = smem[e];
}

// The blocks' counts of every expert -> their first slots: neighbouring threads have neighbouring experts (a warp per expert with the
// blocks as lanes, every load 32 sectors, took 70 us for 128 blocks of 256 experts), groups of threads a share of the blocks each.
__global__ void __launch_bounds__(1024) expert_scan_kernel(RowsArgs a) {
  __shared__ int32_t part[1024], total[PIPE_MAX_EXPERTS], sums[32];
  const int tid = threadIdx.x;
  grid_wait();
  grid_release();
  const int width = (a.E + 31) & ~31, groups = 1024 / width;
  const int group = tid / width, e = tid - group * width;
  const bool here = group < groups && e < a.E;
  const int b0 = static_cast<int>(static_cast<int64_t>(a.blocks) * group / groups), b1 = static_cast<int>(static_cast<int64_t>(a.blocks) * (group + 1) / groups);
  int run = 0;
  if (here) {
#pragma unroll 8
    for (int b = b0; b < b1; ++b) run += __ldcg(a.slots + b * kRBlock + e);
  }
  part[tid] = run;
  __syncthreads();
  int mine = 0;
  if (tid < a.E)
    for (int g = 0; g < groups; ++g) mine += part[g * width + tid];
  int all;
  const int first = prefix_block(mine, sums, all);
  if (tid < a.E) {
    a.offsets[tid] = first;
    if (tid == a.E - 1) a.offsets[a.E] = all;
    total[tid] = first;
  }
  __syncthreads();
  if (here) {
    int at = total[e];
    for (int g = 0; g < group; ++g) at += part[g * width + e];
    int b = b0;
    for (; b + 8 <= b1; b += 8) {   // (eight loads in flight)
      int v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = __ldcg(a.slots + (b + i) * kRBlock + e);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        a.slots[(b + i) * kRBlock + e] = at;
        at += v[i];
      }
    }
    for (; b < b1; ++b) {
      const int v = __ldcg(a.slots + b * kRBlock + e);
      a.slots[b * kRBlock + e] = at;
      at += v;
    }
  }
}

__global__ void __launch_bounds__(256) expert_place_kernel(RowsArgs a) {
  extern __shared__ int32_t smem[];   // [8][E]
  const int warp = threadIdx.x >> 5;
  grid_wait();
  grid_release();
  const int first = static_cast<int>(blockIdx.x) * kRBlock, places = block_places(a);
  const int per = (places + 255) / 256 * 32;
  const int begin = first + min(warp * per, places), end = min(begin + per, first + places);
  count_run(a, begin, end, smem + warp * a.E);
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += 256) {
    prefix_warps<8>(smem, a.E, e);
    const int at = __ldcg(a.slots + first + e);
#pragma unroll
    for (int w = 0; w < 8; ++w) smem[w * a.E + e] += at;
  }
  __syncthreads();   // (the block's first slots are read: its part of d_slots may be overwritten)
  place_run(a, begin, end, smem + warp * a.E);
}

// ---- a token's experts joined: every output is k products in binary32; bound by reading the k rows.  8192 tokens of 6 rows of 2048:
// 46 us, 5.1 TB/s (with eight rows in flight per thread: 57).
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
  if (T > (int64_t{1} << 30) / k) return PIPE_ERR_UNSUPPORTED;   // (a place's number plus a step of a walk stays below 2^31)
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
  a.blocks = a.n / grp::kRBlock;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  auto launch = [&](void (*kernel)(grp::RowsArgs), int blocks, int threads, int smem) {
    if (smem > 48 * 1024 && !grp::allow_dynamic_smem(reinterpret_cast<const void*>(kernel), 32 * PIPE_MAX_EXPERTS * 4)) return false;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, a) != cudaSuccess) return false;
    count_launch(1);
    return true;
  };
  const bool ok = a.n <= grp::kROne ? launch(grp::expert_rows_kernel, 1, 1024, 32 * experts * 4)
                                    : launch(grp::expert_count_kernel, a.blocks, 256, experts * 4) && launch(grp::expert_scan_kernel, 1, 1024, 0) &&
                                          launch(grp::expert_place_kernel, a.blocks, 256, 8 * experts * 4);
  if (!ok) return grp::runtime_failed();
  take_expansion_mark(s);
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
  if (launch_overlapped(kern, dim3(static_cast<unsigned>(blocks)), grp::kCThreads, 1, true, s, a) != cudaSuccess) return grp::runtime_failed();
  count_launch(1);
  take_expansion_mark(s);
  return launch_status();
}
