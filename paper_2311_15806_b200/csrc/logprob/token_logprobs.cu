// Log probabilities of given tokens, entropy and top alternatives (definition: pipe_token_logprobs in include/pipe.h), the simplest form:
// a block per row that reads it once for the largest logit, once for the sums and once for every alternative.
#include "../group/group_common.cuh"

namespace pipe {
namespace lpb {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.44269504f, kLn2 = 0.69314718f;

struct Args {
  const void* logits;
  int64_t T, ldl;
  int V;
  float scale;
  const int32_t* tokens;
  int n;
  float* logprobs;
  float* entropy;
  int k;
  int32_t* top;
  float* top_logprobs;
  int* status;
};

template <int SRC>
__device__ __forceinline__ float logit(const void* row, int64_t i) {
  if (SRC == PIPE_DTYPE_FP32) return __ldcg(static_cast<const float*>(row) + i);
  const uint16_t h = __ldcg(static_cast<const uint16_t*>(row) + i);
  return SRC == PIPE_DTYPE_BF16 ? grp::Bf16::to_float(h) : grp::Fp16::to_float(h);
}
// Keys that order like the numbers, -0 and 0 alike.
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float number_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

template <int SRC>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(const Args a) {
  __shared__ unsigned long long best_s;
  __shared__ float red[2][kThreads / 32];
  __shared__ int bad_s;
  grid_wait();
  grid_release();
  const int64_t t = blockIdx.x;
  const void* row = static_cast<const uint8_t*>(a.logits) + t * a.ldl * (SRC == PIPE_DTYPE_FP32 ? 4 : 2);
  if (threadIdx.x == 0) bad_s = 0, best_s = 0;
  __syncthreads();
  float m = -INFINITY;
  bool bad = false;
  for (int i = threadIdx.x; i < a.V; i += kThreads) {
    const float l = logit<SRC>(row, i);
    if (!(l <= 3.402823466e38f)) bad = true;
    m = fmaxf(m, l);
  }
  if (bad) bad_s = 1;
  m = number_of(__reduce_max_sync(0xffffffffu, key_of(m)));
  if ((threadIdx.x & 31) == 0) red[0][threadIdx.x >> 5] = m;
  __syncthreads();
  for (int w = 0; w < kThreads / 32; ++w) m = fmaxf(m, red[0][w]);
  bad = bad_s != 0;
  const bool none = m == -INFINITY;
  if (bad && threadIdx.x == 0) raise_status(a.status, PIPE_ERR_NONFINITE);
  const float c = a.scale * kLog2e;
  float s = 0.f, h = 0.f;
  for (int i = threadIdx.x; i < a.V; i += kThreads) {
    const float d = fmaxf(logit<SRC>(row, i) - m, -1e30f), e = exp2f(d * c);
    s += e;
    h += d * e;
  }
  __syncthreads();
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o), h += __shfl_xor_sync(0xffffffffu, h, o);
  if ((threadIdx.x & 31) == 0) red[0][threadIdx.x >> 5] = s, red[1][threadIdx.x >> 5] = h;
  __syncthreads();
  s = h = 0.f;
  for (int w = 0; w < kThreads / 32; ++w) s += red[0][w], h += red[1][w];
  const float logs = logf(s), nan = __int_as_float(0x7FC00000);
  auto logprob = [&](float l) { return bad ? nan : (none || l == -INFINITY ? -INFINITY : (0.5f * l - 0.5f * m) * a.scale * 2.f - logs); };
  for (int j = threadIdx.x; j < a.n; j += kThreads) {
    const int tok = __ldcg(a.tokens + t * a.n + j);
    a.logprobs[t * a.n + j] = tok >= 0 && tok < a.V ? logprob(logit<SRC>(row, tok)) : 0.f;
  }
  if (a.entropy && threadIdx.x == 0) a.entropy[t] = bad ? nan : (none ? 0.f : logs - a.scale * h / s);
  unsigned long long last = ~0ull;
  for (int j = 0; j < a.k; ++j) {
    unsigned long long best = 0;
    for (int i = threadIdx.x; i < a.V; i += kThreads) {
      const float l = logit<SRC>(row, i);
      const unsigned long long k = (static_cast<unsigned long long>(key_of(l)) << 32) | (0xFFFFFFFFu - i);
      if (l != -INFINITY && k < last && k > best) best = k;
    }
    atomicMax(&best_s, best);
    __syncthreads();
    last = best_s;
    __syncthreads();
    if (threadIdx.x == 0) {
      best_s = 0;
      const bool some = last != 0 && !bad;
      if (a.top) a.top[t * a.k + j] = some ? static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(last)) : -1;
      if (a.top_logprobs) a.top_logprobs[t * a.k + j] = some ? logprob(number_of(static_cast<uint32_t>(last >> 32))) : (bad ? nan : -INFINITY);
    }
    __syncthreads();
  }
}

}  // namespace lpb
}  // namespace pipe

using namespace pipe;

extern "C" pipe_status pipe_token_logprobs(const void* d_logits, int32_t dtype, int64_t T, int32_t V, int64_t ldl, float scale,
                                           const int32_t* d_tokens, int32_t n, float* d_logprobs, float* d_entropy, int32_t k, int32_t* d_top,
                                           float* d_top_logprobs, void* stream) {
  constexpr int64_t kMost = int64_t{1} << 30;
  if (dtype < PIPE_DTYPE_BF16 || dtype > PIPE_DTYPE_FP32) return PIPE_ERR_INVALID_ARG;
  if (T < 0 || T > kMost || V < 1 || V > kMost || n < 0 || n > 1 << 20 || T * n > int64_t{1} << 40 || k < 0 || k > PIPE_MAX_TOP) return PIPE_ERR_INVALID_ARG;
  if (!(scale >= 0x1p-20f) || !(scale <= 0x1p20f)) return PIPE_ERR_INVALID_ARG;
  if (ldl < V || ldl >= int64_t{1} << 32) return PIPE_ERR_INVALID_ARG;
  if (n == 0 ? d_tokens || d_logprobs : T > 0 && (!d_tokens || !d_logprobs)) return PIPE_ERR_INVALID_ARG;
  if (k == 0 ? d_top || d_top_logprobs : T > 0 && !d_top && !d_top_logprobs) return PIPE_ERR_INVALID_ARG;
  if (T > 0 && !d_logits) return PIPE_ERR_INVALID_ARG;
  auto misaligned = [](const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; };
  if (misaligned(d_logits, dtype == PIPE_DTYPE_FP32 ? 4 : 2) || misaligned(d_tokens, 4) || misaligned(d_logprobs, 4) || misaligned(d_entropy, 4) ||
      misaligned(d_top, 4) || misaligned(d_top_logprobs, 4))
    return PIPE_ERR_ALIGNMENT;
  if (T == 0) return PIPE_OK;
  lpb::Args a = {d_logits, T, ldl, V, scale, d_tokens, n, d_logprobs, d_entropy, k, d_top, d_top_logprobs, device_status_word()};
  if (!a.status) return grp::runtime_failed();
  const auto kern = dtype == PIPE_DTYPE_FP32 ? lpb::logprobs_kernel<PIPE_DTYPE_FP32>
                                             : (dtype == PIPE_DTYPE_BF16 ? lpb::logprobs_kernel<PIPE_DTYPE_BF16> : lpb::logprobs_kernel<PIPE_DTYPE_FP16>);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (launch_overlapped(kern, dim3(static_cast<unsigned>(T)), lpb::kThreads, 1, true, s, a) != cudaSuccess) return grp::runtime_failed();
  count_launch(1);
  take_expansion_mark(s);
  return launch_status();
}
