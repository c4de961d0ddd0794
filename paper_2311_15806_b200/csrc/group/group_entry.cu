// Entry points of the 4-bit layers with group scales: checks of arguments and the choice of a kernel.
#include <mutex>

#include "group_common.cuh"

namespace pipe {
namespace grp {

constexpr int kMostFeatures = 1 << 29;       // channels, doubled, are coordinates of 32 bits
constexpr int64_t kMostRows = int64_t{1} << 30;

static pipe_status check_desc(const pipe_group_desc* d) {
  if (!d) return PIPE_ERR_INVALID_ARG;
  if (d->experts < 1 || d->experts > PIPE_MAX_EXPERTS || d->out_features < 1 || d->in_features < 1) return PIPE_ERR_INVALID_ARG;
  if (d->out_features > kMostFeatures || d->in_features > kMostFeatures) return PIPE_ERR_INVALID_ARG;
  if (d->dtype != PIPE_DTYPE_BF16 && d->dtype != PIPE_DTYPE_FP16) return PIPE_ERR_INVALID_ARG;
  if (d->asymmetric != 0 && d->asymmetric != 1) return PIPE_ERR_INVALID_ARG;
  if (d->group_size < 1) return PIPE_ERR_INVALID_ARG;
  if (d->group_size != 32 && d->group_size != 64 && d->group_size != 128) return PIPE_ERR_UNSUPPORTED;
  if (d->in_features % d->group_size) return PIPE_ERR_SHAPE;
  return PIPE_OK;
}

bool allow_dynamic_smem(const void* kernel, int most) {
  constexpr int kMost = 4096;   // kernels (some twenty) times devices; beyond, the limit is set again by every call, to the same value
  static std::mutex lock;
  static struct { const void* kernel; int device; } done[kMost];
  static int n = 0;
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess) return false;
  const std::lock_guard<std::mutex> held(lock);
  for (int i = 0; i < n; ++i)
    if (done[i].kernel == kernel && done[i].device == device) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess) return false;
  if (n < kMost) done[n++] = {kernel, device};
  return true;
}

static bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

// What both products check alike; fills the call but for its rows.
static pipe_status check_product(const pipe_group_desc* desc, const void* codes, const void* scales, const uint8_t* zeros, const void* x,
                                 int64_t T, int64_t ldx, const void* bias, int32_t act, int64_t N, void* y, int64_t ldy, Call* c) {
  const pipe_status st = check_desc(desc);
  if (st != PIPE_OK) return st;
  if (T < 0 || N < 0 || T > kMostRows || N > kMostRows) return PIPE_ERR_INVALID_ARG;
  if (act < PIPE_ACT_IDENTITY || act > PIPE_ACT_SIGMOID) return PIPE_ERR_INVALID_ARG;
  if (!codes || !scales || (zeros != nullptr) != (desc->asymmetric != 0)) return PIPE_ERR_INVALID_ARG;
  if ((T > 0 && !x) || (N > 0 && !y)) return PIPE_ERR_INVALID_ARG;
  if (ldx < desc->in_features || ldy < desc->out_features) return PIPE_ERR_INVALID_ARG;
  if (misaligned(codes, 16) || misaligned(scales, 2) || misaligned(x, 16) || ldx % 8 || misaligned(bias, 2) || misaligned(y, 2))
    return PIPE_ERR_ALIGNMENT;
  c->E = desc->experts; c->O = desc->out_features; c->I = desc->in_features; c->g = desc->group_size;
  c->KB = c->I / 32;
  c->codes = static_cast<const uint8_t*>(codes);
  c->scales = scales;
  c->zeros = zeros;
  c->x = x; c->T = T; c->ldx = ldx;
  c->rows = nullptr; c->offsets = nullptr;
  c->N = N;
  c->bias = bias;
  c->act = act;
  c->y = y; c->ldy = ldy;
  c->status = nullptr;
  return PIPE_OK;
}

static pipe_status product(Call& c, bool bf16, cudaStream_t stream) {
  if (c.N == 0) return PIPE_OK;
  c.status = device_status_word();
  if (!c.status) return runtime_failed();
  // Up to 16 rows (on experts: on average, rounded up) go to the kernel that holds them in one unit and whose weights are exact.  Either
  // side of the border (us): 4096 -> 11008 on 16 rows 13.3 there, on 17 rows 17.4 on the tensor cores; 11008 -> 4096 the other way round,
  // 13 rows 19.5 to 22 there, 17 rows 16.4 on the tensor cores.
  const int64_t rows = c.offsets ? ceil_div<int64_t>(c.N, c.E) : c.N;
  pipe_status st = rows > 16 ? linear_tc(c, bf16, stream) : PIPE_ERR_UNSUPPORTED;
  if (st == PIPE_ERR_UNSUPPORTED) st = linear_small(c, bf16, stream);
  if (st == PIPE_OK) take_expansion_mark(stream);
  return st;
}

}  // namespace grp
}  // namespace pipe

using namespace pipe;

extern "C" pipe_status pipe_group_layout(const pipe_group_desc* desc, pipe_group_layout_t* h_out) {
  const pipe_status st = grp::check_desc(desc);
  if (st != PIPE_OK) return st;
  if (!h_out) return PIPE_ERR_INVALID_ARG;
  const uint64_t rows = static_cast<uint64_t>(desc->experts) * desc->out_features;
  h_out->groups = desc->in_features / desc->group_size;
  h_out->codes_bytes = rows * desc->in_features / 2;
  h_out->scales_bytes = rows * h_out->groups * 2;
  h_out->zeros_bytes = desc->asymmetric ? rows * h_out->groups : 0;
  return PIPE_OK;
}

extern "C" pipe_status pipe_group_linear(const pipe_group_desc* desc, const void* d_codes, const void* d_scales, const uint8_t* d_zeros,
                                         const void* d_x, int64_t T, int64_t ldx, const void* d_bias, int32_t activation, void* d_y,
                                         int64_t ldy, void* stream) {
  grp::Call c;
  const pipe_status st = grp::check_product(desc, d_codes, d_scales, d_zeros, d_x, T, ldx, d_bias, activation, T, d_y, ldy, &c);
  if (st != PIPE_OK) return st;
  if (c.E != 1) return PIPE_ERR_SHAPE;
  return grp::product(c, desc->dtype == PIPE_DTYPE_BF16, static_cast<cudaStream_t>(stream));
}

extern "C" pipe_status pipe_expert_linear(const pipe_group_desc* desc, const void* d_codes, const void* d_scales, const uint8_t* d_zeros,
                                          const void* d_x, int64_t T, int64_t ldx, const int32_t* d_rows, const int32_t* d_offsets,
                                          int64_t N, const void* d_bias, int32_t activation, void* d_y, int64_t ldy, void* stream) {
  grp::Call c;
  const pipe_status st = grp::check_product(desc, d_codes, d_scales, d_zeros, d_x, T, ldx, d_bias, activation, N, d_y, ldy, &c);
  if (st != PIPE_OK) return st;
  if (!d_offsets) return PIPE_ERR_INVALID_ARG;
  if (grp::misaligned(d_offsets, 4) || grp::misaligned(d_rows, 4)) return PIPE_ERR_ALIGNMENT;
  c.rows = d_rows;
  c.offsets = d_offsets;
  return grp::product(c, desc->dtype == PIPE_DTYPE_BF16, static_cast<cudaStream_t>(stream));
}
