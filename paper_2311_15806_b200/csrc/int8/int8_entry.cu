// Entry points of the products of the 8-bit integer layers: checks of arguments and the choice of a kernel.
#include "int8_common.cuh"

namespace pipe {
namespace i8 {

constexpr int64_t kMostRows = int64_t{1} << 30;
constexpr int kMostFeatures = 1 << 29;

static bool misaligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }

static pipe_status check_desc(const pipe_int8_desc* d) {
  if (!d) return PIPE_ERR_INVALID_ARG;
  if (d->experts < 1 || d->experts > PIPE_MAX_EXPERTS || d->out_features < 1 || d->in_features < 1) return PIPE_ERR_INVALID_ARG;
  if (d->out_features > kMostFeatures || static_cast<int64_t>(d->experts) * d->out_features > kMostRows) return PIPE_ERR_INVALID_ARG;
  if (d->dtype < PIPE_DTYPE_BF16 || d->dtype > PIPE_DTYPE_FP32) return PIPE_ERR_INVALID_ARG;
  if (d->in_features > PIPE_INT8_MAX_FEATURES) return PIPE_ERR_ACC_OVERFLOW;
  return PIPE_OK;
}

static pipe_status product(const pipe_int8_desc* desc, const int8_t* codes, int64_t ldw, const float* scales, const int8_t* xq, int64_t ldx,
                           const float* sx, const int32_t* offsets, int64_t N, const void* bias, int32_t act, void* y, int64_t ldy,
                           cudaStream_t stream) {
  if (N < 0 || N > kMostRows) return PIPE_ERR_INVALID_ARG;
  if (act < PIPE_ACT_IDENTITY || act > PIPE_ACT_SIGMOID) return PIPE_ERR_INVALID_ARG;
  if (!codes || !scales || (N > 0 && (!xq || !sx || !y))) return PIPE_ERR_INVALID_ARG;
  if (ldw < desc->in_features || ldx < desc->in_features || ldy < desc->out_features) return PIPE_ERR_INVALID_ARG;
  const uintptr_t size = desc->dtype == PIPE_DTYPE_FP32 ? 4 : 2;
  if (misaligned(codes, 16) || ldw % 16 || misaligned(xq, 16) || ldx % 16 || misaligned(scales, 4) || misaligned(sx, 4) ||
      misaligned(bias, size) || misaligned(y, size) || misaligned(offsets, 4))
    return PIPE_ERR_ALIGNMENT;
  // (row pitches are strides of tensor copies, below 2^40 bytes)
  if (ldw >= int64_t{1} << 40 || ldx >= int64_t{1} << 40 || ldy >= int64_t{1} << 40) return PIPE_ERR_INVALID_ARG;
  if (N == 0) return PIPE_OK;
  Call c = {};
  c.c.E = desc->experts; c.c.O = desc->out_features; c.c.I = desc->in_features;
  c.c.x = xq; c.c.T = N; c.c.ldx = ldx;
  c.c.offsets = offsets; c.c.N = N;
  c.c.bias = bias; c.c.act = act;
  c.c.y = y; c.c.ldy = ldy;
  c.w = codes; c.ldw = ldw; c.sw = scales; c.sx = sx;
  c.dtype = desc->dtype;
  c.c.status = device_status_word();
  if (!c.c.status) return grp::runtime_failed();
  const pipe_status st = linear_tc(c, stream);
  if (st == PIPE_OK) take_expansion_mark(stream);
  return st;
}

}  // namespace i8
}  // namespace pipe

using namespace pipe;

extern "C" pipe_status pipe_int8_linear(const pipe_int8_desc* desc, const int8_t* d_codes, int64_t ldw, const float* d_scales, const int8_t* d_xq,
                                        int64_t T, int64_t ldx, const float* d_sx, const void* d_bias, int32_t activation, void* d_y, int64_t ldy,
                                        void* stream) {
  const pipe_status st = i8::check_desc(desc);
  if (st != PIPE_OK) return st;
  if (desc->experts != 1) return PIPE_ERR_SHAPE;
  return i8::product(desc, d_codes, ldw, d_scales, d_xq, ldx, d_sx, nullptr, T, d_bias, activation, d_y, ldy, static_cast<cudaStream_t>(stream));
}

extern "C" pipe_status pipe_int8_expert_linear(const pipe_int8_desc* desc, const int8_t* d_codes, int64_t ldw, const float* d_scales,
                                               const int8_t* d_xq, int64_t ldx, const float* d_sx, const int32_t* d_offsets, int64_t N,
                                               const void* d_bias, int32_t activation, void* d_y, int64_t ldy, void* stream) {
  const pipe_status st = i8::check_desc(desc);
  if (st != PIPE_OK) return st;
  if (!d_offsets) return PIPE_ERR_INVALID_ARG;
  return i8::product(desc, d_codes, ldw, d_scales, d_xq, ldx, d_sx, d_offsets, N, d_bias, activation, d_y, ldy, static_cast<cudaStream_t>(stream));
}
