// Quantizer of the 4-bit layers with group scales (definition: pipe_group_quantize in include/pipe.h).
//
// One pass: the weights are read once, everything else is written once; bound by HBM.  A thread takes 8 neighbouring weights, 16
// threads a row's 128 (four, two or one group, whose extrema meet by shuffles), a warp two neighbouring rows, whose 16-byte runs
// of codes are then one 32-byte sector.
#include "group_common.cuh"

namespace pipe {
namespace grp {

constexpr int kQThreads = 256;
constexpr int kQRows = kQThreads / 16;   // rows of a block

struct QuantArgs {
  const void* w;
  int64_t ldw, rows;     // rows = E * O
  int O, I, g, groups, KB;
  uint8_t* codes;
  uint16_t* scales;
  uint8_t* zeros;
  float* values;
  int64_t ldv;
  int wide;              // source rows are 16-byte aligned
  int wide_v;            // and so are the rows of values
  int tiles;             // ceil(I / 128)
  int* status;
};

// The integers nearest the exact quotients w / s (s > 0), ties to even.  An estimate rounded by an addition (1.5 * 2^23, where the
// spacing of binary32 is one) is off by one at most.  The remainder w - q s is exact: w has 24 bits, s at most 11 and q few, so the
// remainder, no larger than w unless q is 0, is a whole number of units of w's last place.  Only where it reaches half a step, on a
// tie or where the estimate went wrong, is anything more done.
__device__ __forceinline__ float settle_code(float w, float s, float q) {
  const float r = fmaf(-q, s, w), twice = 2.f * fabsf(r);
  if (twice > s || (twice == s && (static_cast<int>(q) & 1))) q += r > 0.f ? 1.f : -1.f;
  return q;
}
template <int N>
__device__ __forceinline__ void nearest_codes(const float (&w)[N], float s, float inv, bool fast, float (&q)[N]) {
  float edge = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    q[i] = __fsub_rn(__fadd_rn(fast ? __fmul_rn(w[i], inv) : __fdiv_rn(w[i], s), 12582912.f), 12582912.f);
    edge = fmaxf(edge, fabsf(fmaf(-q[i], s, w[i])));
  }
  if (2.f * edge >= s) {
#pragma unroll
    for (int i = 0; i < N; ++i) q[i] = settle_code(w[i], s, q[i]);
  }
}

template <class S>
__device__ __forceinline__ void load8(const S* p, bool wide, float (&v)[8]);
template <>
__device__ __forceinline__ void load8<float>(const float* p, bool wide, float (&v)[8]) {
  if (wide) {
    const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = p[i];
  }
}
template <class H>
__device__ __forceinline__ void load8_half(const uint16_t* p, bool wide, float (&v)[8]) {
  if (wide) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t u[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = H::to_float(static_cast<uint16_t>(u[i] & 0xffffu));
      v[2 * i + 1] = H::to_float(static_cast<uint16_t>(u[i] >> 16));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = H::to_float(p[i]);
  }
}

template <class H, int SRC, bool ASYM>
__global__ void __launch_bounds__(kQThreads) group_quantize_kernel(QuantArgs a) {
  grid_wait();
  grid_release();
  const int64_t row = static_cast<int64_t>(blockIdx.x / a.tiles) * kQRows + (threadIdx.x >> 4);
  const int tile = blockIdx.x % a.tiles;
  const int i0 = tile * 128 + 8 * (threadIdx.x & 15);
  const bool here = row < a.rows && i0 < a.I;
  float w[8];
  if (here) {
    if (SRC == PIPE_DTYPE_FP32) load8<float>(static_cast<const float*>(a.w) + row * a.ldw + i0, a.wide, w);
    else if (SRC == PIPE_DTYPE_BF16) load8_half<Bf16>(static_cast<const uint16_t*>(a.w) + row * a.ldw + i0, a.wide, w);
    else load8_half<Fp16>(static_cast<const uint16_t*>(a.w) + row * a.ldw + i0, a.wide, w);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = 0.f;
  }
  // extrema of the group: of 8 in the thread, then over its 4, 8 or 16 threads
  float lo = 0.f, hi = 0.f;
  bool finite = true;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    finite = finite && fabsf(w[i]) <= 3.402823466e38f;
    if (ASYM) {
      lo = fminf(lo, w[i]);
      hi = fmaxf(hi, w[i]);
    } else {
      hi = fmaxf(hi, fabsf(w[i]));
    }
  }
  for (int d = 1; d < a.g / 8; d <<= 1) {
    hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
    if (ASYM) lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
  }
  const uint16_t sh = H::from_float(ASYM ? __fdiv_rn(__fsub_rn(hi, lo), 15.f) : __fdiv_rn(hi, 7.f));
  const float s = H::to_float(sh);
  finite = finite && s <= 3.402823466e38f;
  if (!finite) raise_status(a.status, PIPE_ERR_NONFINITE);
  const bool fast = quant_step_is_fast(s);
  const float inv = fast ? __frcp_rn(s) : 0.f;
  float z = ASYM ? 0.f : 8.f;
  uint32_t word = ASYM ? 0u : 0x88888888u;
  float c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = 0.f;
  if (s > 0.f && finite) {
    if (ASYM) {
      float first[1] = {-lo}, q[1];
      nearest_codes(first, s, inv, fast, q);
      z = fminf(q[0], 15.f);
    }
    float q[8];
    nearest_codes(w, s, inv, fast, q);
    word = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      c[i] = ASYM ? fminf(fmaxf(q[i], -z), 15.f - z) : fminf(fmaxf(q[i], -7.f), 7.f);
      // (the code in the low bits of a sum on top of 2^23)
      word |= (__float_as_uint(c[i] + (8388608.f + z)) & 15u) << (4 * ((i >> 1) + 4 * (i & 1)));
    }
  }
  if (!here) return;
  const int64_t e = row / a.O;
  const int o = static_cast<int>(row - e * a.O);
  *reinterpret_cast<uint32_t*>(a.codes + ((e * a.KB + (i0 >> 5)) * a.O + o) * 16 + ((i0 >> 3) & 3) * 4) = word;
  if (i0 % a.g == 0) {
    const int64_t at = (e * a.groups + i0 / a.g) * a.O + o;
    a.scales[at] = sh;
    if (ASYM) a.zeros[at] = static_cast<uint8_t>(z);
  }
  if (a.values) {
    float* v = a.values + row * a.ldv + i0;
    if (a.wide_v) {
      *reinterpret_cast<float4*>(v) = make_float4(c[0] * s, c[1] * s, c[2] * s, c[3] * s);
      *reinterpret_cast<float4*>(v + 4) = make_float4(c[4] * s, c[5] * s, c[6] * s, c[7] * s);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = c[i] * s;
    }
  }
}

template <class H, bool ASYM>
static void (*quantize_kernel(int src))(QuantArgs) {
  return src == PIPE_DTYPE_FP32 ? group_quantize_kernel<H, PIPE_DTYPE_FP32, ASYM>
                                : (src == PIPE_DTYPE_BF16 ? group_quantize_kernel<H, PIPE_DTYPE_BF16, ASYM> : group_quantize_kernel<H, PIPE_DTYPE_FP16, ASYM>);
}

}  // namespace grp
}  // namespace pipe

using namespace pipe;

extern "C" pipe_status pipe_group_quantize(const pipe_group_desc* desc, const void* d_W, int32_t w_dtype, int64_t ldw, void* d_codes,
                                           void* d_scales, uint8_t* d_zeros, float* d_values, int64_t ldv, void* stream) {
  pipe_group_layout_t lay;
  const pipe_status st = pipe_group_layout(desc, &lay);
  if (st != PIPE_OK) return st;
  if (w_dtype < PIPE_DTYPE_BF16 || w_dtype > PIPE_DTYPE_FP32) return PIPE_ERR_INVALID_ARG;
  if (!d_W || !d_codes || !d_scales || (d_zeros != nullptr) != (desc->asymmetric != 0)) return PIPE_ERR_INVALID_ARG;
  if (ldw < desc->in_features || (d_values && ldv < desc->in_features)) return PIPE_ERR_INVALID_ARG;
  const uintptr_t size = w_dtype == PIPE_DTYPE_FP32 ? 4 : 2;
  if ((reinterpret_cast<uintptr_t>(d_W) & (size - 1)) || (reinterpret_cast<uintptr_t>(d_codes) & 15) ||
      (reinterpret_cast<uintptr_t>(d_scales) & 1) || (reinterpret_cast<uintptr_t>(d_values) & 3))
    return PIPE_ERR_ALIGNMENT;
  grp::QuantArgs a;
  a.w = d_W;
  a.ldw = ldw;
  a.rows = static_cast<int64_t>(desc->experts) * desc->out_features;
  a.O = desc->out_features;
  a.I = desc->in_features;
  a.g = desc->group_size;
  a.groups = lay.groups;
  a.KB = a.I / 32;
  a.codes = static_cast<uint8_t*>(d_codes);
  a.scales = static_cast<uint16_t*>(d_scales);
  a.zeros = d_zeros;
  a.values = d_values;
  a.ldv = ldv;
  a.wide = !(reinterpret_cast<uintptr_t>(d_W) & 15) && (ldw * size) % 16 == 0;
  a.wide_v = d_values && !(reinterpret_cast<uintptr_t>(d_values) & 15) && ldv % 4 == 0;
  a.tiles = ceil_div(a.I, 128);
  const int64_t blocks = ceil_div<int64_t>(a.rows, grp::kQRows) * a.tiles;
  if (blocks >= (int64_t{1} << 31)) return PIPE_ERR_UNSUPPORTED;
  a.status = device_status_word();
  if (!a.status) return PIPE_ERR_CUDA;
  const bool bf16 = desc->dtype == PIPE_DTYPE_BF16;
  void (*k)(grp::QuantArgs) = bf16 ? (desc->asymmetric ? grp::quantize_kernel<grp::Bf16, true>(w_dtype) : grp::quantize_kernel<grp::Bf16, false>(w_dtype))
                                   : (desc->asymmetric ? grp::quantize_kernel<grp::Fp16, true>(w_dtype) : grp::quantize_kernel<grp::Fp16, false>(w_dtype));
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (launch_overlapped(k, dim3(static_cast<unsigned>(blocks)), grp::kQThreads, 1, true, s, a) != cudaSuccess) return PIPE_ERR_CUDA;
  count_launch(1);
  take_expansion_mark(s);
  return launch_status();
}
