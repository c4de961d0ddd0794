// Quantizer of the 4-bit layers with group scales (definition: pipe_group_quantize in include/pipe.h).
//
// One pass: the weights are read once, everything else is written once; bound by HBM.  16 threads take a row's 128 weights, each the
// four from 4 l on and the four from 64 + 4 l on, so that every load and store of a warp is of whole neighbouring lines (eight
// neighbours a thread left half-written sectors: the values of 11008 x 4096 at 3.5 TB/s); the extrema of one, two or four groups meet
// by shuffles; neighbouring threads join their codes to words.  A warp has two neighbouring rows, whose 16-byte runs of codes are then
// one sector.  A block walks its share of the rows, the next row's weights in flight.  11008 x 4096 from bf16, asymmetric, with values:
// 65 us, 4.5 TB/s; its issue slots are 79 % busy.
#include "group_common.cuh"

namespace pipe {
namespace grp {

constexpr int kQThreads = 256;
constexpr int kQRows = kQThreads / 16;   // rows of a block

struct QuantArgs {
  const void* w;
  int64_t ldw;
  int O, I, g, groups, KB;
  uint8_t* codes;
  uint16_t* scales;
  uint8_t* zeros;
  float* values;
  int64_t ldv;
  int wide;              // source rows are 16-byte aligned
  int wide_v;            // and so are the rows of values
  int* status;
};

// The integers nearest the exact quotients w / s (s > 0), ties to even.  An estimate rounded by an addition (1.5 * 2^23, where the
// spacing of binary32 is one) is off by one at most.  The remainder w - q s is exact: w has 24 bits, s at most 11 and q few, so the
// remainder, no larger than w unless q is 0, is a whole number of units of w's last place.  Only where it reaches half a step, on a
// tie or where the estimate went wrong, is anything more done.
__device__ __noinline__ float settle_code(float w, float s, float q) {
  const float r = fmaf(-q, s, w), twice = 2.f * fabsf(r);
  if (twice > s || (twice == s && (static_cast<int>(q) & 1))) q += r > 0.f ? 1.f : -1.f;
  return q;
}
__device__ __noinline__ float rounded_quotient(float w, float s) { return rintf(__fdiv_rn(w, s)); }
template <int N>
__device__ __forceinline__ void nearest_codes(const float (&w)[N], float s, float inv, bool fast, float (&q)[N]) {
  if (fast) {
#pragma unroll
    for (int i = 0; i < N; ++i) q[i] = __fsub_rn(__fmaf_rn(w[i], inv, 12582912.f), 12582912.f);
  } else {   // a step without a usable reciprocal
#pragma unroll
    for (int i = 0; i < N; ++i) q[i] = rounded_quotient(w[i], s);
  }
  float edge = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) edge = fmaxf(edge, fabsf(fmaf(-q[i], s, w[i])));
  if (2.f * edge >= s) {
#pragma unroll
    for (int i = 0; i < N; ++i) q[i] = settle_code(w[i], s, q[i]);   // (out of line: a few times in a million)
  }
}

// Four neighbouring weights as they lie in memory, and as numbers.
template <int SRC>
struct Four {
  uint32_t u[SRC == PIPE_DTYPE_FP32 ? 4 : 2];
  __device__ __forceinline__ void load(const uint8_t* from, bool wide) {
    if constexpr (SRC == PIPE_DTYPE_FP32) {
      if (wide) {
        const uint4 a = __ldcg(reinterpret_cast<const uint4*>(from));
        u[0] = a.x; u[1] = a.y; u[2] = a.z; u[3] = a.w;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) u[i] = __ldcg(reinterpret_cast<const uint32_t*>(from) + i);
      }
    } else {
      if (wide) {
        const uint2 a = __ldcg(reinterpret_cast<const uint2*>(from));
        u[0] = a.x; u[1] = a.y;
      } else {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(from);
#pragma unroll
        for (int i = 0; i < 2; ++i) u[i] = __ldcg(p + 2 * i) | (static_cast<uint32_t>(__ldcg(p + 2 * i + 1)) << 16);
      }
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (uint32_t& v : u) v = 0;
  }
  __device__ __forceinline__ void numbers(float* v) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (SRC == PIPE_DTYPE_FP32) {
        v[i] = __uint_as_float(u[i]);
      } else {
        const uint16_t h = static_cast<uint16_t>(u[i >> 1] >> (16 * (i & 1)));
        v[i] = SRC == PIPE_DTYPE_BF16 ? Bf16::to_float(h) : Fp16::to_float(h);
      }
    }
  }
};

// What a thread makes of N of a group's weights, lo and hi being the group's extrema (hi alone: its largest magnitude).
template <class H, bool ASYM, int N>
__device__ __forceinline__ bool quantize_part(const float* w, float lo, float hi, uint16_t& sh, float& s, float& z, float (&c)[N]) {
  sh = H::from_float(ASYM ? __fdiv_rn(__fsub_rn(hi, lo), 15.f) : __fdiv_rn(hi, 7.f));
  s = H::to_float(sh);
  const bool finite = s <= 3.402823466e38f;
  z = ASYM ? 0.f : 8.f;
#pragma unroll
  for (int i = 0; i < N; ++i) c[i] = 0.f;
  if (s > 0.f && finite) {
    const bool fast = quant_step_is_fast(s);
    const float inv = fast ? __frcp_rn(s) : 0.f;
    if (ASYM) {
      const float first[1] = {-lo};
      float q[1];
      nearest_codes(first, s, inv, fast, q);
      z = fminf(q[0], 15.f);
    }
    float v[N], q[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = w[i];
    nearest_codes(v, s, inv, fast, q);
#pragma unroll
    for (int i = 0; i < N; ++i) c[i] = ASYM ? fminf(fmaxf(q[i], -z), 15.f - z) : fminf(fmaxf(q[i], -7.f), 7.f);
  }
  return finite;
}

template <class H, int SRC, bool ASYM, int G>   // G: weights of a group
__global__ void __launch_bounds__(kQThreads) group_quantize_kernel(QuantArgs a) {
  grid_wait();
  grid_release();
  const int l = threadIdx.x & 15, tile = static_cast<int>(blockIdx.x) * 128, e = static_cast<int>(blockIdx.z);
  // addresses of this thread's first row, and what takes them to its next one
  int o = static_cast<int>(blockIdx.y) * kQRows + (threadIdx.x >> 4);
  const int step = static_cast<int>(gridDim.y) * kQRows;
  constexpr int kSize = SRC == PIPE_DTYPE_FP32 ? 4 : 2;
  const int64_t row = static_cast<int64_t>(e) * a.O + o;
  const uint8_t* src = static_cast<const uint8_t*>(a.w) + (row * a.ldw + tile + 4 * l) * kSize;
  const int word_at = tile + 64 * (l & 1) + 4 * (l & ~1);   // the first code of this thread's word of eight
  uint8_t* code = a.codes + ((static_cast<int64_t>(e) * a.KB + (word_at >> 5)) * a.O + o) * 16 + ((word_at >> 3) & 3) * 4;
  int64_t meta[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) meta[h] = (static_cast<int64_t>(e) * a.groups + (tile + 64 * h + 4 * l) / G) * a.O + o;
  float* value = a.values + (a.values ? row * a.ldv + tile + 4 * l : 0);
  const bool inside[2] = {tile + 4 * l < a.I, tile + 64 + 4 * l < a.I};   // (I is a multiple of 32: a thread's four are inside or not)
  const int64_t src_step = step * a.ldw * kSize, value_step = step * a.ldv;
  // the next row's weights are asked for before this one's are looked at
  Four<SRC> next[2];
  auto ask = [&](int row_o) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      if (row_o < a.O && inside[h]) next[h].load(src + 64 * h * kSize, a.wide);
      else next[h].zero();
    }
    src += src_step;
  };
  ask(o);
  // (whole warps go on while one of their rows is left)
  for (; __any_sync(0xffffffffu, o < a.O); o += step, code += step * 16ll, meta[0] += step, meta[1] += step, value += value_step) {
    float w[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) next[h].numbers(w + 4 * h);
    ask(o + step);
    float lo[2], hi[2], most = 0.f;   // most: the largest magnitude, a NaN if there is one
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float* v = w + 4 * h;
      const float m = max3_abs_nan(max3_abs_nan(v[0], v[1], 0.f), v[2], v[3]);
      most = max3_abs_nan(most, m, 0.f);
      lo[h] = ASYM ? fminf(fminf(fminf(v[0], v[1]), fminf(v[2], v[3])), 0.f) : 0.f;
      hi[h] = ASYM ? max3(max3(v[0], v[1], 0.f), v[2], v[3]) : m;
    }
    bool finite = most <= 3.402823466e38f;
    if constexpr (G == 128) {   // one group: both halves
      hi[0] = hi[1] = fmaxf(hi[0], hi[1]);
      lo[0] = lo[1] = fminf(lo[0], lo[1]);
    }
#pragma unroll
    for (int d = 1; d < (G == 32 ? 8 : 16); d <<= 1) {
      hi[0] = fmaxf(hi[0], __shfl_xor_sync(0xffffffffu, hi[0], d));
      if (ASYM) lo[0] = fminf(lo[0], __shfl_xor_sync(0xffffffffu, lo[0], d));
      if (G != 128) {
        hi[1] = fmaxf(hi[1], __shfl_xor_sync(0xffffffffu, hi[1], d));
        if (ASYM) lo[1] = fminf(lo[1], __shfl_xor_sync(0xffffffffu, lo[1], d));
      }
    }
    uint16_t sh[2];
    float s[2], z[2], c[2][4];
    if constexpr (G == 128) {
      float all[8];
      finite = quantize_part<H, ASYM, 8>(w, lo[0], hi[0], sh[0], s[0], z[0], all) && finite;
      sh[1] = sh[0];
      s[1] = s[0];
      z[1] = z[0];
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i >> 2][i & 3] = all[i];
    } else {
      finite = quantize_part<H, ASYM, 4>(w, lo[0], hi[0], sh[0], s[0], z[0], c[0]) && finite;
      finite = quantize_part<H, ASYM, 4>(w + 4, lo[1], hi[1], sh[1], s[1], z[1], c[1]) && finite;
    }
    if (!finite) raise_status(a.status, PIPE_ERR_NONFINITE);
    // Codes 4 l .. 4 l + 3 are the first or the second half of a word of eight: pairs (0, 1) and (2, 3) or (4, 5) and (6, 7), in nibbles
    // i and i + 4.  Even threads write the word of the first half of the 128, odd ones that of the second.
    uint32_t word[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t u = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i)   // (the code in the low bits of a sum on top of 2^23)
        u |= (__float_as_uint(c[h][i] + (8388608.f + z[h])) & 15u) << (4 * ((i >> 1) + 4 * (i & 1)));
      word[h] = u << (8 * (l & 1));
      word[h] |= __shfl_xor_sync(0xffffffffu, word[h], 1);
    }
    if (o < a.O && word_at < a.I) *reinterpret_cast<uint32_t*>(code) = l & 1 ? word[1] : word[0];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (o < a.O && inside[h]) {
        if (G == 128 ? h == 0 && l == 0 : (4 * l) % G == 0) {
          a.scales[meta[h]] = sh[h];
          if (ASYM) a.zeros[meta[h]] = static_cast<uint8_t>(z[h]);
        }
        if (a.values) {
          float* v = value + 64 * h;
          if (a.wide_v) {
            __stcg(reinterpret_cast<float4*>(v), make_float4(c[h][0] * s[h], c[h][1] * s[h], c[h][2] * s[h], c[h][3] * s[h]));
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = c[h][i] * s[h];
          }
        }
      }
  }
}

using QuantKernel = void (*)(QuantArgs);
template <class H, int SRC, bool ASYM>
static QuantKernel quantize_kernel(int g) {
  return g == 32 ? group_quantize_kernel<H, SRC, ASYM, 32> : (g == 64 ? group_quantize_kernel<H, SRC, ASYM, 64> : group_quantize_kernel<H, SRC, ASYM, 128>);
}
template <class H, bool ASYM>
static QuantKernel quantize_kernel(int src, int g) {
  return src == PIPE_DTYPE_FP32 ? quantize_kernel<H, PIPE_DTYPE_FP32, ASYM>(g)
                                : (src == PIPE_DTYPE_BF16 ? quantize_kernel<H, PIPE_DTYPE_BF16, ASYM>(g) : quantize_kernel<H, PIPE_DTYPE_FP16, ASYM>(g));
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
  const int64_t row_blocks = ceil_div(a.O, grp::kQRows);
  // as many blocks as two rounds of eight on every SM need, each walking its share of the rows
  const int64_t across = static_cast<int64_t>(ceil_div(a.I, 128)) * desc->experts, want = ceil_div<int64_t>(2 * 8 * kPlanSMs, across);
  const dim3 grid(ceil_div(a.I, 128), static_cast<unsigned>(row_blocks < want ? row_blocks : want), desc->experts);
  a.status = device_status_word();
  if (!a.status) return grp::runtime_failed();
  const bool bf16 = desc->dtype == PIPE_DTYPE_BF16;
  const grp::QuantKernel k =
      bf16 ? (desc->asymmetric ? grp::quantize_kernel<grp::Bf16, true>(w_dtype, a.g) : grp::quantize_kernel<grp::Bf16, false>(w_dtype, a.g))
           : (desc->asymmetric ? grp::quantize_kernel<grp::Fp16, true>(w_dtype, a.g) : grp::quantize_kernel<grp::Fp16, false>(w_dtype, a.g));
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (launch_overlapped(k, grid, grp::kQThreads, 1, true, s, a) != cudaSuccess) return grp::runtime_failed();
  count_launch(1);
  take_expansion_mark(s);
  return launch_status();
}
