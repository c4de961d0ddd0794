// Rows to int8 by a scale of their own (definition: pipe_int8_quantize in include/pipe.h).
//
// One pass, bound by HBM: a row's values stay in registers between the search for the largest magnitude and the codes.  P threads take
// a row, four neighbouring values at a time, so that every load and store of a warp is of whole neighbouring lines; the largest
// magnitude is found on the values' bits, which order like the magnitudes, a NaN above all.  Rows beyond what the registers hold are
// read a second time.
#include "int8_common.cuh"

namespace pipe {
namespace i8 {

constexpr int kQHeld = 8;   // fours of values that a thread holds

struct QuantArgs {
  const void* x;
  int64_t T, ldx, N;
  int I;
  const int32_t* rows;
  const int32_t* count;
  int8_t* codes;
  int64_t ldc;
  float* scales;
  float* values;
  int64_t ldv;
  int wide_x, wide_c, wide_v;   // fours of values, codes, values behind the codes are aligned to their size
  int* status;
};

// The code by its definition: the quotient in binary64, whose rounding (2^-53 of it) cannot reach a border between two codes that the
// exact quotient of two binary32 numbers is not on (it differs from an odd multiple of one half by 2^-33 or not at all).
__device__ __noinline__ float exact_code(float x, float s) {
  return fminf(fmaxf(static_cast<float>(rint(static_cast<double>(x) / static_cast<double>(s))), -127.f), 127.f);
}

// Four neighbouring values as they lie in memory.
template <int SRC>
struct Four {
  static constexpr int kWords = SRC == PIPE_DTYPE_FP32 ? 4 : 2;
  uint32_t u[kWords];
  __device__ __forceinline__ void load(const uint8_t* row, int i, int I, bool wide) {   // values i .. i + 3 of a row of I; zeros behind it
    if constexpr (SRC == PIPE_DTYPE_FP32) {
      const uint32_t* p = reinterpret_cast<const uint32_t*>(row) + i;
      if (wide && i + 4 <= I) {
        const uint4 a = __ldcg(reinterpret_cast<const uint4*>(p));
        u[0] = a.x; u[1] = a.y; u[2] = a.z; u[3] = a.w;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = i + j < I ? __ldcg(p + j) : 0u;
      }
    } else {
      const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + i;
      if (wide && i + 4 <= I) {
        const uint2 a = __ldcg(reinterpret_cast<const uint2*>(p));
        u[0] = a.x; u[1] = a.y;
      } else {
#pragma unroll
        for (int j = 0; j < 2; ++j)
          u[j] = (i + 2 * j < I ? __ldcg(p + 2 * j) : 0u) | (i + 2 * j + 1 < I ? static_cast<uint32_t>(__ldcg(p + 2 * j + 1)) << 16 : 0u);
      }
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (uint32_t& v : u) v = 0;
  }
  // the larger of `most` and the magnitudes (16-bit types: in both halves)
  __device__ __forceinline__ uint32_t magnitude(uint32_t most) const {
    if constexpr (SRC == PIPE_DTYPE_FP32) return max(max(most, max(u[0] & 0x7FFFFFFFu, u[1] & 0x7FFFFFFFu)), max(u[2] & 0x7FFFFFFFu, u[3] & 0x7FFFFFFFu));
    else return __vmaxu2(most, __vmaxu2(u[0] & 0x7FFF7FFFu, u[1] & 0x7FFF7FFFu));
  }
  __device__ __forceinline__ float value(int j) const {
    if constexpr (SRC == PIPE_DTYPE_FP32) return __uint_as_float(u[j]);
    const uint16_t h = static_cast<uint16_t>(u[j >> 1] >> (16 * (j & 1)));
    return SRC == PIPE_DTYPE_BF16 ? grp::Bf16::to_float(h) : grp::Fp16::to_float(h);
  }
};
template <int SRC>
__device__ __forceinline__ float as_number(uint32_t magnitude) {   // of Four::magnitude, over a whole row
  if constexpr (SRC == PIPE_DTYPE_FP32) return __uint_as_float(magnitude);
  const uint16_t h = static_cast<uint16_t>(max(magnitude & 0xFFFFu, magnitude >> 16));
  return SRC == PIPE_DTYPE_BF16 ? grp::Bf16::to_float(h) : grp::Fp16::to_float(h);
}

// P threads of a row; a block of 256 threads, or of P where that is more.
template <int SRC, int P>
__global__ void __launch_bounds__(P > 256 ? P : 256) int8_quantize_kernel(const QuantArgs a) {
  constexpr int kThreads = P > 256 ? P : 256, kRows = kThreads / P;
  constexpr int kSize = SRC == PIPE_DTYPE_FP32 ? 4 : 2;
  __shared__ uint32_t most_s[kThreads / 32];
  grid_wait();
  grid_release();
  const int l = threadIdx.x % P;
  const int64_t slot = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / P;
  const int64_t slots = a.count ? min(static_cast<int64_t>(max(__ldcg(a.count), 0)), a.N) : a.N;
  const bool mine = slot < slots;
  int64_t r = slot;
  if (mine && a.rows) r = __ldcg(a.rows + slot);
  const int I = mine && r >= 0 && r < a.T ? a.I : 0;   // values to be read
  const uint8_t* row = static_cast<const uint8_t*>(a.x) + (I ? r * a.ldx * kSize : 0);

  Four<SRC> held[kQHeld];
  uint32_t most = 0;
#pragma unroll
  for (int k = 0; k < kQHeld; ++k) {
    const int i = 4 * (k * P + l);
    if (i < I) held[k].load(row, i, I, a.wide_x);
    else held[k].zero();
  }
#pragma unroll
  for (int k = 0; k < kQHeld; ++k) most = held[k].magnitude(most);
  for (int i = 4 * (kQHeld * P + l); i < I; i += 4 * P) {
    Four<SRC> f;
    f.load(row, i, I, a.wide_x);
    most = f.magnitude(most);
  }
  float top = as_number<SRC>(most);
  most = __reduce_max_sync(0xffffffffu, __float_as_uint(top));
  if (P > 32) {
    if ((threadIdx.x & 31) == 0) most_s[threadIdx.x >> 5] = most;
    __syncthreads();
    const int first = (threadIdx.x / P) * (P / 32);
#pragma unroll
    for (int w = 0; w < P / 32; ++w) most = max(most, most_s[first + w]);
  }
  if (!mine) return;
  top = __uint_as_float(most);
  const bool finite = top <= 3.402823466e38f;
  const float s = __fdiv_rn(top, 127.f);
  if (l == 0) {
    a.scales[slot] = s;
    if (!finite) raise_status(a.status, PIPE_ERR_NONFINITE);
  }
  const bool fast = quant_step_is_fast(s), some = finite && s > 0.f;
  const float inv = fast ? __frcp_rn(s) : 0.f;
  int8_t* codes = a.codes + slot * a.ldc;
  float* values = a.values ? a.values + slot * a.ldv : nullptr;
  auto put = [&](const Four<SRC>& f, int i) {
    float q[4] = {0.f, 0.f, 0.f, 0.f};
    if (some) {
      // An estimate rounded by an addition (1.5 * 2^23, where the spacing of binary32 is one) is off by one at most.  The remainder
      // x - q s is exact: a multiple of the last place of s (of half of it where |x| < s), and at most s.  Where it reaches half a step,
      // on a tie or where the estimate went wrong, the definition is evaluated.
      float edge = fast ? 0.f : s;
      if (fast) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          q[j] = __fsub_rn(__fmaf_rn(f.value(j), inv, 12582912.f), 12582912.f);
          edge = fmaxf(edge, fabsf(fmaf(-q[j], s, f.value(j))));
        }
      }
      if (2.f * edge >= s) {
#pragma unroll
        for (int j = 0; j < 4; ++j) q[j] = exact_code(f.value(j), s);
      }
    }
    if (a.wide_c && i + 4 <= a.I) {
      *reinterpret_cast<uint32_t*>(codes + i) = pack4_low_bytes(q[0] + 12582912.f, q[1] + 12582912.f, q[2] + 12582912.f, q[3] + 12582912.f);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i + j < a.I) codes[i + j] = static_cast<int8_t>(static_cast<int>(q[j]));
    }
    if (values) {
      if (a.wide_v && i + 4 <= a.I) {
        __stcg(reinterpret_cast<float4*>(values + i), make_float4(q[0] * s, q[1] * s, q[2] * s, q[3] * s));
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (i + j < a.I) values[i + j] = q[j] * s;
      }
    }
  };
#pragma unroll
  for (int k = 0; k < kQHeld; ++k) {
    const int i = 4 * (k * P + l);
    if (i < a.I) put(held[k], i);
  }
  for (int64_t i = 4 * (static_cast<int64_t>(kQHeld) * P + l); i < a.I; i += 4 * P) {
    Four<SRC> f;
    if (I) f.load(row, static_cast<int>(i), I, a.wide_x);
    else f.zero();
    put(f, static_cast<int>(i));
  }
}

using QuantKernel = void (*)(QuantArgs);
template <int SRC>
static QuantKernel quantize_kernel(int P) {
  return P == 32 ? int8_quantize_kernel<SRC, 32> : (P == 128 ? int8_quantize_kernel<SRC, 128> : int8_quantize_kernel<SRC, 512>);
}

}  // namespace i8
}  // namespace pipe

using namespace pipe;

extern "C" pipe_status pipe_int8_quantize(const void* d_x, int32_t x_dtype, int64_t T, int32_t I, int64_t ldx, const int32_t* d_rows, int64_t N,
                                          const int32_t* d_count, int8_t* d_codes, int64_t ldc, float* d_scales, float* d_values, int64_t ldv,
                                          void* stream) {
  constexpr int64_t kMostRows = int64_t{1} << 30;
  if (x_dtype < PIPE_DTYPE_BF16 || x_dtype > PIPE_DTYPE_FP32) return PIPE_ERR_INVALID_ARG;
  if (T < 0 || T > kMostRows || N < 0 || N > kMostRows || I < 1 || I > 1 << 29) return PIPE_ERR_INVALID_ARG;
  if ((T > 0 && N > 0 && !d_x) || (N > 0 && (!d_codes || !d_scales))) return PIPE_ERR_INVALID_ARG;
  if (ldx < I || ldc < I || (d_values && ldv < I)) return PIPE_ERR_INVALID_ARG;
  if (ldx >= int64_t{1} << 32 || ldc >= int64_t{1} << 32 || (d_values && ldv >= int64_t{1} << 32)) return PIPE_ERR_INVALID_ARG;   // (bytes of all rows in 64 bits)
  if (!d_rows && N != T) return PIPE_ERR_SHAPE;
  const uintptr_t size = x_dtype == PIPE_DTYPE_FP32 ? 4 : 2;
  auto misaligned = [](const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; };
  if (misaligned(d_x, size) || misaligned(d_scales, 4) || misaligned(d_values, 4) || misaligned(d_rows, 4) || misaligned(d_count, 4))
    return PIPE_ERR_ALIGNMENT;
  if (N == 0) return PIPE_OK;
  i8::QuantArgs a;
  a.x = d_x; a.T = T; a.ldx = ldx; a.N = N; a.I = I;
  a.rows = d_rows; a.count = d_count;
  a.codes = d_codes; a.ldc = ldc;
  a.scales = d_scales;
  a.values = d_values; a.ldv = ldv;
  a.wide_x = !misaligned(d_x, 4 * size) && ldx % 4 == 0;
  a.wide_c = !misaligned(d_codes, 4) && ldc % 4 == 0;
  a.wide_v = !misaligned(d_values, 16) && ldv % 4 == 0;
  a.status = device_status_word();
  if (!a.status) return grp::runtime_failed();
  // the fewest threads whose registers hold a row
  const int P = I <= 4 * i8::kQHeld * 32 ? 32 : (I <= 4 * i8::kQHeld * 128 ? 128 : 512);
  const i8::QuantKernel k = x_dtype == PIPE_DTYPE_FP32 ? i8::quantize_kernel<PIPE_DTYPE_FP32>(P)
                                                       : (x_dtype == PIPE_DTYPE_BF16 ? i8::quantize_kernel<PIPE_DTYPE_BF16>(P) : i8::quantize_kernel<PIPE_DTYPE_FP16>(P));
  const int threads = P > 256 ? P : 256;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (launch_overlapped(k, dim3(static_cast<unsigned>(ceil_div<int64_t>(N, threads / P))), threads, 1, true, s, a) != cudaSuccess) return grp::runtime_failed();
  count_launch(1);
  take_expansion_mark(s);
  return launch_status();
}
