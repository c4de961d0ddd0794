// Rows to int8 by a scale of their own (definition: pipe_int8_quantize in include/pipe.h).
//
// One pass: a row's values stay in registers between the search for the largest magnitude and the codes.  P threads take a row,
// neighbouring values W at a time, every load and store of a warp of whole neighbouring lines: eight of 16 bits, four where values are
// written too (their 16-byte stores would leave half-written sectors otherwise).  The largest magnitude is found on the values' bits,
// which order like the magnitudes, a NaN above all.  Rows beyond what the registers hold are read a second time.  Bound by HBM where
// values are written; otherwise by nothing alone: some 7 instructions a value and 100 a thread and row, with the rows that the registers let stand
// on an SM.  11008 rows of 4096 bf16: 29 us (4.6 TB/s, 71 % of the issue slots, 55 % of the warps), with values 50 (6.3 TB/s).
#include "int8_common.cuh"

namespace pipe {
namespace i8 {

constexpr int kQHeld = 32;   // values that a thread holds

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
  int wide_x, wide_c, wide_v;   // W values, W codes, four values behind the codes are aligned to their size
  int* status;
};

// The code by its definition: the quotient in binary64, whose rounding (2^-53 of it) cannot reach a border between two codes that the
// exact quotient of two binary32 numbers is not on (it differs from an odd multiple of one half by 2^-33 or not at all).
__device__ __noinline__ float exact_code(float x, float s) {
  return fminf(fmaxf(static_cast<float>(rint(static_cast<double>(x) / static_cast<double>(s))), -127.f), 127.f);
}

// W neighbouring values as they lie in memory.
template <int SRC, int W>
struct Run {
  static constexpr int kWords = SRC == PIPE_DTYPE_FP32 ? W : W / 2;
  uint32_t u[kWords];
  __device__ __forceinline__ void load(const uint8_t* row, int i, int I, bool wide) {   // values i .. of a row of I; zeros behind it
    const uint8_t* at = row + static_cast<int64_t>(i) * (SRC == PIPE_DTYPE_FP32 ? 4 : 2);
    if (wide && i + W <= I) {
      if constexpr (kWords == 4) {
        const uint4 a = __ldcg(reinterpret_cast<const uint4*>(at));
        u[0] = a.x; u[1] = a.y; u[2] = a.z; u[3] = a.w;
      } else {
        const uint2 a = __ldcg(reinterpret_cast<const uint2*>(at));
        u[0] = a.x; u[1] = a.y;
      }
    } else if constexpr (SRC == PIPE_DTYPE_FP32) {
#pragma unroll
      for (int j = 0; j < W; ++j) u[j] = i + j < I ? __ldcg(reinterpret_cast<const uint32_t*>(at) + j) : 0u;
    } else {
      const uint16_t* p = reinterpret_cast<const uint16_t*>(at);
#pragma unroll
      for (int j = 0; j < W / 2; ++j)
        u[j] = (i + 2 * j < I ? __ldcg(p + 2 * j) : 0u) | (i + 2 * j + 1 < I ? static_cast<uint32_t>(__ldcg(p + 2 * j + 1)) << 16 : 0u);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (uint32_t& v : u) v = 0;
  }
  // the larger of `most` and the magnitudes (16-bit types: in both halves)
  __device__ __forceinline__ uint32_t magnitude(uint32_t most) const {
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
      if constexpr (SRC == PIPE_DTYPE_FP32) most = max(most, u[j] & 0x7FFFFFFFu);
      else most = __vmaxu2(most, u[j] & 0x7FFF7FFFu);
    }
    return most;
  }
  __device__ __forceinline__ float value(int j) const {
    if constexpr (SRC == PIPE_DTYPE_FP32) return __uint_as_float(u[j]);
    else if constexpr (SRC == PIPE_DTYPE_BF16) return __uint_as_float(j & 1 ? u[j >> 1] & 0xFFFF0000u : u[j >> 1] << 16);
    else return grp::Fp16::to_float(static_cast<uint16_t>(u[j >> 1] >> (16 * (j & 1))));
  }
};
template <int SRC>
__device__ __forceinline__ float as_number(uint32_t magnitude) {   // of Run::magnitude, over a whole row
  if constexpr (SRC == PIPE_DTYPE_FP32) return __uint_as_float(magnitude);
  const uint16_t h = static_cast<uint16_t>(max(magnitude & 0xFFFFu, magnitude >> 16));
  return SRC == PIPE_DTYPE_BF16 ? grp::Bf16::to_float(h) : grp::Fp16::to_float(h);
}

// P threads of a row; a block of 256 threads, or of P where that is more.
template <int SRC, int W, int P>
__global__ void __launch_bounds__(P > 256 ? P : 256, (W == 8 ? 1280 : 1024) / (P > 256 ? P : 256)) int8_quantize_kernel(const QuantArgs a) {
  constexpr int kThreads = P > 256 ? P : 256, kRows = kThreads / P, kRuns = kQHeld / W;
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

  Run<SRC, W> held[kRuns];
#pragma unroll
  for (int k = 0; k < kRuns; ++k) {
    const int i = W * (k * P + l);
    if (i < I) held[k].load(row, i, I, a.wide_x);
    else held[k].zero();
  }
  uint32_t most = 0;
#pragma unroll
  for (int k = 0; k < kRuns; ++k) most = held[k].magnitude(most);
  for (int i = kQHeld * P + W * l; i < I; i += W * P) {   // (I is below 2^29 + 1)
    Run<SRC, W> f;
    f.load(row, i, I, a.wide_x);
    most = f.magnitude(most);
  }
  most = __reduce_max_sync(0xffffffffu, __float_as_uint(as_number<SRC>(most)));
  if (P > 32) {
    if ((threadIdx.x & 31) == 0) most_s[threadIdx.x >> 5] = most;
    __syncthreads();
    most = __reduce_max_sync(0xffffffffu, most_s[(threadIdx.x / P) * (P / 32) + (threadIdx.x & 31) % (P / 32)]);
  }
  if (!mine) return;
  const float top = __uint_as_float(most);
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
  const f32x2 inv2 = both_f2(inv), less2 = both_f2(-s), magic2 = both_f2(12582912.f);
  auto put = [&](const Run<SRC, W>& f, int i) {
    // An estimate rounded by an addition (1.5 * 2^23, where the spacing of binary32 is one, and the code the low byte) is off by one at
    // most.  The remainder x - q s is exact: a multiple of the last place of s (of half of it where |x| < s), and at most s.  Where it
    // reaches half a step, on a tie or where the estimate went wrong, it tells by how much.  (Values of 16 bits come that near to a tie once in
    // some ten thousand, whole warps of eight each one time in forty: by the quotient in binary64 that took a third of all instructions.)
    f32x2 q[W / 2];
    uint32_t word[W / 4];
    float u[W], edge = 0.f;
#pragma unroll
    for (int h = 0; h < W / 2; ++h) {
      const f32x2 x = pack_f2(f.value(2 * h), f.value(2 * h + 1)), sum = fma_f2(x, inv2, magic2);
      unpack_f2(sum, u[2 * h], u[2 * h + 1]);
      q[h] = sub_f2(sum, magic2);
      float r0, r1;
      unpack_f2(fma_f2(q[h], less2, x), r0, r1);
      edge = max3_abs(edge, r0, r1);
    }
    auto set = [&](int h, float e0, float e1) {
      q[h] = pack_f2(e0, e1);
      u[2 * h] = e0 + 12582912.f;
      u[2 * h + 1] = e1 + 12582912.f;
    };
    if (!fast) {   // (a step without a usable reciprocal, zero and infinity among them)
#pragma unroll
      for (int h = 0; h < W / 2; ++h) {
        const float e0 = some ? exact_code(f.value(2 * h), s) : 0.f, e1 = some ? exact_code(f.value(2 * h + 1), s) : 0.f;
        set(h, e0, e1);
      }
    } else if (2.f * edge >= s) {
#pragma unroll
      for (int h = 0; h < W / 2; ++h) {
        float e[2];
        unpack_f2(q[h], e[0], e[1]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float r = fmaf(-e[j], s, f.value(2 * h + j)), twice = 2.f * fabsf(r);
          if (twice > s || (twice == s && (__float_as_uint(u[2 * h + j]) & 1))) e[j] += r > 0.f ? 1.f : -1.f;   // (an odd code lies in an odd sum)
        }
        set(h, e[0], e[1]);
      }
    }
#pragma unroll
    for (int h = 0; h < W / 4; ++h) word[h] = pack4_low_bytes(u[4 * h], u[4 * h + 1], u[4 * h + 2], u[4 * h + 3]);
    if (a.wide_c && i + W <= a.I) {
      if constexpr (W == 8) *reinterpret_cast<uint2*>(codes + i) = make_uint2(word[0], word[1]);
      else *reinterpret_cast<uint32_t*>(codes + i) = word[0];
    } else {
#pragma unroll
      for (int j = 0; j < W; ++j)
        if (i + j < a.I) codes[i + j] = static_cast<int8_t>(word[j >> 2] >> (8 * (j & 3)));
    }
    if constexpr (W == 4) {
      if (values) {
        float v[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) unpack_f2(mul_f2(q[h], both_f2(s)), v[2 * h], v[2 * h + 1]);
        if (a.wide_v && i + 4 <= a.I) {
          __stcg(reinterpret_cast<float4*>(values + i), make_float4(v[0], v[1], v[2], v[3]));
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (i + j < a.I) values[i + j] = v[j];
        }
      }
    }
  };
#pragma unroll
  for (int k = 0; k < kRuns; ++k) {
    const int i = W * (k * P + l);
    if (i < a.I) put(held[k], i);
  }
  for (int i = kQHeld * P + W * l; i < a.I; i += W * P) {
    Run<SRC, W> f;
    if (I) f.load(row, i, a.I, a.wide_x);
    else f.zero();
    put(f, i);
  }
}

using QuantKernel = void (*)(QuantArgs);
template <int SRC, int W>
static QuantKernel quantize_kernel(int P) {
  switch (P) {
    case 32: return int8_quantize_kernel<SRC, W, 32>;
    case 64: return int8_quantize_kernel<SRC, W, 64>;
    case 128: return int8_quantize_kernel<SRC, W, 128>;
    case 256: return int8_quantize_kernel<SRC, W, 256>;
    default: return int8_quantize_kernel<SRC, W, 512>;
  }
}
template <int SRC>
static QuantKernel quantize_kernel(int P, bool values) {
  if constexpr (SRC != PIPE_DTYPE_FP32)
    if (!values) return quantize_kernel<SRC, 8>(P);
  return quantize_kernel<SRC, 4>(P);
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
  const int W = d_values || size == 4 ? 4 : 8;
  a.wide_x = !misaligned(d_x, W * size) && ldx % W == 0;
  a.wide_c = !misaligned(d_codes, W) && ldc % W == 0;
  a.wide_v = !misaligned(d_values, 16) && ldv % 4 == 0;
  a.status = device_status_word();
  if (!a.status) return grp::runtime_failed();
  // The fewest threads whose registers hold a row (32, 64, 128, 256 and 512 threads, us): 4096 rows of 4096 bf16 22, 19, 13, 16, 27; 20000 of 512
  // 11, 15, 26, 44, 104; 4096 of 11008 with values 121, 109, 78, 62, 59.
  int P = 32;
  while (P < 512 && I > i8::kQHeld * P) P *= 2;
  const i8::QuantKernel k = x_dtype == PIPE_DTYPE_FP32 ? i8::quantize_kernel<PIPE_DTYPE_FP32>(P, d_values)
                                                       : (x_dtype == PIPE_DTYPE_BF16 ? i8::quantize_kernel<PIPE_DTYPE_BF16>(P, d_values) : i8::quantize_kernel<PIPE_DTYPE_FP16>(P, d_values));
  const int threads = P > 256 ? P : 256;
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (launch_overlapped(k, dim3(static_cast<unsigned>(ceil_div<int64_t>(N, threads / P))), threads, 1, true, s, a) != cudaSuccess) return grp::runtime_failed();
  count_launch(1);
  take_expansion_mark(s);
  return launch_status();
}
