// What the kernels of the 8-bit integer layers share (formats and entry points: include/pipe.h).
#pragma once

#include "../group/group_common.cuh"

namespace pipe {
namespace i8 {

// One call of pipe_int8_linear (c.offsets = nullptr: one expert that owns all N rows) or pipe_int8_expert_linear.
struct Call {
  grp::Call c;          // E, O, I; x: int8 [T, I] with T = N, ldx in bytes; offsets, N; bias, act, y, ldy; status
  const int8_t* w;      // E * O rows of I, pitch ldw
  int64_t ldw;
  const float* sw;      // [E * O]
  const float* sx;      // [N]
  int dtype;            // of bias and y
};

// The types of bias and outputs.
struct Fp32 {
  static constexpr int kBytes = 4;
  static __device__ __forceinline__ uint32_t pack(float, float) { return 0; }   // (of 16-bit types only)
  static __device__ __forceinline__ float load(const void* p, int64_t i) { return __ldcg(static_cast<const float*>(p) + i); }
  static __device__ __forceinline__ void store(void* p, int64_t i, float v) { static_cast<float*>(p)[i] = v; }
};
template <class H>
struct Half {
  static constexpr int kBytes = 2;
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) { return H::pack(lo, hi); }
  static __device__ __forceinline__ float load(const void* p, int64_t i) { return H::to_float(__ldcg(static_cast<const uint16_t*>(p) + i)); }
  static __device__ __forceinline__ void store(void* p, int64_t i, float v) { static_cast<uint16_t*>(p)[i] = H::from_float(v); }
};
using Bf16 = Half<grp::Bf16>;
using Fp16 = Half<grp::Fp16>;

// The output from an exact sum: one rounding each of the sum, its product with the channel's scale, and (fused with the bias) that with
// the token's.
__device__ __forceinline__ float scaled(int acc, float sw, float sx, float bias) { return fmaf(__fmul_rn(static_cast<float>(acc), sw), sx, bias); }

// sigma of N values for outputs of 32 bits: the formulas of grp::quick_activation, with what the exponent of two loses by
// its rounding (2^-18 of sigma(-80), 2^-17 of GELU(-13)) brought in behind the exponential.  Within 2^-20 of sigma, GELU 2^-19: the exponential is
// off by 5, the reciprocal and its argument by 4, the polynomial and its fit by 5, the products by 3 units of 2^-24.  Two at a time because it
// stands in the drain (4096 rows to 11008 channels from 256 values, us, identity 41, SiLU 55, GELU 69; one at a time 61 and 78; without the
// remainder 54 and 65).
template <int N>
__device__ __forceinline__ void activate32(float (&v)[N], int kind) {
  constexpr float kHead = 1.44269502f, kTail = 1.92596299e-8f, kLn2 = 0.693147182f;   // log2 e = kHead + kTail
  const f32x2 one = both_f2(1.f);
  auto bounded = [](float x, float most) {   // |x|, a NaN kept: behind `most` the exponential is 0 (the remainder of an infinite product is no number)
    float d;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(fabsf(x)), "f"(most));
    return d;
  };
  if (kind == PIPE_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      float p, q, e0, e1, r0, r1;
      const f32x2 a = pack_f2(bounded(v[i], 16.f), bounded(v[i + 1], 16.f));
      const f32x2 square = mul_f2(a, a), over = fma_f2(mul_f2(a, both_f2(-1.f)), a, square);   // a^2 = square - over
      const f32x2 z = mul_f2(square, both_f2(0.5f * kHead));
      f32x2 rest = fma_f2(square, both_f2(-0.5f * kHead), z);
      rest = fma_f2(over, both_f2(0.5f * kHead), fma_f2(square, both_f2(-0.5f * kTail), rest));
      unpack_f2(z, p, q);
      asm("ex2.approx.f32 %0, %1;" : "=f"(e0) : "f"(-p));
      asm("ex2.approx.f32 %0, %1;" : "=f"(e1) : "f"(-q));
      f32x2 e = pack_f2(e0, e1);
      e = fma_f2(mul_f2(rest, both_f2(kLn2)), e, e);
      unpack_f2(fma_f2(a, both_f2(0.305f), one), p, q);
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(p));
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(q));
      const f32x2 t = pack_f2(r0, r1);
      f32x2 u = both_f2(0.03663886f);
      u = fma_f2(u, t, both_f2(-0.15274605f));
      u = fma_f2(u, t, both_f2(0.18531485f));
      u = fma_f2(u, t, both_f2(-0.037620626f));
      u = fma_f2(u, t, both_f2(0.12084037f));
      u = fma_f2(u, t, both_f2(0.1034737f));
      u = fma_f2(u, t, both_f2(0.12245868f));
      u = mul_f2(mul_f2(fma_f2(u, t, both_f2(0.12164024f)), t), e);
      unpack_f2(u, p, q);
      v[i] = __fmul_rn(v[i], v[i] >= 0.f ? __fsub_rn(1.f, p) : p);
      v[i + 1] = __fmul_rn(v[i + 1], v[i + 1] >= 0.f ? __fsub_rn(1.f, q) : q);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 2) {
      float p, q, e0, e1, r0, r1;
      const f32x2 a = pack_f2(bounded(v[i], 128.f), bounded(v[i + 1], 128.f));
      const f32x2 z = mul_f2(a, both_f2(kHead)), rest = fma_f2(a, both_f2(-kTail), fma_f2(a, both_f2(-kHead), z));
      unpack_f2(z, p, q);
      asm("ex2.approx.f32 %0, %1;" : "=f"(e0) : "f"(-p));
      asm("ex2.approx.f32 %0, %1;" : "=f"(e1) : "f"(-q));
      f32x2 e = pack_f2(e0, e1);
      e = fma_f2(mul_f2(rest, both_f2(kLn2)), e, e);
      unpack_f2(add_f2(e, one), p, q);
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(p));
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(q));
      unpack_f2(e, e0, e1);
      if (v[i] >= 0.f) e0 = 1.f;
      if (v[i + 1] >= 0.f) e1 = 1.f;
      v[i] = __fmul_rn(kind == PIPE_ACT_SILU ? __fmul_rn(v[i], e0) : e0, r0);   // (a NaN is not >= 0: e is NaN then)
      v[i + 1] = __fmul_rn(kind == PIPE_ACT_SILU ? __fmul_rn(v[i + 1], e1) : e1, r1);
    }
  }
}

// sigma of N values: the formulas of grp::quick_activation with every rounding spelled out, so that all kernels give the same bits (a
// product and a sum that the compiler may or may not join gave a row another last bit in another kernel).  They are made for outputs of 16
// bits: the rounded argument of the exponential costs up to 2^-17 of sigma(v).
template <class H, int N>
__device__ __forceinline__ void activate(float (&v)[N], int kind) {
  if (kind == PIPE_ACT_IDENTITY) return;
  if (kind == PIPE_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm("max.NaN.f32 %0, %1, %2;" : "=f"(v[i]) : "f"(v[i]), "f"(0.f));
  } else if constexpr (H::kBytes == 4) {
    activate32(v, kind);
  } else if (kind == PIPE_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float e, t;
      asm("ex2.approx.f32 %0, %1;" : "=f"(e) : "f"(__fmul_rn(__fmul_rn(v[i], v[i]), -0.72134752f)));
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(__fmaf_rn(fabsf(v[i]), 0.305f, 1.f)));
      float q = 0.03663886f;
      q = __fmaf_rn(q, t, -0.15274605f);
      q = __fmaf_rn(q, t, 0.18531485f);
      q = __fmaf_rn(q, t, -0.037620626f);
      q = __fmaf_rn(q, t, 0.12084037f);
      q = __fmaf_rn(q, t, 0.1034737f);
      q = __fmaf_rn(q, t, 0.12245868f);
      q = __fmul_rn(__fmul_rn(__fmaf_rn(q, t, 0.12164024f), t), e);
      v[i] = __fmul_rn(v[i], v[i] >= 0.f ? __fsub_rn(1.f, q) : q);
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float e, r;
      asm("ex2.approx.f32 %0, %1;" : "=f"(e) : "f"(__fmul_rn(fabsf(v[i]), -1.44269504f)));
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(__fadd_rn(1.f, e)));
      if (v[i] >= 0.f) e = 1.f;
      v[i] = __fmul_rn(kind == PIPE_ACT_SILU ? __fmul_rn(v[i], e) : e, r);   // (a NaN is not >= 0: e is NaN then)
    }
  }
}

pipe_status linear_tc(const Call& c, cudaStream_t stream);

}  // namespace i8
}  // namespace pipe
