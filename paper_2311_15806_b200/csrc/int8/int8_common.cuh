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

// sigma of N values: the formulas of grp::quick_activation with every rounding spelled out, so that all kernels give the same bits (a
// product and a sum that the compiler may or may not join gave a row another last bit in another kernel).
template <int N>
__device__ __forceinline__ void activate(float (&v)[N], int kind) {
  if (kind == PIPE_ACT_IDENTITY) return;
  if (kind == PIPE_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm("max.NaN.f32 %0, %1, %2;" : "=f"(v[i]) : "f"(v[i]), "f"(0.f));
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
