// What the kernels of the 4-bit layers with group scales share (formats and entry points: include/pipe.h).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "group_plan.h"
#include "pipe_common.cuh"

namespace pipe {
namespace grp {

// One call of pipe_group_linear (offsets = nullptr: one expert that owns all N rows) or pipe_expert_linear.
struct Call {
  int E, O, I, g;
  int KB;                 // I / 32: runs of 32 codes, the rows of 16 bytes of the code array
  const uint8_t* codes;   // [E, KB, O, 16]
  const void* scales;     // [E, I/g, O]
  const uint8_t* zeros;   // the same shape, or nullptr
  const void* x;          // [T, I] pitch ldx
  int64_t T, ldx;
  const int32_t* rows;    // [N] or nullptr
  const int32_t* offsets; // [E + 1] or nullptr
  int64_t N;
  const void* bias;       // [E, O] or nullptr
  int act;
  void* y;                // [N, O] pitch ldy
  int64_t ldy;
  int* status;
};

// CTAs of a cluster: rank, count, the barrier of all their threads, and reads of another one's shared memory.
__device__ __forceinline__ int cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return static_cast<int>(r);
}
__device__ __forceinline__ int cluster_ctas() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return static_cast<int>(r);
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_address(const void* own, int rank) {
  uint32_t d;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(d) : "r"(static_cast<uint32_t>(__cvta_generic_to_shared(own))), "r"(rank));
  return d;
}
__device__ __forceinline__ float cluster_load(const float* own, int rank) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(cluster_address(own, rank)) : "memory");
  return v;
}
__device__ __forceinline__ int cluster_load(const int32_t* own, int rank) {
  int v;
  asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(cluster_address(own, rank)) : "memory");
  return v;
}

// The two element types: packed arithmetic on pairs, and the number whose low mantissa bits a 4-bit code can be or-ed into
// (128 + u in bf16, 1024 + u in fp16: both exact, as is the difference of two of them).  kOver: the least magnitude of a scale whose
// fifteenfold is beyond the type's range when rounded to it; kInf: infinity.  (As they lie in memory.)
struct Bf16 {
  using T = __nv_bfloat16;
  static constexpr uint32_t kBase = 0x43004300u;
  static constexpr uint32_t kOver = 0x7D89u, kInf = 0x7F80u;   // (1.0625 * 2^124 times 15 is the largest number of the type)
  static __device__ __forceinline__ uint32_t add2(uint32_t a, uint32_t b) {   // (one fused operation; an addition costs two)
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(0x3F803F80u), "r"(b));
    return d;
  }
  static __device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
  }
  static __device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b) {   // (magnitudes; the signs mean nothing)
    uint32_t d;
    asm("max.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
  }
  static __device__ __forceinline__ float to_float(uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }
  static __device__ __forceinline__ uint16_t from_float(float v) { return __bfloat16_as_ushort(__float2bfloat16_rn(v)); }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
  }
  static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};
struct Fp16 {
  using T = __half;
  static constexpr uint32_t kBase = 0x64006400u;
  static constexpr uint32_t kOver = 0x6C44u, kInf = 0x7C00u;   // (4368 times 15 is 65520, which rounds to infinity)
  static __device__ __forceinline__ uint32_t add2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("add.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
  }
  static __device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
  }
  static __device__ __forceinline__ uint32_t max_abs2(uint32_t a, uint32_t b) {   // (magnitudes; the signs mean nothing)
    uint32_t d;
    asm("max.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
  }
  static __device__ __forceinline__ float to_float(uint16_t v) { return __half2float(__ushort_as_half(v)); }
  static __device__ __forceinline__ uint16_t from_float(float v) { return __half_as_ushort(__float2half_rn(v)); }
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t d;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
  }
  static __device__ __forceinline__ void mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  }
};

// Pair i (codes 2i, 2i + 1) of a word, each on top of the base.
template <class H>
__device__ __forceinline__ uint32_t code_pair(uint32_t w, int i) {
  uint32_t d;   // (shifted & mask) | base in one three-input operation
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(d) : "r"(w >> (4 * i)), "r"(0x000F000Fu), "r"(H::kBase));
  return d;
}
// What takes the base and the zero point z (8 for a symmetric layer) away from a pair again: minus their sum, in both halves.
template <class H>
__device__ __forceinline__ uint32_t zero_pair(uint32_t z) {
  return (H::kBase | 0x80008000u) | z | (z << 16);
}

// sigma of N sums, with SiLU and sigmoid on the approximate exponential and reciprocal (2^-22 and 2^-23 of their values, the
// exponential's argument rounded: |v| 2^-24): far below half a step of a 16-bit output.  The exponential is that of -|v|, which cannot
// overflow: sigmoid(v) = t / (1 + t) and SiLU v t / (1 + t) for v < 0, t = exp v, keep every value that the type has (an exponential of -v
// overflows from v = -88.7 on, where bf16 has numbers down to v = -92 and more).  GELU is v Phi(v), Phi(-u) = exp(-u^2 / 2) t P(t) with
// t = 1 / (1 + 0.305 u) and P of degree 7, fitted here to Phi(-u) exp(u^2 / 2) on 0 <= u <= 14.5 with the least relative distance, 2^-23.3
// (weighted least squares on Chebyshev points); v (1 + erf) / 2 cancels for v < 0, 4 % off at -5.  The kind is asked once for all of them: asked per
// value, unrolled, it took a drain 85 cycles a value.
template <int N>
__device__ __forceinline__ void quick_activation(float (&v)[N], int kind) {
  if (kind == PIPE_ACT_IDENTITY) return;
  if (kind == PIPE_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm("max.NaN.f32 %0, %1, %2;" : "=f"(v[i]) : "f"(v[i]), "f"(0.f));   // (an ordinary maximum makes a NaN a 0)
  } else if (kind == PIPE_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float e, t;
      asm("ex2.approx.f32 %0, %1;" : "=f"(e) : "f"(v[i] * v[i] * -0.72134752f));
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t) : "f"(fmaf(fabsf(v[i]), 0.305f, 1.f)));
      float q = 0.03663886f;
      q = fmaf(q, t, -0.15274605f);
      q = fmaf(q, t, 0.18531485f);
      q = fmaf(q, t, -0.037620626f);
      q = fmaf(q, t, 0.12084037f);
      q = fmaf(q, t, 0.1034737f);
      q = fmaf(q, t, 0.12245868f);
      q = fmaf(q, t, 0.12164024f) * t * e;
      v[i] *= v[i] >= 0.f ? 1.f - q : q;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float e, r;
      asm("ex2.approx.f32 %0, %1;" : "=f"(e) : "f"(fabsf(v[i]) * -1.44269504f));
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + e));
      if (v[i] >= 0.f) e = 1.f;
      v[i] = (kind == PIPE_ACT_SILU ? v[i] * e : e) * r;   // (a NaN is not >= 0: e is NaN then)
    }
  }
}

// Offsets of 32 experts, lo and hi of this lane's (lo = hi = 0 behind the last, which lane `last` has), made ascending: an offset below
// one before it counts as that one, so that no row has two experts and the units stay as few as their bound.  top: the last offset of
// the experts before, and then of these.
__device__ __forceinline__ void make_ascending(int& lo, int& hi, int& top, bool here, int last) {
  if (__any_sync(0xffffffffu, here && (hi < lo || lo < top))) {
    lo = max(lo, top);
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, lo, d);
      if ((threadIdx.x & 31) >= d) lo = max(lo, v);
    }
    hi = max(hi, lo);
  }
  top = __shfl_sync(0xffffffffu, hi, last);
}

// The rows cut into units of at most `per` rows of one expert, numbered expert by expert.  The table, unit_ints(E) integers of shared
// memory: first[e], the units before expert e (first[E]: all of them), begin[e] and end[e], its rows.  Offsets are taken as clamped to
// [0, N] and ascending, whatever they hold.
template <int THREADS>
__device__ __forceinline__ void build_units(const Call& c, int per, int32_t* table) {
  for (int e = threadIdx.x; e < c.E; e += THREADS) {
    int64_t lo = 0, hi = c.N;
    if (c.offsets) {
      lo = __ldcg(c.offsets + e);
      hi = __ldcg(c.offsets + e + 1);
      lo = lo < 0 ? 0 : (lo > c.N ? c.N : lo);
      hi = hi < 0 ? 0 : (hi > c.N ? c.N : hi);
    }
    table[c.E + 1 + e] = static_cast<int32_t>(lo);   // N < 2^31
    table[2 * c.E + 1 + e] = static_cast<int32_t>(hi);
  }
  __syncthreads();
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    int before = 0, top = 0;
    for (int e0 = 0; e0 < c.E; e0 += 32) {
      const int e = e0 + lane;
      int lo = 0, hi = 0;
      if (e < c.E) {
        lo = table[c.E + 1 + e];
        hi = table[2 * c.E + 1 + e];
      }
      make_ascending(lo, hi, top, e < c.E, min(31, c.E - 1 - e0));
      if (e < c.E) {
        table[c.E + 1 + e] = lo;
        table[2 * c.E + 1 + e] = hi;
      }
      const int mine = (hi - lo + per - 1) / per;
      int upto = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += v;
      }
      if (e < c.E) table[e] = before + upto - mine;
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) table[c.E] = before;
  }
  // (a barrier of the block follows)
}
struct Unit {
  int e;
  int lo, hi;   // its rows
};
__device__ __forceinline__ Unit unit_at(const int32_t* table, int E, int per, int u) {
  int lo = 0, hi = E;   // the last e with first[e] <= u
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (table[mid] <= u) lo = mid;
    else hi = mid;
  }
  Unit r;
  r.e = lo;
  const int end = table[2 * E + 1 + lo];
  r.lo = table[E + 1 + lo] + (u - table[lo]) * per;
  r.hi = end - r.lo < per ? end : r.lo + per;
  return r;
}
inline int64_t most_units(const Call& c, int per) { return most_units(c.offsets != nullptr, c.N, c.E, per); }

// What a failed call of the runtime leaves behind is taken away with it: launch_status() of this thread's next call would report it.
inline pipe_status runtime_failed() {
  cudaGetLastError();
  return PIPE_ERR_CUDA;
}
// Lets a kernel be launched with up to `most` bytes of dynamic shared memory on the current device.  That limit is the kernel's, for all
// host threads: it is set once, to the most that any call asks for, so that no call lowers it under another one's launch.
bool allow_dynamic_smem(const void* kernel, int most);

pipe_status linear_small(const Call& c, bool bf16, cudaStream_t stream);
pipe_status linear_tc(const Call& c, bool bf16, cudaStream_t stream);

}  // namespace grp
}  // namespace pipe
