// Log probabilities of given tokens, entropy and top alternatives (definition: pipe_token_logprobs in include/pipe.h).
//
// One pass over the logits: a thread keeps the largest logit it has met, m, and under it the sums of exp(z - z_m) and of
// (l - m) exp(z - z_m), scaled anew when m grows; threads, warps and the CTAs of a row's cluster are joined likewise.  Bound by HBM, closely
// followed by the exponentials (one a logit) and the issue slots: 2048 rows of 128000 bf16 without alternatives 83 us, 6.3 TB/s; with 10 of
// them 101 (what a CTA does behind the pass is some 3 us in which it reads little).
// The alternatives cost no work in that pass: the k-th largest of the groups of threads' largest logits is not above the row's k-th
// largest, so only threads with one at least as large can hold an alternative, some k of them, and their logits alone are looked at
// again, in L2.  What is found (some more than k) is ranked by counting.  Where too many are found, as among equal
// logits, the k-th largest logit is settled by halving and the first of those equal to it are taken in the row's order.
#include "../group/group_common.cuh"

namespace pipe {
namespace lpb {

constexpr float kLog2e = 1.44269504f, kLn2 = 0.69314718f;
constexpr float kFar = -1e30f;     // differences below have probability 0 at every scale (2^-20 at least)
constexpr float kExact = 16777216.f;   // numbers up to it are rounded by one at most
constexpr uint32_t kOutside = 0x7F800001u;   // a given token that is none (of NaNs there is one)
constexpr int kFound = 544;        // most logits that are ranked: no less than a cluster's PIPE_MAX_TOP each
constexpr int kCluster = 8;
constexpr int kWide = 512, kMiddle = 256, kNarrow = 128, kResident = 1536, kRoomy = 1024;   // threads of a CTA, and of an SM
constexpr int kAhead = 4;                                      // vectors that a thread has in flight
static_assert(kFound >= kCluster * PIPE_MAX_TOP && kFound % 2 == 0, "");

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

// Keys that order like the numbers, -0 and 0 alike (adding 0 makes them one).
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float number_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }
constexpr uint32_t kNoneKey = 0x007FFFFFu;   // of -Inf
__device__ __forceinline__ float max_nan(float a, float b) {
  float d;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
  return d;
}
__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// 16 bytes of logits.
template <int SRC>
struct Vec {
  static constexpr int kLogits = SRC == PIPE_DTYPE_FP32 ? 4 : 8, kSize = SRC == PIPE_DTYPE_FP32 ? 4 : 2;
  uint32_t u[4];
  __device__ __forceinline__ void load(const uint8_t* p) {
    const uint4 a = __ldcg(reinterpret_cast<const uint4*>(p));
    u[0] = a.x; u[1] = a.y; u[2] = a.z; u[3] = a.w;
  }
  __device__ __forceinline__ void fill() {   // -Inf: not there
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = SRC == PIPE_DTYPE_FP32 ? 0xFF800000u : (SRC == PIPE_DTYPE_BF16 ? 0xFF80FF80u : 0xFC00FC00u);
  }
  __device__ __forceinline__ float at(int i) const {
    if constexpr (SRC == PIPE_DTYPE_FP32) return __uint_as_float(u[i]);
    else if constexpr (SRC == PIPE_DTYPE_BF16) return __uint_as_float(i & 1 ? u[i >> 1] & 0xFFFF0000u : u[i >> 1] << 16);
    else return grp::Fp16::to_float(static_cast<uint16_t>(i & 1 ? u[i >> 1] >> 16 : u[i >> 1]));
  }
  // (bf16: what is below kFar, -Inf among it, made that, a NaN kept)
  __device__ __forceinline__ void raise() {
    if constexpr (SRC == PIPE_DTYPE_BF16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) u[i] = larger2(u[i], 0xF14AF14Au);   // (-1.00025e30, no more than kFar)
    }
  }
  // the largest of these, a NaN if there is one
  static __device__ __forceinline__ uint32_t larger2(uint32_t a, uint32_t b) {
    uint32_t d;
    if constexpr (SRC == PIPE_DTYPE_BF16) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    else asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
  }
  template <int N>
  static __device__ __forceinline__ float largest(const Vec (&v)[N]) {
    if constexpr (SRC == PIPE_DTYPE_FP32) {
      float m = v[0].at(0);
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i + j) m = max_nan(m, v[j].at(i));
      return m;
    } else {
      uint32_t m = v[0].u[0];
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (i + j) m = larger2(m, v[j].u[i]);
      Vec one;
      one.u[0] = m;
      return max_nan(one.at(0), one.at(1));
    }
  }
};
template <int SRC>
__device__ __forceinline__ float logit(const uint8_t* row, int64_t i) {
  if constexpr (SRC == PIPE_DTYPE_FP32) return __ldcg(reinterpret_cast<const float*>(row) + i);
  const uint16_t h = __ldcg(reinterpret_cast<const uint16_t*>(row) + i);
  return SRC == PIPE_DTYPE_BF16 ? grp::Bf16::to_float(h) : grp::Fp16::to_float(h);
}

// The sums over some logits: m the largest (-Inf: none; a NaN or +Inf: no distribution), s = sum 2^z and h = sum z 2^z with
// z = c (l - m), c = scale log2 e.
struct Sums {
  float m, s, h;
};
// Those of N neighbouring lanes joined, the same in all of them (c: scale log2 e).
template <int N>
__device__ __forceinline__ Sums joined(const Sums& own, float c) {
  Sums r = own;
  if constexpr (N == 32) {
    asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r.m) : "f"(own.m));
  } else {
#pragma unroll
    for (int o = N / 2; o; o >>= 1) r.m = max_nan(r.m, __shfl_xor_sync(0xffffffffu, r.m, o));
  }
  const float z = fmaxf(fmaxf(own.m - fmaxf(r.m, -3.402823466e38f), kFar) * c, kFar), f = ex2(z);
  r.s = own.s * f;
  r.h = (own.h + own.s * z) * f;
#pragma unroll
  for (int o = N / 2; o; o >>= 1) {
    r.s += __shfl_xor_sync(0xffffffffu, r.s, o);
    r.h += __shfl_xor_sync(0xffffffffu, r.h, o);
  }
  return r;
}

// What of a row this CTA reads: `head` logits before the first 16-byte boundary (the first CTA's), vectors first .. end - 1 of those that
// begin there, and `tail` logits behind the last (the last CTA's).  Thread t has vectors first + t, first + t + B, .. and the t-th logit
// of head and tail.
struct Part {
  const uint8_t* row;
  const uint8_t* vectors;
  int head, tail, first, end, tail_at, head_all;
};
template <int SRC>
__device__ __forceinline__ Part part_of(const Args& a, int64_t t, int crank, int ctas) {   // (ctas: a power of two)
  constexpr int kLogits = Vec<SRC>::kLogits, kSize = Vec<SRC>::kSize;
  Part p;
  p.row = static_cast<const uint8_t*>(a.logits) + t * a.ldl * kSize;
  p.head_all = min(a.V, static_cast<int>((16 - (reinterpret_cast<uintptr_t>(p.row) & 15)) & 15) / kSize);
  p.vectors = p.row + p.head_all * kSize;
  const int all = (a.V - p.head_all) / kLogits;
  const int shift = 31 - __clz(ctas);
  p.first = static_cast<int>(static_cast<int64_t>(all) * crank >> shift);
  p.end = static_cast<int>(static_cast<int64_t>(all) * (crank + 1) >> shift);
  p.head = crank == 0 ? p.head_all : 0;
  p.tail_at = p.head_all + all * kLogits;
  p.tail = crank == ctas - 1 ? a.V - p.tail_at : 0;
  return p;
}

// A logit and its place as one number, larger for what is listed first: the key above, the place's complement below.  0: none.
using Entry = unsigned long long;
__device__ __forceinline__ Entry entry_of(float l, int i) { return (static_cast<Entry>(key_of(l)) << 32) | (0xFFFFFFFFu - static_cast<uint32_t>(i)); }
__device__ __forceinline__ uint32_t key_in(Entry e) { return static_cast<uint32_t>(e >> 32); }
__device__ __forceinline__ int place_in(Entry e) { return static_cast<int>(0xFFFFFFFFu - static_cast<uint32_t>(e)); }

constexpr int kGroups = 256, kFewGroups = 32;
// Up to so many alternatives the bound is that of kFewGroups groups: 31 logits are found for the 20 largest, on average, 12 for 10.  By few
// groups and by more (us, bf16): 4000 x 16000 k = 10 35.3, 36.1, 16 39.1, 38.9, 20 43.4, 41.0, 21 44.7, 41.5, 28 56, 46; 2048 x 128000 10 99.1, 101.6, 16
// 104.7, 106.9, 20 109.7, 108.6, 21 114, 107, 28 126, 115; one row of 32000 10 5.6, 5.9, 20 6.3, 6.2, 24 7.4, 6.9.
constexpr int kFewAlternatives = 20;
constexpr int kFewFound = 64;          // that one warp ranks, or a CTA hands to its cluster's first
static_assert(kFewFound >= PIPE_MAX_TOP && kCluster * kFewFound <= kFound, "");

// Shared memory of the search for the alternatives.
template <int B>
struct Search {
  alignas(16) Entry entry[kFound + 2];
  alignas(16) uint32_t group[kGroups];   // the largest logits of groups of threads, as keys
  int found, kept;
  uint32_t least;
  int run[2][B / 32];
};

// The logits of this CTA's part that are not below `least` (the key of a number), of threads whose largest, `own`, is not: entered, as long
// as there is room, and counted in s.found, or (COUNT) this thread's finds counted only.  Four vectors of a lane at a time: its own where no
// thread has more, otherwise the warp's lanes share out those of four threads.
// (All that follows the pass is written for few instructions: with 80 KB of them, as it was, every step waited for code.)
template <int SRC, int B, bool COUNT>
__device__ __forceinline__ int look_again(Search<B>& s, const Part& p, uint32_t own, uint32_t least) {
  constexpr int kLogits = Vec<SRC>::kLogits;
  const int lane = threadIdx.x & 31, first = p.first + static_cast<int>(threadIdx.x);
  const float bound = number_of(least);
  const bool mine = own >= least, few = p.end - p.first <= 4 * B;
  int finds = 0;
  auto enter = [&](int at, float l, int place) {
    if (at < kFound) s.entry[at] = entry_of(l, place);
  };
  uint32_t which = __ballot_sync(0xffffffffu, mine);
  while (which) {
    int from[4];   // a lane's vectors, one of each (p.end: none)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (few) {
        from[j] = mine ? first + j * B : p.end;
      } else {
        from[j] = which ? first - lane + __ffs(which) - 1 + lane * B : p.end;
        which &= which - 1;
      }
    }
    if (few) which = 0;
    for (int at = 0; p.first + at < p.end; at += 32 * B) {   // (at most 2^28 vectors)
      Vec<SRC> w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (from[j] + at < p.end) w[j].load(p.vectors + (from[j] + at) * int64_t{16});
        else w[j].fill();
      }
      uint32_t hits = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < kLogits; ++i) hits |= w[j].at(i) >= bound ? 1u << (j * kLogits + i) : 0u;
      if (COUNT) {
        finds += __popc(hits);
      } else if (hits) {
        int to = atomicAdd(&s.found, __popc(hits));
        for (; hits; hits &= hits - 1, ++to) {
          const int bit = __ffs(hits) - 1, j = bit / kLogits;
          Vec<SRC> v = w[0];   // that of the hit
          int place = from[0];
#pragma unroll
          for (int o = 1; o < 4; ++o)
            if (j == o) {
              v = w[o];
              place = from[o];
            }
          float l = v.at(0);
#pragma unroll
          for (int i = 1; i < kLogits; ++i)
            if (bit % kLogits == i) l = v.at(i);
          enter(to, l, p.head_all + (place + at) * kLogits + bit % kLogits);
        }
      }
      if (few) break;
    }
  }
#pragma unroll 1
  for (int of = 0; of < 2; ++of) {
    if (static_cast<int>(threadIdx.x) >= (of ? p.tail : p.head)) continue;
    const int at = (of ? p.tail_at : 0) + static_cast<int>(threadIdx.x);
    const float l = logit<SRC>(p.row, at);
    if (!(l >= bound)) continue;
    if (COUNT) ++finds;
    else enter(atomicAdd(&s.found, 1), l, at);
  }
  return finds;
}

// put(i, entry) for the k largest of the entries, or all of them, i their rank, by threads from .. of the CTA or, where they are few, by the
// first warp alone.  (A barrier has to stand before, and behind unless they are few.)
template <int B, class F>
__device__ __forceinline__ void rank(Search<B>& s, int count, int k, F put) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (count > 2 * k + 64) {
    // first brought down to some more than k by one warp, by halving between the least and the largest of their keys
    if (warp == 0) {
      const uint32_t* key = reinterpret_cast<const uint32_t*>(s.entry) + 1;   // (of entry i: key[2 i])
      uint32_t lo = ~0u, hi = 0;
      for (int i = lane; i < count; i += 32) {
        const uint32_t v = key[2 * i];
        hi = max(hi, v);
        lo = min(lo, v);
      }
      lo = __reduce_min_sync(0xffffffffu, lo);
      hi = __reduce_max_sync(0xffffffffu, hi);
      int n = count;
      while (lo < hi && n > k + 16) {
        const uint32_t half = lo + (hi - lo + 1) / 2;
        int c = 0;
#pragma unroll 4
        for (int i = lane; i < count; i += 32) c += key[2 * i] >= half;
        c = __reduce_add_sync(0xffffffffu, c);
        if (c >= k) {
          lo = half;
          n = c;
        } else {
          hi = half - 1;
        }
      }
      int kept = 0;
      for (int i0 = 0; i0 < count; i0 += 32) {
        const Entry e = i0 + lane < count ? s.entry[i0 + lane] : 0;
        const bool in = e != 0 && key_in(e) >= lo;
        const uint32_t m = __ballot_sync(0xffffffffu, in);   // (these have been read: what is written lies at or before them)
        if (in) s.entry[kept + __popc(m & ((1u << lane) - 1))] = e;
        kept += __popc(m);
        __syncwarp();
      }
      if (lane == 0) s.kept = kept;
    }
    __syncthreads();
    count = s.kept;
  }
  const bool few = count <= kFewFound;
  if (few && warp != 0) return;
  if (threadIdx.x == 0) s.entry[count] = 0;   // (read with the last one where their number is odd)
  if (few) __syncwarp();
  else __syncthreads();
  for (int i = threadIdx.x; i < count; i += few ? 32 : B) {
    const Entry e = s.entry[i];
    int above = 0;
#pragma unroll 4
    for (int j = 0; j < count; j += 2) {
      const ulonglong2 two = *reinterpret_cast<const ulonglong2*>(s.entry + j);
      above += (two.x > e) + (two.y > e);
    }
    if (above < k) put(above, e);
  }
}

// The largest logits of groups of threads, for search (a barrier has to stand between).  m: the largest of this thread's.
template <int B>
__device__ __forceinline__ bool few_groups(const Part& p, int k) {   // (every group has logits then)
  return k <= kFewAlternatives && p.end - p.first >= B;
}
template <int B>
__device__ __forceinline__ void group(Search<B>& s, const Part& p, float m, int k) {
  uint32_t most = key_of(m);
  if (threadIdx.x == 0) s.found = 0;
  if (few_groups<B>(p, k)) {
    constexpr int kSize = B / kFewGroups;
#pragma unroll
    for (int o = 1; o < kSize; o *= 2) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (threadIdx.x % kSize == 0) s.group[threadIdx.x / kSize] = most;
    return;
  }
  int size = 1;
  if (B > kGroups) {
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
    size = 2;
    if (k <= 32) {
      most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
      size = 4;
    }
  }
  for (int i = threadIdx.x; i < kGroups; i += B)
    if (i >= B / size) s.group[i] = 0;
  if (threadIdx.x % size == 0) s.group[threadIdx.x / size] = most;
}

// Where more logits than there is room for are not below the bound: fills s.entry with the k first of this CTA's part, in any order.
template <int SRC, int B>
__device__ __noinline__ int search_by_halves(Search<B>& s, const Part p, uint32_t own, uint32_t least, int k) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // The key of the k-th largest, by halving between that bound and the largest.
  uint32_t hi = 0;
  for (int g = lane; g < (few_groups<B>(p, k) ? kFewGroups : kGroups); g += 32) hi = max(hi, s.group[g]);
  hi = __reduce_max_sync(0xffffffffu, hi);
  for (int turn = 0; least < hi; turn ^= 1) {   // (the same in all threads; at least k logits reach `least`)
    const uint32_t mid = least + (hi - least + 1) / 2;
    int c = look_again<SRC, B, true>(s, p, own, mid);
    c = __reduce_add_sync(0xffffffffu, c);
    if (lane == 0) s.run[turn][warp] = c;
    __syncthreads();
    c = 0;
#pragma unroll
    for (int w = 0; w < B / 32; ++w) c += s.run[turn][w];
    if (c >= k) least = mid;
    else hi = mid - 1;
  }
  // Those above it, fewer than k, in any order; then the first that are equal to it, in the row's order.
  __syncthreads();
  if (threadIdx.x == 0) s.found = 0;
  __syncthreads();
  look_again<SRC, B, false>(s, p, own, least + 1);
  __syncthreads();
  int have = s.found;
  constexpr int kLogits = Vec<SRC>::kLogits;
  const float bound = number_of(least);
  const int steps = (p.end - p.first + B - 1) / B;   // of the block through its vectors; the head before, the tail behind
  for (int st = -1; st <= steps && have < k; ++st) {
    uint32_t equal = 0;
    int base = 0;
    if (st < 0 || st == steps) {
      base = st < 0 ? static_cast<int>(threadIdx.x) : p.tail_at + static_cast<int>(threadIdx.x);
      if (static_cast<int>(threadIdx.x) < (st < 0 ? p.head : p.tail)) equal = logit<SRC>(p.row, base) == bound;
    } else {
      const int v = p.first + st * B + static_cast<int>(threadIdx.x);
      base = p.head_all + v * kLogits;
      if (v < p.end) {
        Vec<SRC> w;
        w.load(p.vectors + v * int64_t{16});
#pragma unroll
        for (int i = 0; i < kLogits; ++i) equal |= static_cast<uint32_t>(w.at(i) == bound) << i;
      }
    }
    int upto = __popc(equal);
    const int mine = upto;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, d);
      if (lane >= d) upto += v;
    }
    if (lane == 31) s.run[0][warp] = upto;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < B / 32; ++w) {
      if (w < warp) before += s.run[0][w];
      all += s.run[0][w];
    }
    int at = have + before + upto - mine;
    for (; equal && at < k; equal &= equal - 1, ++at) s.entry[at] = entry_of(bound, base + __ffs(equal) - 1);
    have = min(have + all, k);
    __syncthreads();
  }
  return have;
}

// Fills s.entry with logits of this CTA's part, in any order, the k first of them among these or all that there are; returns their number,
// kFound at most.  m: the largest of this thread's.
template <int SRC, int B>
__device__ __forceinline__ int search(Search<B>& s, const Part& p, float m, int k) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t own = key_of(m);
  // A bound for the k-th largest: of disjoint groups of threads at least k have one as large (or kNoneKey + 1, the least that is not masked,
  // where there are fewer than k).  Of 32 groups that is the k-th largest, of more one not far below it, by halving.
  if (warp == 0) {
    uint32_t lo = kNoneKey + 1;
    if (few_groups<B>(p, k)) {
      const uint32_t mine = s.group[lane];
      int above = 0;
#pragma unroll
      for (int i = 0; i < kFewGroups; i += 4) {
        const uint4 four = *reinterpret_cast<const uint4*>(s.group + i);
        above += (four.x > mine) + (four.y > mine) + (four.z > mine) + (four.w > mine);
      }
      lo = max(lo, __reduce_min_sync(0xffffffffu, above < k ? mine : ~0u));
    } else {
      uint32_t mine[kGroups / 32], hi = 0;
#pragma unroll
      for (int i = 0; i < kGroups / 32; ++i) {
        mine[i] = s.group[32 * i + lane];
        hi = max(hi, mine[i]);
      }
      if (k <= 32) lo = max(lo, __reduce_min_sync(0xffffffffu, hi));   // (every lane has a group as large as that)
      hi = __reduce_max_sync(0xffffffffu, hi);
      int n = kGroups;
      while (lo < hi && n > k + (k >> 2) + 2) {
        const uint32_t mid = lo + (hi - lo + 1) / 2;
        int c = 0;
#pragma unroll
        for (int i = 0; i < kGroups / 32; ++i) c += mine[i] >= mid;
        c = __reduce_add_sync(0xffffffffu, c);
        if (c >= k) {
          lo = mid;
          n = c;
        } else {
          hi = mid - 1;
        }
      }
    }
    if (lane == 0) s.least = lo;
  }
  __syncthreads();
  const uint32_t least = s.least;
  look_again<SRC, B, false>(s, p, own, least);
  __syncthreads();
  const int found = s.found;
  return found <= kFound ? found : search_by_halves<SRC, B>(s, p, own, least, k);
}

// B threads a CTA, R an SM; a CTA a row, or with kRoomy threads an SM a cluster of them.  ENT: the entropy is wanted.
template <int SRC, int B, int R, bool ENT>
__global__ void __launch_bounds__(B, R / B) logprobs_kernel(const Args a) {
  constexpr int kLogits = Vec<SRC>::kLogits;
  __shared__ Search<B> search_s;
  __shared__ Sums warp_s[B / 32];
  __shared__ Sums own_s;                     // this CTA's
  __shared__ int count_s;
  __shared__ Entry top_s[PIPE_MAX_TOP];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  constexpr bool kClusters = R == kRoomy;   // (the others have one CTA a row)
  const int ctas = kClusters ? grp::cluster_ctas() : 1, crank = kClusters ? grp::cluster_rank() : 0;
  const int64_t t = blockIdx.x >> (31 - __clz(ctas));
  const Part p = part_of<SRC>(a, t, crank, ctas);
  const float c = a.scale * kLog2e;
  grid_wait();
  grid_release();

  // a given token and its logit, on their way while the row is read
  const int turn = static_cast<int>(threadIdx.x + 32) & (B - 1);   // (the last warp's first: the first one has the alternatives' bound to find)
  auto given_of = [&](int64_t at) {   // its bits, or kOutside, which no number has
    const int token = __ldcg(a.tokens + at);
    if (token < 0 || token >= a.V) return kOutside;
    const float l = logit<SRC>(p.row, token);
    return __float_as_uint(l == l ? l : __int_as_float(0x7FC00000));
  };
  uint32_t given = kOutside;
  if (crank == 0 && turn < a.n) given = given_of(t * a.n + turn);
  // The pass.  z is formed by one fused operation, c l - ref with ref = c m rounded: the same ref for all, so that what its rounding adds to
  // every z, one at most as long as c m is within kExact, cancels in the end.  Beyond that ref stays at kExact: the sums are then no use, but
  // nothing in them is infinite as long as m is negative, and they are made anew (below) should m stay there.
  Sums own = {-INFINITY, 0.f, 0.f};
  float ref = -kExact;
  f32x2 s2 = both_f2(0.f), h2 = both_f2(0.f);
  auto grow = [&](float m) {   // a new largest logit
    const float to = fminf(fmaxf(m * c, -kExact), kExact), z = ref - to, f = ex2(z);
    if (ENT) h2 = mul_f2(fma_f2(s2, both_f2(z), h2), both_f2(f));
    s2 = mul_f2(s2, both_f2(f));
    own.m = m;
    ref = to;
  };
  auto take = [&](Vec<SRC> (&v)[kAhead], int some) {   // `some` of these are there: the same number in a whole warp
    const float m = max_nan(own.m, Vec<SRC>::largest(v));
    if (!(m <= own.m)) grow(m);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (j >= some) break;
      if (ENT) v[j].raise();
#pragma unroll
      for (int i = 0; i < kLogits; i += 2) {
        f32x2 z = fma_f2(pack_f2(v[j].at(i), v[j].at(i + 1)), both_f2(c), both_f2(-ref));
        float z0, z1;
        unpack_f2(z, z0, z1);
        if (ENT && SRC != PIPE_DTYPE_BF16) {   // (an infinite z times its power would be no number)
          z0 = fmaxf(z0, kFar);
          z1 = fmaxf(z1, kFar);
          z = pack_f2(z0, z1);
        }
        const f32x2 e = pack_f2(ex2(z0), ex2(z1));
        s2 = add_f2(s2, e);
        if (ENT) h2 = fma_f2(z, e, h2);
      }
    }
  };
  // whole batches first: loads at fixed distances, nothing to be asked for each (with conditions: 8 instructions a logit, of which 4 its own)
  int v0 = p.first + static_cast<int>(threadIdx.x);
  const uint8_t* from = p.vectors + v0 * int64_t{16};
  for (; v0 - lane + 31 + (kAhead - 1) * B < p.end; v0 += kAhead * B, from += kAhead * B * 16) {   // (at most 2^28 vectors)
    Vec<SRC> v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) v[j].load(from + j * B * 16);
    take(v, kAhead);
  }
  if (v0 - lane < p.end) {
    Vec<SRC> v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (v0 + j * B < p.end) v[j].load(from + j * B * 16);
      else v[j].fill();
    }
    take(v, (p.end - (v0 - lane) + B - 1) / B);
  }
#pragma unroll
  for (int which = 0; which < 2; ++which)
    if (static_cast<int>(threadIdx.x) < (which ? p.tail : p.head)) {
      const float l = logit<SRC>(p.row, (which ? p.tail_at : 0) + static_cast<int>(threadIdx.x)), m = max_nan(own.m, l);
      if (!(m <= own.m)) grow(m);
      const float z = fmaxf(fmaf(l, c, -ref), kFar), e = ex2(z);
      s2 = add_f2(s2, pack_f2(e, 0.f));
      h2 = fma_f2(both_f2(z), pack_f2(e, 0.f), h2);
    }
  const float mine = own.m;
  {
    float x, y;
    unpack_f2(s2, x, y);
    own.s = x + y;
    unpack_f2(h2, x, y);
    own.h = x + y;
  }
  if (fabsf(mine * c) <= kExact) {   // from ref to c m
    const float z = fmaf(mine, c, -ref), f = ex2(-z);
    own.h = (own.h - own.s * z) * f;
    own.s *= f;
  } else if (fabsf(mine) <= 3.402823466e38f) {
    // (a thread that has nothing but masked by large negative numbers, as a rule): once more, by differences
    own.s = own.h = 0.f;
    auto add = [&](float l) {
      const float z = fmaxf(fmaxf(l - mine, kFar) * c, kFar), e = ex2(z);
      own.s += e;
      own.h += z * e;
    };
    for (int v = p.first + static_cast<int>(threadIdx.x); v < p.end; v += B) {
      Vec<SRC> w;
      w.load(p.vectors + v * int64_t{16});
#pragma unroll
      for (int i = 0; i < kLogits; ++i) add(w.at(i));
    }
    if (static_cast<int>(threadIdx.x) < p.head) add(logit<SRC>(p.row, threadIdx.x));
    if (static_cast<int>(threadIdx.x) < p.tail) add(logit<SRC>(p.row, p.tail_at + static_cast<int>(threadIdx.x)));
  }
  own = joined<32>(own, c);
  if (a.k > 0) group(search_s, p, mine, a.k);
  if (lane == 0) warp_s[warp] = own;
  __syncthreads();
  own = joined<B / 32>(warp_s[lane & (B / 32 - 1)], c);   // (in every lane)
  // What the row's first CTA writes, when `own` is the row's.
  const float nan = __int_as_float(0x7FC00000);
  // (halves: the difference of two logits may be beyond the type's range where its product with the scale is not)
  auto is_bad = [&] { return !(own.m <= 3.402823466e38f); };
  auto logprob = [&](float l, float logs) {
    return is_bad() ? nan : (own.m == -INFINITY || l == -INFINITY ? -INFINITY : (0.5f * l - 0.5f * own.m) * a.scale * 2.f - logs);
  };
  // (the largest logit's term is 1, so no sum is less; what two exponentials of opposite numbers lose may have left it 2^-24 below, and a log
  // probability above 0)
  auto log_sum = [&] { return logf(fmaxf(own.s, 1.f)); };
  auto write_sums = [&] {
    if (turn >= max(a.n, 1)) return;
    const float logs = log_sum();
    if (turn == 0) {
      if (is_bad()) raise_status(a.status, PIPE_ERR_NONFINITE);
      if (ENT) a.entropy[t] = is_bad() ? nan : (own.m == -INFINITY ? 0.f : fmaxf(logs - kLn2 * own.h / own.s, 0.f));
    }
    for (int j = turn; j < a.n; j += B) {
      if (j >= B) given = given_of(t * a.n + j);
      a.logprobs[t * a.n + j] = given != kOutside ? logprob(__uint_as_float(given), logs) : 0.f;
    }
  };
  auto write_alternatives = [&](int count) {   // of the entries, and none behind them
    for (int i = count + static_cast<int>(threadIdx.x); i < a.k; i += B) {
      if (a.top) a.top[t * a.k + i] = -1;
      if (a.top_logprobs) a.top_logprobs[t * a.k + i] = is_bad() ? nan : -INFINITY;
    }
    if (count <= 0) return;
    const float logs = log_sum();
    rank(search_s, count, a.k, [&](int i, Entry e) {
      if (a.top) a.top[t * a.k + i] = place_in(e);
      if (a.top_logprobs) a.top_logprobs[t * a.k + i] = logprob(number_of(key_in(e)), logs);
    });
  };
  if (ctas == 1) write_sums();
  if (ctas == 1 && a.k == 0) return;
  // (a row that is no distribution has no alternatives, in whichever CTA that shows)
  int count = a.k > 0 && own.m <= 3.402823466e38f ? search<SRC, B>(search_s, p, mine, a.k) : 0;
  if (ctas == 1) {
    write_alternatives(count);
    return;
  }
  if (count > kFewFound) {
    __syncthreads();
    rank(search_s, count, a.k, [&](int i, Entry e) { top_s[i] = e; });
    __syncthreads();
    count = a.k;
    for (int i = threadIdx.x; i < count; i += B) search_s.entry[i] = top_s[i];
  }
  if (threadIdx.x == 0) {
    own_s = own;
    count_s = count;
  }
  grp::cluster_sync();
  if (crank == 0) {
    Sums others = {-INFINITY, 0.f, 0.f};
    const int from = lane & (kCluster - 1);
    int upto = 0;   // entries of the CTAs up to this lane's
    if (from < ctas) {
      others = Sums{grp::cluster_load(&own_s.m, from), grp::cluster_load(&own_s.s, from), grp::cluster_load(&own_s.h, from)};
      upto = grp::cluster_load(&count_s, from);
    }
    own = joined<kCluster>(others, c);
#pragma unroll
    for (int d = 1; d < kCluster; d *= 2) {
      const int v = __shfl_up_sync(0xffffffffu, upto, d);
      if (from >= d) upto += v;
    }
    // a warp for every other CTA's entries
    for (int r = warp + 1; r < ctas; r += B / 32) {
      const int at = __shfl_sync(0xffffffffu, upto, r - 1), n = __shfl_sync(0xffffffffu, upto, r) - at;
      for (int i = lane; i < n; i += 32)
        asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(search_s.entry[at + i]) : "r"(grp::cluster_address(search_s.entry + i, r)) : "memory");
    }
    count = __shfl_sync(0xffffffffu, upto, kCluster - 1);
  }
  grp::cluster_sync();   // (no CTA leaves while another reads its memory)
  if (crank != 0) return;
  write_sums();
  write_alternatives(is_bad() ? 0 : count);
}

using Kernel = void (*)(Args);
template <int SRC>
static Kernel logprobs_of(int threads, bool roomy, bool entropy) {
  if (roomy) return entropy ? logprobs_kernel<SRC, kWide, kRoomy, true> : logprobs_kernel<SRC, kWide, kRoomy, false>;
  if (threads == kWide) return entropy ? logprobs_kernel<SRC, kWide, kResident, true> : logprobs_kernel<SRC, kWide, kResident, false>;
  if (threads == kMiddle) return entropy ? logprobs_kernel<SRC, kMiddle, kResident, true> : logprobs_kernel<SRC, kMiddle, kResident, false>;
  return entropy ? logprobs_kernel<SRC, kNarrow, kResident, true> : logprobs_kernel<SRC, kNarrow, kResident, false>;
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
  // Threads of a row: behind the pass a CTA is some 3 us busy with joins, search and ranking whatever its size, so that many rows want many
  // small CTAs on an SM, a long row one that reads it fast, and rows that are all on the chip at once as many threads as there are.  With 10
  // alternatives and the entropy (us; 128, 256 and 512 threads): 4000 rows of 16 KB 27, 34, 58, of 40 KB 42, 49, 71, of 64 KB 61, 60, 79, of
  // 128 KB 128, 102, 111, of 256 KB 255, 202, 186; 300 rows of 16 KB 7.3, 5.9, 7.9; 290 of 128 KB 256 threads 15.1, 512 12.9.
  const int64_t bytes = static_cast<int64_t>(V) * (dtype == PIPE_DTYPE_FP32 ? 4 : 2), roomy_ctas = lpb::kRoomy / lpb::kWide * kPlanSMs;
  int threads = bytes <= 49152 ? lpb::kNarrow : (bytes <= 163840 ? lpb::kMiddle : lpb::kWide);
  if (T <= 3 * kPlanSMs && bytes > 8192 && threads < lpb::kMiddle) threads = lpb::kMiddle;
  if (T <= roomy_ctas && bytes > 16384) threads = lpb::kWide;
  // CTAs of 512 that are on the chip at once at 64 registers a thread have as many: 30 rows of 256 KB 9.6 us (at 40: 11.3).
  const bool roomy = threads == lpb::kWide && T <= roomy_ctas;
  // A few long rows have several CTAs (1, 2, 4 and 8): one row of 256 KB 9.6, 8.6, 8.2, 7.5, 60 rows 13.3, 11.2, 11.8, 18.0, one of 64 KB 5.9,
  // 6.4, 6.8, 7.6.
  int ctas = 1;
  while (roomy && ctas < lpb::kCluster && bytes > 98304 && T * ctas * 2 <= kPlanSMs) ctas *= 2;
  const lpb::Kernel kern = dtype == PIPE_DTYPE_FP32 ? lpb::logprobs_of<PIPE_DTYPE_FP32>(threads, roomy, d_entropy != nullptr)
                                                    : (dtype == PIPE_DTYPE_BF16 ? lpb::logprobs_of<PIPE_DTYPE_BF16>(threads, roomy, d_entropy != nullptr)
                                                                                : lpb::logprobs_of<PIPE_DTYPE_FP16>(threads, roomy, d_entropy != nullptr));
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (launch_overlapped(kern, dim3(static_cast<unsigned>(T * ctas)), threads, ctas, true, s, a) != cudaSuccess) return grp::runtime_failed();
  count_launch(1);
  take_expansion_mark(s);
  return launch_status();
}
