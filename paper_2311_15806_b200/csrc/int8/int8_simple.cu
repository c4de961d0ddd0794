// Products of the 8-bit integer layers, the simplest form: a block of 16 x 16 threads, an output each, four codes at a time.
#include "int8_common.cuh"

namespace pipe {
namespace i8 {

template <class H>
__global__ void __launch_bounds__(256) int8_simple_kernel(const Call p, int otiles) {
  extern __shared__ int32_t table[];
  __shared__ uint32_t ws[16][17], xs[16][17];
  grid_wait();
  grid_release();
  const grp::Call& c = p.c;
  grp::build_units<256>(c, 16, table);
  __syncthreads();
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int64_t tiles = static_cast<int64_t>(table[c.E]) * otiles;
  for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
    const grp::Unit u = grp::unit_at(table, c.E, 16, static_cast<int>(t / otiles));
    const int o0 = static_cast<int>(t % otiles) * 16;
    int acc = 0;
    for (int k0 = 0; k0 < c.I; k0 += 64) {
      const int k = k0 + 4 * tx;
      auto word = [&](const int8_t* row) {
        uint32_t v = 0;
        for (int j = 0; j < 4; ++j)
          if (k + j < c.I) v |= static_cast<uint32_t>(static_cast<uint8_t>(__ldcg(row + k + j))) << (8 * j);
        return v;
      };
      ws[ty][tx] = o0 + ty < c.O ? word(p.w + (static_cast<int64_t>(u.e) * c.O + o0 + ty) * p.ldw) : 0u;
      xs[ty][tx] = u.lo + ty < u.hi ? word(static_cast<const int8_t*>(c.x) + (u.lo + ty) * c.ldx) : 0u;
      __syncthreads();
      for (int j = 0; j < 16; ++j) acc = __dp4a(static_cast<int>(xs[ty][j]), static_cast<int>(ws[tx][j]), acc);
      __syncthreads();
    }
    const int o = o0 + tx, row = u.lo + ty;
    if (o < c.O && row < u.hi) {
      const int64_t ch = static_cast<int64_t>(u.e) * c.O + o;
      float v[1] = {scaled(acc, __ldcg(p.sw + ch), __ldcg(p.sx + row), c.bias ? H::load(c.bias, ch) : 0.f)};
      grp::quick_activation(v, c.act);
      H::store(c.y, row * c.ldy + o, v[0]);
    }
  }
}

pipe_status linear_simple(const Call& c, cudaStream_t stream) {
  const int otiles = ceil_div(c.c.O, 16);
  const int64_t tiles = grp::most_units(c.c, 16) * otiles;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(static_cast<unsigned>(tiles < 65536 ? tiles : 65536));
  cfg.blockDim = dim3(256);
  cfg.dynamicSmemBytes = grp::unit_ints(c.c.E) * 4;
  cfg.stream = stream;
  const auto k = c.dtype == PIPE_DTYPE_FP32 ? int8_simple_kernel<Fp32> : (c.dtype == PIPE_DTYPE_BF16 ? int8_simple_kernel<Bf16> : int8_simple_kernel<Fp16>);
  if (cudaLaunchKernelEx(&cfg, k, c, otiles) != cudaSuccess) return grp::runtime_failed();
  count_launch(1);
  return launch_status();
}

}  // namespace i8
}  // namespace pipe
