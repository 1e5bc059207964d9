// lm_seq.cuh -- packed sequences of the attention kernels: a block finds its sequence by a scan over all of them, so the grid needs no
// more than an upper bound of the units and the host never reads lengths.
#pragma once
#include <cstdint>

namespace aqd {
namespace seq {

// Sum of a block's threads' counts, and the sum before each. red: a word for each warp.
__device__ __forceinline__ uint64_t block_scan(uint64_t v, uint64_t* red, uint64_t& before) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  uint64_t s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t u = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += u;
  }
  __syncthreads();  // (red may still be read from the last call)
  if (lane == 31) red[warp] = s;
  __syncthreads();
  uint64_t total = 0, base = 0;
  for (int w = 0; w < warps; ++w) {
    const uint64_t u = red[w];
    if (w < warp) base += u;
    total += u;
  }
  before = base + s - v;
  return total;
}

}  // namespace seq
}  // namespace aqd
