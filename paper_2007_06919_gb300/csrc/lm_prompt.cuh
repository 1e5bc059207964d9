// lm_prompt.cuh -- what the two kernels of attention over packed prompts share: the exponential, packed pairs, and a block's job.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "kernels.h"
#include "lm_seq.cuh"

namespace aqd {
namespace prompt {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack(float a, float b, __half*) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack(float a, float b, __nv_bfloat16*) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
struct Job {
  int32_t found, start, queries, kv_start, keys, tile;
};
__device__ __forceinline__ int clamp_at(int64_t v, int64_t most) { return (int)(v < 0 ? 0 : v > most ? most : v); }

// Unit `unit`'s sequence and tile of `rows` queries, the last tiles of a sequence (which see the most keys) first.
static __device__ __forceinline__ bool find_job(const PromptArgs& p, int rows, int unit, Job* job, uint64_t* red) {
  if (threadIdx.x == 0) job->found = 0;
  uint64_t base = 0;
  for (int b = 0; b < p.seqs; b += blockDim.x) {
    const int s = b + threadIdx.x;
    int start = 0, queries = 0, tiles = 0;
    if (s < p.seqs) {
      start = clamp_at(p.starts[s], p.tokens);
      const int end = clamp_at(p.starts[s + 1], p.tokens);
      queries = end > start ? end - start : 0;
      tiles = (queries + rows - 1) / rows;
    }
    uint64_t before;
    const uint64_t total = seq::block_scan((uint64_t)tiles, red, before);
    const int64_t first = (int64_t)(base + before);
    if (unit >= first && unit < first + tiles) {
      const int32_t* ks = p.kv_starts ? p.kv_starts : p.starts;
      const int k0 = clamp_at(ks[s], p.kv_tokens), k1 = clamp_at(ks[s + 1], p.kv_tokens);
      *job = {1, start, queries, k0, k1 > k0 ? k1 - k0 : 0, tiles - 1 - (int)(unit - first)};
    }
    base += total;
    if ((uint64_t)unit < base) break;
  }
  __syncthreads();
  return job->found != 0;
}


}  // namespace prompt
}  // namespace aqd
