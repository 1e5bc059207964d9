// lm_prompt.cuh -- what the two kernels of attention over packed prompts share: the exponential, packed pairs, and a block's job.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

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
// Scores' factor in powers of two, neither 0 nor infinite (a difference of 0 times it is 0).
__device__ __forceinline__ float factor(float scale) { return fminf(fmaxf(scale * kLog2e, 1.4e-45f), 3.402823466e38f); }
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

// Values that the causal order hides from a row, in the last tiles of keys that its block takes: a weight of 0 does not keep out a NaN or an infinity, since 0
// times it is NaN. Rows behind whose last key such a value lies are taken again after the products, key by key, one warp a row. (16,384 tokens of 32 heads of 128 whose
// last value row holds a NaN, 127 rows a head: 41 ms, where the call takes 1.3; with a lane to a key, and its 32 rows' sectors in turn, 157.)

__device__ __forceinline__ float2 pair_of(uint32_t w, __half*) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ float2 pair_of(uint32_t w, __nv_bfloat16*) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }

// The last of the keys lo .. hi - 1 whose value row has a NaN or an infinity, or -1: a lane to a key. row(t, i): 16 bytes of it.
template <class T, int D, class Row>
__device__ __forceinline__ int last_not_finite(int lo, int hi, Row row) {
  constexpr uint32_t kExponent = std::is_same<T, __half>::value ? 0x7c007c00u : 0x7f807f80u, kLow = kExponent & 0xffffu;
  const int lane = threadIdx.x & 31;
  for (int end = hi; end > lo; end -= 32) {
    const int t = end - 32 + lane;
    bool bad = false;
    if (t >= lo) {
#pragma unroll 4
      for (int i = 0; i < D / 8; ++i) {
        const uint4 x = row(t, i);
        const uint32_t w[4] = {x.x & kExponent, x.y & kExponent, x.z & kExponent, x.w & kExponent};
#pragma unroll
        for (int j = 0; j < 4; ++j) bad = bad || (w[j] & 0xffffu) == kLow || w[j] >= kLow << 16;
      }
    }
    const uint32_t found = __ballot_sync(0xffffffffu, bad);
    if (found) return end - 1 - __clz(found);
  }
  return -1;
}
// Keys that row `at` of a job's sequence sees, in causal order.
__device__ __forceinline__ int seen_by(const Job& jb, int at) {
  const int64_t see = (int64_t)at + (jb.keys - jb.queries) + 1;
  return (int)(see < 0 ? 0 : see > jb.keys ? jb.keys : see);
}
// Output of row `at` of a job's sequence, eight keys at a time: a lane has D / 32 channels of each, adds up its part of their scores, and the lanes' parts are
// added so that lane n is left with key n's (and those lanes with it that have its number but for higher bits); weights times values as above.
template <class T, int D>
__device__ __forceinline__ void attend_again(const PromptArgs& p, const Job& jb, int head, int at) {
  constexpr int kPairs = D / 64, kKeys = 8;
  const int lane = threadIdx.x & 31, kvh = head / (p.heads / p.kv_heads), lim = seen_by(jb, at);
  const T* k = static_cast<const T*>(p.k) + (int64_t)jb.kv_start * p.ldk + (int64_t)kvh * p.ldkh + lane * (D / 32);
  const T* v = static_cast<const T*>(p.v) + (int64_t)jb.kv_start * p.ldv + (int64_t)kvh * p.ldvh + lane * (D / 32);
  const float c2 = factor(p.scale);
  float m = -INFINITY, l = 0.0f;
  float2 q[kPairs], o[kPairs];
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    q[i] = pair_of(*reinterpret_cast<const uint32_t*>(static_cast<const T*>(p.q) + (int64_t)(jb.start + at) * p.ldq + (int64_t)head * p.ldqh + lane * (D / 32) + 2 * i), (T*)nullptr);
    o[i] = make_float2(0.0f, 0.0f);
  }
  for (int t0 = 0; t0 < lim; t0 += kKeys) {
    const int here = lim - t0 < kKeys ? lim - t0 : kKeys;
    uint32_t x[kKeys][kPairs];
    auto load = [&](const T* rows, int64_t ld) {
#pragma unroll
      for (int j = 0; j < kKeys; ++j)
#pragma unroll
        for (int i = 0; i < kPairs; ++i) x[j][i] = j < here ? *reinterpret_cast<const uint32_t*>(rows + (t0 + j) * ld + 2 * i) : 0u;
    };
    load(k, p.ldk);
    float s[kKeys];
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {
      s[j] = 0.0f;
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const float2 u = pair_of(x[j][i], (T*)nullptr);
        s[j] = fmaf(q[i].x, u.x, fmaf(q[i].y, u.y, s[j]));
      }
    }
    load(v, p.ldv);  // (on its way while the scores are added)
#pragma unroll
    for (int n = kKeys / 2; n > 0; n >>= 1)
#pragma unroll
      for (int j = 0; j < n; ++j) {  // a lane keeps one of keys j and j + n, and gives the other away
        const bool upper = lane & n;
        const float mine = upper ? s[j + n] : s[j], other = upper ? s[j] : s[j + n];
        s[j] = mine + __shfl_xor_sync(0xffffffffu, other, n);
      }
    float score = s[0];
#pragma unroll
    for (int n = kKeys; n < 32; n <<= 1) score += __shfl_xor_sync(0xffffffffu, score, n);
    if ((lane & (kKeys - 1)) >= here) score = -INFINITY;
    float top = score;
    for (int n = kKeys / 2; n > 0; n >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, n));
    top = fmaxf(m, top);
    const float ref = top == -INFINITY ? 0.0f : top, f = ex2((m - ref) * c2), w = ex2((score - ref) * c2);
    const uint32_t w2 = pack(w, w, (T*)nullptr);
    m = top;
    l = fmaf(l, f, w);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) { o[i].x *= f; o[i].y *= f; }
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {  // (keys behind the last: weights of 0, values of 0)
      const float y = pair_of(__shfl_sync(0xffffffffu, w2, j), (T*)nullptr).x;
#pragma unroll
      for (int i = 0; i < kPairs; ++i) {
        const float2 u = pair_of(x[j][i], (T*)nullptr);
        o[i].x = fmaf(y, u.x, o[i].x);
        o[i].y = fmaf(y, u.y, o[i].y);
      }
    }
    bool lost = true;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) lost = lost && isnan(o[i].x) && isnan(o[i].y);
    if (__all_sync(0xffffffffu, lost)) break;  // (nothing is left to find)
  }
  for (int n = kKeys / 2; n > 0; n >>= 1) l += __shfl_xor_sync(0xffffffffu, l, n);
  const float inv = m == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l;
  T* y = static_cast<T*>(p.out) + (int64_t)(jb.start + at) * p.ldo + (int64_t)head * p.ldoh + lane * (D / 32);
#pragma unroll
  for (int i = 0; i < kPairs; ++i) *reinterpret_cast<uint32_t*>(y + 2 * i) = pack(o[i].x * inv, o[i].y * inv, (T*)nullptr);
}

}  // namespace prompt
}  // namespace aqd
