// lm_distill.cu -- distillation from a teacher's top logits: the loss of each token, its normalizer, and the gradient.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/aqd.h"
#include "kernels.h"

namespace aqd {
namespace distill {

constexpr int kThreads = 256;
constexpr int kMaxTop = 1024;

__device__ __forceinline__ float load_f32(const float* p) { return *p; }
__device__ __forceinline__ float load_f32(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ float load_f32(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_f32(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f32(__half* p, float v) { *p = __float2half_rn(v); }
__device__ __forceinline__ void store_f32(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// The running maximum m and sum s = sum exp(z - m) of a softmax; an empty share is (-inf, 0).
struct Soft {
  float m, s;
};
__device__ __forceinline__ Soft join(Soft a, Soft b) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) return {m, a.s + b.s};  // nothing yet (or NaN sums, which stay)
  return {m, a.s * expf(a.m - m) + b.s * expf(b.m - m)};
}
__device__ __forceinline__ Soft add(Soft a, float z) {
  if (z <= a.m) { a.s += z == -INFINITY ? 0.0f : expf(z - a.m); return a; }
  // a new maximum (or a NaN, which the sum keeps)
  return {z > a.m ? z : a.m, (a.m == -INFINITY ? a.s : a.s * expf(a.m - z)) + (z > a.m ? (z < INFINITY ? 1.0f : NAN) : z)};
}
__device__ __forceinline__ Soft shfl_join(Soft v) {
  for (int o = 16; o > 0; o >>= 1)
    v = join(v, Soft{__shfl_xor_sync(0xffffffffu, v.m, o), __shfl_xor_sync(0xffffffffu, v.s, o)});
  return v;
}
__device__ Soft block_join(Soft v, Soft* sh) {
  v = shfl_join(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  v = sh[0];
  for (int w = 1; w < kThreads / 32; ++w) v = join(v, sh[w]);
  return v;
}
__device__ float block_sum(float v, float* sh) {
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0.0f;
  for (int w = 0; w < kThreads / 32; ++w) v += sh[w];
  return v;
}

// One block per token.
template <class T>
__global__ void __launch_bounds__(kThreads) distill_kernel(const DistillArgs p) {
  __shared__ int sidx[kMaxTop];
  __shared__ float sp[kMaxTop], slz[kMaxTop];
  __shared__ Soft ssoft[kThreads / 32];
  __shared__ float ssum[kThreads / 32];
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(p.logits) + row * p.ld_logits;
  T* g = p.grad ? static_cast<T*>(p.grad) + row * p.ld_grad : nullptr;
  const float rt = 1.0f / p.tau;
  const float w = p.row_weight ? p.row_weight[row] : 1.0f;
  // the kept places; an empty one has index -1
  Soft t{-INFINITY, 0.0f};
  for (int j = threadIdx.x; j < p.top; j += kThreads) {
    const int64_t i = p.index[row * p.top + j];
    const float z = p.teacher[row * p.top + j] * rt;
    const bool in = i >= 0 && i < p.vocab && z != -INFINITY;
    sidx[j] = in ? (int)i : -1;
    sp[j] = z;
    slz[j] = in ? load_f32(x + i) * rt : 0.0f;
    if (in) t = add(t, z);
  }
  t = block_join(t, ssoft);
  const bool live = w != 0.0f && (t.m != -INFINITY || t.s != 0.0f);
  float lse = 0.0f;
  if (p.lse_in) lse = p.lse_in[row];
  else if (live || p.lse) {
    Soft s{-INFINITY, 0.0f};
    for (int v = threadIdx.x; v < p.vocab; v += kThreads) s = add(s, load_f32(x + v) * rt);
    s = block_join(s, ssoft);
    lse = s.m == -INFINITY && s.s == 0.0f ? -INFINITY : s.m + logf(s.s);
    if (p.lse && threadIdx.x == 0) p.lse[row] = lse;
  }
  if (!live) {  // the gradient after the last read of the logits, which it may replace
    if (p.loss && threadIdx.x == 0) p.loss[row] = 0.0f;
    if (g)
      for (int v = threadIdx.x; v < p.vocab; v += kThreads) store_f32(g + v, 0.0f);
    return;
  }
  const float lt = t.m + logf(t.s);
  float loss = 0.0f;
  for (int j = threadIdx.x; j < p.top; j += kThreads) {
    const float lp = sp[j] - lt, pj = sidx[j] >= 0 ? expf(lp) : 0.0f;
    if (pj != 0.0f) loss += pj * (lp - (slz[j] - lse));
    sp[j] = pj;
  }
  loss = block_sum(loss, ssum);
  if (p.loss && threadIdx.x == 0) p.loss[row] = w * loss;
  if (!g) return;
  const float f = w * rt;
  for (int v = threadIdx.x; v < p.vocab; v += kThreads) store_f32(g + v, f * expf(load_f32(x + v) * rt - lse));
  __syncthreads();
  for (int j = threadIdx.x; j < p.top; j += kThreads) {
    const int i = sidx[j];
    if (i < 0) continue;
    float pj = 0.0f;
    for (int l = 0; l < p.top; ++l) pj += sidx[l] == i ? sp[l] : 0.0f;
    store_f32(g + i, f * (expf(slz[j] - lse) - pj));
  }
}

}  // namespace distill

int launch_distill(const DistillArgs& a, cudaStream_t stream, std::string* err) {
  const unsigned grid = (unsigned)a.tokens;
  if (a.dtype == AQD_F32) distill::distill_kernel<float><<<grid, distill::kThreads, 0, stream>>>(a);
  else if (a.dtype == AQD_F16) distill::distill_kernel<__half><<<grid, distill::kThreads, 0, stream>>>(a);
  else distill::distill_kernel<__nv_bfloat16><<<grid, distill::kThreads, 0, stream>>>(a);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) { *err = std::string("distillation launch: ") + cudaGetErrorString(e); return AQD_ERR_CUDA; }
  return 0;
}

}  // namespace aqd
