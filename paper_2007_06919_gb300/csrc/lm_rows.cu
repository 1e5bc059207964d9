// lm_rows.cu -- rows of activations to 8-bit codes with one scale per row: a plain matrix, the root-mean-square norm
// with the residual's addition, and the gated activation between a feed-forward's products.
//
// With a = max_k |u_k| a row's codes are rne(u_k * 127 / a) and its scale a / 127. Under the norm,
// u_k = h_k w_k / rms(h): the factor 1 / rms cancels in the codes, so they need only max_k |h_k w_k|, which the same pass
// over the row gives as sum h^2; the scale takes the factor.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/aqd.h"
#include "kernels.h"

namespace aqd {
namespace rows {

constexpr float kTiny = 7.52316385e-37f;  // 2^-120: 127 / a stays finite above it

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float load_any(const void* p, int64_t i, int dtype) {
  if (dtype == AQD_F32) return static_cast<const float*>(p)[i];
  if (dtype == AQD_F16) return __half2float(static_cast<const __half*>(p)[i]);
  return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
__device__ __forceinline__ void store_any(void* p, int64_t i, int dtype, float v) {
  if (dtype == AQD_F32) static_cast<float*>(p)[i] = v;
  else if (dtype == AQD_F16) static_cast<__half*>(p)[i] = __float2half_rn(v);
  else static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
}

__device__ __forceinline__ float activate(float g, int act) {
  if (act == AQD_ACT_SILU) return g / (1.0f + expf(-g));
  return 0.5f * g * (1.0f + tanhf(0.7978845608f * (g + 0.044715f * g * g * g)));
}

// u_k of the row (under the norm without the factor 1 / rms), and h_k.
template <RowOp kOp>
__device__ __forceinline__ float unit(const RowArgs& p, int64_t row, int k, float* h) {
  float u = load_any(p.a, row * p.lda + k, p.dtype);
  if constexpr (kOp == kRowNorm) {
    if (p.b) u += load_any(p.b, row * p.ldb + k, p.dtype);
    *h = u;
    u *= load_any(p.weight, k, p.weight_dtype);
  }
  if constexpr (kOp == kRowGated) u = activate(u, p.act) * load_any(p.b, row * p.ldb + k, p.dtype);
  return u;
}

// One block per row: a pass for the statistics, a pass for the codes.
template <RowOp kOp>
__global__ void __launch_bounds__(256) rows_kernel(const RowArgs p) {
  __shared__ float ssum[8];
  __shared__ uint32_t smax[8];
  const int64_t row = blockIdx.x;
  float ss = 0.0f, h = 0.0f;
  uint32_t top = 0;  // |u| as its bits: they order as the magnitudes do, a NaN above all
  for (int k = threadIdx.x; k < p.cols; k += 256) {
    const float u = unit<kOp>(p, row, k, &h);
    if (kOp == kRowNorm) ss = fmaf(h, h, ss);
    top = max(top, __float_as_uint(fabsf(u)));
  }
  for (int o = 16; o > 0; o >>= 1) {
    ss += __shfl_xor_sync(0xffffffffu, ss, o);
    top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
  }
  if ((threadIdx.x & 31) == 0) { ssum[threadIdx.x >> 5] = ss; smax[threadIdx.x >> 5] = top; }
  __syncthreads();
  ss = 0.0f; top = 0;
  for (int w = 0; w < 8; ++w) { ss += ssum[w]; top = max(top, smax[w]); }
  const float a = __uint_as_float(top);
  float inv = 0.0f, scale = 0.0f;
  if (!(a < INFINITY) || !(ss < INFINITY)) scale = NAN;
  else if (a >= kTiny) {
    inv = 127.0f / a;
    scale = a / 127.0f;
    if (kOp == kRowNorm) scale *= rsqrtf(ss / (float)p.cols + p.eps);
  }
  if (threadIdx.x == 0) p.scales[row] = scale;
  for (int k = threadIdx.x; k < p.cols; k += 256) {
    const float u = unit<kOp>(p, row, k, &h);
    const float c = inv == 0.0f ? 0.0f : rintf(u * inv);
    if (kOp == kRowNorm && p.sum) store_any(p.sum, row * p.ld_sum + k, p.dtype, h);
    if (p.codes) p.codes[row * p.ld_codes + k] = (int8_t)c;
    if (p.values) store_any(p.values, row * p.ld_values + k, p.values_dtype, c * scale);
  }
}

}  // namespace rows

int launch_rows(RowOp op, const RowArgs& a, cudaStream_t stream, std::string* err) {
  const unsigned grid = (unsigned)a.rows;
  if (op == kRowPlain) rows::rows_kernel<kRowPlain><<<grid, 256, 0, stream>>>(a);
  else if (op == kRowNorm) rows::rows_kernel<kRowNorm><<<grid, 256, 0, stream>>>(a);
  else rows::rows_kernel<kRowGated><<<grid, 256, 0, stream>>>(a);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) { *err = std::string("row quantizer launch: ") + cudaGetErrorString(e); return AQD_ERR_CUDA; }
  return 0;
}

}  // namespace aqd
