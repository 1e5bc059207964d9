// lm_linear.cu -- product of int8 codes with a scale per token and per output channel: weight layout and the
// CUDA-core kernel, which takes any shape, stride and alignment.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/aqd.h"
#include "kernels.h"

namespace aqd {
namespace lin {

// Rows of k codes plus 128, as bytes (what the conversion to F16 starts from), padded with code 0 to whole chunks of
// 128; and the header's first word, the most chunks in a row that any row of weights lets an FP32 accumulator sum exactly:
// those of every window of that length have sum |w| * 128 <= 2^24. (8 chunks always do.) One warp per row.
__global__ void __launch_bounds__(128) prepare_kernel(const int8_t* __restrict__ codes, int64_t ld, int32_t n, int32_t k,
                                                      int64_t pitch, uint8_t* __restrict__ out) {
  __shared__ uint16_t sums[4][1024];  // sum |w| of each chunk (at most 128 * 128)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int chunks = (int)(pitch / 128);
  int most = chunks;
  for (int64_t row = (int64_t)blockIdx.x * 4 + warp; row < n; row += (int64_t)gridDim.x * 4) {
    for (int c = 0; c < chunks; ++c) {
      uint32_t word = 0;
      int s = 0;
      for (int j = 0; j < 4; ++j) {
        const int i = c * 128 + lane * 4 + j;
        const int w = i < k ? codes[row * ld + i] : 0;
        s += w < 0 ? -w : w;
        word |= (uint32_t)(uint8_t)(w + 128) << (8 * j);
      }
      *reinterpret_cast<uint32_t*>(out + kLinHeader + row * pitch + c * 128 + lane * 4) = word;
      s = __reduce_add_sync(0xffffffffu, s);
      if (lane == 0) sums[warp][c] = (uint16_t)s;
    }
    __syncwarp();
    if (lane == 0) {  // windows (lo, hi]: each hi's longest with a sum in range; the shortest of those that could not grow
      int lo = 0, sum = 0;
      for (int hi = 0; hi < chunks; ++hi) {
        sum += sums[warp][hi];
        while (sum > 131072) {
          sum -= sums[warp][lo++];
          const int len = hi - lo + 1;
          if (len < most) most = len;
        }
      }
    }
    __syncwarp();
  }
  if (lane == 0) atomicMin(reinterpret_cast<int*>(out), most);
}

__device__ __forceinline__ void store_y(const LinArgs& p, int64_t m, int n, int acc) {
  const int64_t i = m * p.ldy + n;
  if (p.y_dtype == AQD_I32) { static_cast<int32_t*>(p.y)[i] = acc; return; }
  float v = __fmul_rn(__fmul_rn(__int2float_rn(acc), p.x_scale[m]), p.w_scale[n]);
  if (p.bias) v = __fadd_rn(v, p.bias[n]);
  if (p.y_dtype == AQD_F32) static_cast<float*>(p.y)[i] = v;
  else if (p.y_dtype == AQD_F16) static_cast<__half*>(p.y)[i] = __float2half_rn(v);
  else static_cast<__nv_bfloat16*>(p.y)[i] = __float2bfloat16_rn(v);
}

constexpr int kTM = 32, kTN = 64, kTK = 64;

// 32 tokens x 64 channels per block of 256 threads, 8 outputs a thread, four products per __dp4a.
__global__ void __launch_bounds__(256) linear_direct_kernel(const LinArgs p) {
  __shared__ int sx[kTM][kTK / 4 + 1], sw[kTN][kTK / 4 + 1];
  const int64_t pitch = ((int64_t)p.k + 127) / 128 * 128;
  const int64_t m0 = (int64_t)blockIdx.y * kTM;
  const int n0 = blockIdx.x * kTN;
  const int tn = threadIdx.x & 31, tm = threadIdx.x >> 5;
  int acc[4][2] = {};
  for (int k0 = 0; k0 < p.k; k0 += kTK) {
    for (int i = threadIdx.x; i < kTM * kTK / 4; i += 256) {
      const int r = i / (kTK / 4), c = i % (kTK / 4), k = k0 + 4 * c;
      uint32_t v = 0;
      if (m0 + r < p.m)
        for (int j = 0; j < 4; ++j)
          if (k + j < p.k) v |= (uint32_t)(uint8_t)p.x[(m0 + r) * p.ldx + k + j] << (8 * j);
      sx[r][c] = (int)v;
    }
    for (int i = threadIdx.x; i < kTN * kTK / 4; i += 256) {
      const int r = i / (kTK / 4), c = i % (kTK / 4);
      sw[r][c] = n0 + r < p.n ? (int)(*reinterpret_cast<const uint32_t*>(p.w + kLinHeader + (n0 + r) * pitch + k0 + 4 * c) ^ 0x80808080u) : 0;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < kTK / 4; ++c) {
      const int w0 = sw[tn][c], w1 = sw[tn + 32][c];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int x = sx[tm * 4 + i][c];
        acc[i][0] = __dp4a(x, w0, acc[i][0]);
        acc[i][1] = __dp4a(x, w1, acc[i][1]);
      }
    }
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 2; ++j) {
      const int64_t m = m0 + tm * 4 + i;
      const int n = n0 + tn + 32 * j;
      if (m < p.m && n < p.n) store_y(p, m, n, acc[i][j]);
    }
}

}  // namespace lin

static int launched(const char* what, std::string* err) {
  const cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) return 0;
  *err = std::string(what) + cudaGetErrorString(e);
  return AQD_ERR_CUDA;
}

int launch_linear_prepare(const int8_t* codes, int64_t ld, int32_t n, int32_t k, uint8_t* out, cudaStream_t stream,
                          std::string* err) {
  const cudaError_t e = cudaMemsetAsync(out, 0x7f, 4, stream);
  if (e != cudaSuccess) { *err = std::string("weight preparation: ") + cudaGetErrorString(e); return AQD_ERR_CUDA; }
  lin::prepare_kernel<<<n < 4864 ? (n + 3) / 4 : 1216, 128, 0, stream>>>(codes, ld, n, k, lin_pitch(k), out);
  return launched("weight preparation launch: ", err);
}

size_t linear_workspace_bytes(int64_t m, int32_t n, int32_t k) { return linear_tc_workspace_bytes(m, n); }

int launch_linear(const LinArgs& a, cudaStream_t stream, std::string* err) {
  if (a.m > 8 && linear_tc_takes(a)) return launch_linear_tc(a, stream, err);
  // rows of blocks in pieces of the grid's second dimension
  constexpr int64_t kRows = 65535LL * lin::kTM;
  const size_t es = a.y_dtype == AQD_F32 || a.y_dtype == AQD_I32 ? 4 : 2;
  for (int64_t m = 0; m < a.m; m += kRows) {
    LinArgs p = a;
    p.m = a.m - m < kRows ? a.m - m : kRows;
    p.x += m * a.ldx;
    if (p.x_scale) p.x_scale += m;
    p.y = static_cast<uint8_t*>(p.y) + (size_t)m * a.ldy * es;
    const dim3 grid((unsigned)((p.n + lin::kTN - 1) / lin::kTN), (unsigned)((p.m + lin::kTM - 1) / lin::kTM));
    lin::linear_direct_kernel<<<grid, 256, 0, stream>>>(p);
    if (const int st = launched("8-bit product launch: ", err)) return st;
  }
  return 0;
}

}  // namespace aqd
