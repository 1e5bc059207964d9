// lm_rows.cu -- rows of activations to 8-bit codes with one scale per row: a plain matrix, the root-mean-square norm
// with the residual's addition, and the gated activation between a feed-forward's products.
//
// With a = max_k |u_k| a row's codes are rne(u_k * 127 / a) and its scale a / 127. Under the norm,
// u_k = h_k w_k / rms(h): the factor 1 / rms cancels in the codes, so they need only max_k |h_k w_k|, which the same pass
// over the row gives as sum h^2; the scale takes the factor.
//
// All three are bound by memory. rows_kernel keeps a row in registers between its statistics and its codes, so it is
// read once: a warp per short row, a block per longer one, 16-byte accesses where all tensors allow them. Rows
// longer than a block's registers hold (16,384 values) take rows_long_kernel, which reads them twice (the second time from L2).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "../../include/aqd.h"
#include "kernels.h"

namespace aqd {
namespace rows {

constexpr float kTiny = 7.52316385e-37f;  // 2^-120: 127 / a stays finite above it
constexpr float kRound = 12582912.0f;     // 1.5 * 2^23: x + kRound has x rounded to nearest even in its low bits, for |x| < 2^22

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void store_any(void* p, int64_t i, int dtype, float v) {
  if (dtype == AQD_F32) static_cast<float*>(p)[i] = v;
  else if (dtype == AQD_F16) static_cast<__half*>(p)[i] = __float2half_rn(v);
  else static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
}

// kE adjacent values as float32 and back: one access of kE * sizeof(T) bytes (16; 32 in two; or a single value).
template <class T>
__device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b);
template <>
__device__ __forceinline__ void unpack2<__half>(uint32_t w, float& a, float& b) {
  const float2 f = __half22float2(*reinterpret_cast<__half2*>(&w));
  a = f.x; b = f.y;
}
template <>
__device__ __forceinline__ void unpack2<__nv_bfloat16>(uint32_t w, float& a, float& b) {
  a = __uint_as_float(w << 16); b = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __half*) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat16*) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <int kE, class T>
__device__ __forceinline__ void load_vec(const T* p, float (&f)[kE]) {
  if constexpr (kE == 1) f[0] = to_f32(*p);
  else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < kE; i += 4) {
      const float4 v = *reinterpret_cast<const float4*>(p + i);
      f[i] = v.x; f[i + 1] = v.y; f[i + 2] = v.z; f[i + 3] = v.w;
    }
  } else if constexpr (kE == 8) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    unpack2<T>(v.x, f[0], f[1]); unpack2<T>(v.y, f[2], f[3]); unpack2<T>(v.z, f[4], f[5]); unpack2<T>(v.w, f[6], f[7]);
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    unpack2<T>(v.x, f[0], f[1]); unpack2<T>(v.y, f[2], f[3]);
  }
}
template <int kE, class T>
__device__ __forceinline__ void store_vec(T* p, const float (&f)[kE]) {
  if constexpr (kE == 1) store_any(p, 0, sizeof(T) == 4 ? AQD_F32 : (std::is_same<T, __half>::value ? AQD_F16 : AQD_BF16), f[0]);
  else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < kE; i += 4) *reinterpret_cast<float4*>(p + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
  } else if constexpr (kE == 8) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack2(f[0], f[1], p), pack2(f[2], f[3], p), pack2(f[4], f[5], p), pack2(f[6], f[7], p));
  } else {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack2(f[0], f[1], p), pack2(f[2], f[3], p));
  }
}
template <int kE>
__device__ __forceinline__ void load_vec_any(const void* p, int64_t i, int dtype, float (&f)[kE]) {
  if (dtype == AQD_F32) load_vec<kE>(static_cast<const float*>(p) + i, f);
  else if (dtype == AQD_F16) load_vec<kE>(static_cast<const __half*>(p) + i, f);
  else load_vec<kE>(static_cast<const __nv_bfloat16*>(p) + i, f);
}
template <int kE>
__device__ __forceinline__ void store_vec_any(void* p, int64_t i, int dtype, const float (&f)[kE]) {
  if (dtype == AQD_F32) store_vec<kE>(static_cast<float*>(p) + i, f);
  else if (dtype == AQD_F16) store_vec<kE>(static_cast<__half*>(p) + i, f);
  else store_vec<kE>(static_cast<__nv_bfloat16*>(p) + i, f);
}

// Both activations are g times a logistic function: (1 + tanh z) / 2 = 1 / (1 + e^-2z), which loses nothing for z << 0 as 1 + tanh z
// does. e^x and the quotient by the fast hardware functions: within 2^-21 of their size for |x| <= 8, far inside half a code's step.
__device__ __forceinline__ float activate(float g, int act) {
  const float z = act == AQD_ACT_SILU ? g : 1.5957691216f * fmaf(0.044715f * g * g, g, g);  // 2 sqrt(2 / pi)
  return __fdividef(g, 1.0f + __expf(-z));
}

// A row's codes: u * inv rounded; its scale. (rms: of the row, under the norm, else 1 / rms is 1)
__device__ __forceinline__ void row_scale(float a, float ss, float rrms, float& inv, float& scale) {
  inv = 0.0f;
  scale = 0.0f;
  if (!(a < INFINITY) || !(ss < INFINITY)) scale = NAN;
  else if (a >= kTiny) {
    inv = 127.0f / a;
    scale = a / 127.0f * rrms;
  }
}

// The codes and values of kE adjacent u (which they replace).
template <int kE>
__device__ __forceinline__ void write_codes(const RowArgs& p, int64_t row, int64_t k, float inv, float scale, float (&u)[kE]) {
  uint32_t q[kE];
#pragma unroll
  for (int j = 0; j < kE; ++j) {
    const float t = inv == 0.0f ? kRound : fmaf(u[j], inv, kRound);
    q[j] = __float_as_uint(t);
    u[j] = (t - kRound) * scale;
  }
  if (p.codes) {
    int8_t* c = p.codes + row * p.ld_codes + k;
    if constexpr (kE == 1) *c = (int8_t)q[0];
    else {
      uint32_t w[kE / 4];
#pragma unroll
      for (int j = 0; j < kE; j += 4) w[j / 4] = __byte_perm(__byte_perm(q[j], q[j + 1], 0x0040), __byte_perm(q[j + 2], q[j + 3], 0x0040), 0x5410);
      if constexpr (kE == 8) *reinterpret_cast<uint2*>(c) = make_uint2(w[0], w[1]);
      else *reinterpret_cast<uint32_t*>(c) = w[0];
    }
  }
  if (p.values) store_vec_any<kE>(p.values, row * p.ld_values + k, p.values_dtype, u);
}

// kWarpRow: a warp per row, else a block; kV vectors of kE elements a thread (32 values of 32 bits take a block of at most 512).
template <class T, RowOp kOp, int kE, int kV, bool kWarpRow>
__global__ void __launch_bounds__(kWarpRow ? 256 : (kV * kE >= 32 ? 512 : 1024)) rows_kernel(const RowArgs p) {
  __shared__ float ssum[32];
  __shared__ uint32_t smax[32];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t row = kWarpRow ? (int64_t)blockIdx.x * (blockDim.x >> 5) + warp : (int64_t)blockIdx.x;
  if (kWarpRow && row >= p.rows) return;
  const int first = (kWarpRow ? lane : (int)threadIdx.x) * kE, step = (kWarpRow ? 32 : (int)blockDim.x) * kE;
  const T* a = static_cast<const T*>(p.a) + row * p.lda;
  const T* b = static_cast<const T*>(p.b) + row * p.ldb;
  float u[kV][kE];
  float ss = 0.0f;
  uint32_t top = 0;  // |u| as its bits: they order as the magnitudes do, a NaN above all
  if constexpr (kOp == kRowPlain) {
#pragma unroll
    for (int i = 0; i < kV; ++i)
      if (first + i * step < p.cols) load_vec<kE>(a + first + i * step, u[i]);
  } else {
    float v[kV][kE];
#pragma unroll
    for (int i = 0; i < kV; ++i)
      if (first + i * step < p.cols) {
        load_vec<kE>(a + first + i * step, u[i]);
        if (kOp == kRowGated || p.b) load_vec<kE>(b + first + i * step, v[i]);
      }
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const int k = first + i * step;
      if (k >= p.cols) break;
      if constexpr (kOp == kRowNorm) {
        if (p.b) {
#pragma unroll
          for (int j = 0; j < kE; ++j) u[i][j] += v[i][j];
        }
        if (p.sum) store_vec<kE>(static_cast<T*>(p.sum) + row * p.ld_sum + k, u[i]);
        float w[kE];
        load_vec_any<kE>(p.weight, k, p.weight_dtype, w);
#pragma unroll
        for (int j = 0; j < kE; ++j) {
          ss = fmaf(u[i][j], u[i][j], ss);
          u[i][j] *= w[j];
        }
      } else {
#pragma unroll
        for (int j = 0; j < kE; ++j) u[i][j] = activate(u[i][j], p.act) * v[i][j];
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    if (first + i * step >= p.cols) break;
#pragma unroll
    for (int j = 0; j < kE; ++j) top = max(top, __float_as_uint(fabsf(u[i][j])));
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if (kOp == kRowNorm)
    for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  if constexpr (!kWarpRow) {
    if (lane == 0) { ssum[warp] = ss; smax[warp] = top; }
    __syncthreads();
    const int warps = blockDim.x >> 5;
    top = __reduce_max_sync(0xffffffffu, lane < warps ? smax[lane] : 0u);
    if (kOp == kRowNorm) {
      ss = lane < warps ? ssum[lane] : 0.0f;
      for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    }
  }
  float inv, scale;
  row_scale(__uint_as_float(top), ss, kOp == kRowNorm ? rsqrtf(ss / (float)p.cols + p.eps) : 1.0f, inv, scale);
  if (first == 0) p.scales[row] = scale;
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const int k = first + i * step;
    if (k >= p.cols) break;
    write_codes<kE>(p, row, k, inv, scale, u[i]);
  }
}

// kE values u_k of the row (under the norm without the factor 1 / rms), and h_k.
template <class T, RowOp kOp, int kE>
__device__ __forceinline__ void units(const RowArgs& p, int64_t row, int64_t k, float (&u)[kE], float (&h)[kE]) {
  load_vec<kE>(static_cast<const T*>(p.a) + row * p.lda + k, u);
  if constexpr (kOp != kRowPlain) {
    float v[kE];
    if (kOp == kRowGated || p.b) load_vec<kE>(static_cast<const T*>(p.b) + row * p.ldb + k, v);
    if constexpr (kOp == kRowNorm) {
      if (p.b) {
#pragma unroll
        for (int j = 0; j < kE; ++j) u[j] += v[j];
      }
      load_vec_any<kE>(p.weight, k, p.weight_dtype, v);
#pragma unroll
      for (int j = 0; j < kE; ++j) { h[j] = u[j]; u[j] *= v[j]; }
    } else {
#pragma unroll
      for (int j = 0; j < kE; ++j) u[j] = activate(u[j], p.act) * v[j];
    }
  }
}

// One block per row of any length: a pass for the statistics, a pass for the codes. (The sum, which may replace an input,
// is written in the second pass, by the thread that reads the inputs there.)
template <class T, RowOp kOp, int kE>
__global__ void __launch_bounds__(512) rows_long_kernel(const RowArgs p) {
  __shared__ float ssum[16];
  __shared__ uint32_t smax[16];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int64_t row = blockIdx.x;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float ss = 0.0f, u[kE], h[kE];
  uint32_t top = 0;
  for (int64_t k = (int64_t)threadIdx.x * kE; k < p.cols; k += 512 * kE) {
    units<T, kOp, kE>(p, row, k, u, h);
#pragma unroll
    for (int j = 0; j < kE; ++j) {
      if (kOp == kRowNorm) ss = fmaf(h[j], h[j], ss);
      top = max(top, __float_as_uint(fabsf(u[j])));
    }
  }
  top = __reduce_max_sync(0xffffffffu, top);
  for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  if (lane == 0) { ssum[warp] = ss; smax[warp] = top; }
  __syncthreads();
  top = __reduce_max_sync(0xffffffffu, smax[lane & 15]);
  ss = lane < 16 ? ssum[lane] : 0.0f;
  for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
  float inv, scale;
  row_scale(__uint_as_float(top), ss, kOp == kRowNorm ? rsqrtf(ss / (float)p.cols + p.eps) : 1.0f, inv, scale);
  if (threadIdx.x == 0) p.scales[row] = scale;
  for (int64_t k = (int64_t)threadIdx.x * kE; k < p.cols; k += 512 * kE) {
    units<T, kOp, kE>(p, row, k, u, h);
    if (kOp == kRowNorm && p.sum) store_vec<kE>(static_cast<T*>(p.sum) + row * p.ld_sum + k, h);
    write_codes<kE>(p, row, k, inv, scale, u);
  }
}

static cudaError_t start(void (*kernel)(RowArgs), unsigned grid, unsigned threads, const RowArgs& a, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

static bool whole(const void* p, int64_t ld, int size, int bytes) {
  return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0 && (ld * size) % bytes == 0);
}
static int size_of(int dtype) { return dtype == AQD_F32 ? 4 : 2; }

template <class T, RowOp kOp>
static cudaError_t run(const RowArgs& a, cudaStream_t stream) {
  constexpr int kE = 16 / sizeof(T);
  const int ts = (int)sizeof(T), vs = size_of(a.values_dtype), wbytes = kE * size_of(a.weight_dtype) > 16 ? 16 : kE * size_of(a.weight_dtype);
  const bool vec = a.cols % kE == 0 && whole(a.a, a.lda, ts, 16) && whole(a.b, a.ldb, ts, 16) && whole(a.sum, a.ld_sum, ts, 16) &&
                   whole(a.codes, a.ld_codes, 1, kE) && whole(a.values, a.ld_values, vs, kE * vs > 16 ? 16 : kE * vs) &&
                   whole(a.weight, 0, 1, wbytes);
  const unsigned rows = (unsigned)a.rows;
  auto block = [](int64_t n, int v) { return (unsigned)(((n + v - 1) / v + 31) / 32 * 32); };  // threads for n units, v each
  if (vec) {
    const int64_t n = a.cols / kE;
    // A warp with up to 4 vectors a lane, where the rows fill the GPU that way; a block with one vector a thread for few rows (the
    // shortest chain), with up to 4 for many (fewer warps to wait at each row's end).
    if (n <= 32) return start(rows_kernel<T, kOp, kE, 1, true>, (rows + 7) / 8, 256, a, stream);
    if (n <= 128 && rows > 608) return start(rows_kernel<T, kOp, kE, 4, true>, (rows + 7) / 8, 256, a, stream);
    if (n <= 1024 && rows <= 304) return start(rows_kernel<T, kOp, kE, 1, false>, rows, block(n, 1), a, stream);
    constexpr int kV = 32 / kE;
    if (n <= 512 * kV) return start(rows_kernel<T, kOp, kE, kV, false>, rows, block(n, kV), a, stream);
    return start(rows_long_kernel<T, kOp, kE>, rows, 512, a, stream);
  }
  if (a.cols <= 256 && rows > 608) return start(rows_kernel<T, kOp, 1, 8, true>, (rows + 7) / 8, 256, a, stream);
  if (a.cols <= 8192) return start(rows_kernel<T, kOp, 1, 8, false>, rows, block(a.cols, 8), a, stream);
  if (a.cols <= 16384) return start(rows_kernel<T, kOp, 1, 32, false>, rows, block(a.cols, 32), a, stream);
  return start(rows_long_kernel<T, kOp, 1>, rows, 512, a, stream);
}
template <class T>
static cudaError_t run_op(RowOp op, const RowArgs& a, cudaStream_t stream) {
  if (op == kRowPlain) return run<T, kRowPlain>(a, stream);
  if (op == kRowNorm) return run<T, kRowNorm>(a, stream);
  return run<T, kRowGated>(a, stream);
}

}  // namespace rows

int launch_rows(RowOp op, const RowArgs& a, cudaStream_t stream, std::string* err) {
  cudaError_t e = a.dtype == AQD_F32   ? rows::run_op<float>(op, a, stream)
                  : a.dtype == AQD_F16 ? rows::run_op<__half>(op, a, stream)
                                       : rows::run_op<__nv_bfloat16>(op, a, stream);
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) { *err = std::string("row quantizer launch: ") + cudaGetErrorString(e); return AQD_ERR_CUDA; }
  return 0;
}

}  // namespace aqd
