// lm_rows.cu -- rows of activations to 8-bit codes with one scale per row: a plain matrix, the root-mean-square norm
// with the residual's addition, and the gated activation between a feed-forward's products.
//
// With a = max_k |u_k| a row's codes are rne(u_k * 127 / a) and its scale a / 127. Under the norm,
// u_k = h_k w_k / rms(h): the factor 1 / rms cancels in the codes, so they need only max_k |h_k w_k|, which the same pass
// over the row gives as sum h^2; the scale takes the factor.
//
// All three are bound by memory, and a row's codes need all of it: it waits on chip in between, so it is read once. Short rows
// wait in registers (rows_kernel: a warp or a block each), longer ones in shared memory (rows_held_kernel), of a block or of a cluster's
// blocks, and rows longer than that are read twice, the second time from L2 (rows_long_kernel). 16-byte accesses where the
// tensors lie so that these are possible.
// (4096 x 4096 bf16, the norm with its residual, codes and values: 26 us, 5.8 TB/s; 4096 x 12288 f16, gated: 56 us, 6.2 TB/s.)
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "../../include/aqd.h"
#include "common.cuh"
#include "kernels.h"
#include "tc_ptx.cuh"

namespace aqd {
namespace rows {

constexpr float kTiny = 7.52316385e-37f;  // 2^-120: 127 / a stays finite above it
constexpr float kMinNormal = 1.17549435e-38f;  // 2^-126
constexpr int kHeldBytes = 72 * 1024;  // shared memory of a held row: three blocks share an SM
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

// Vectors of rows that start `off` elements into one: vector v holds the row's elements from v kE - off on, whole ones inside the row
// (for kShift false always), the first and last of them cut by its ends.
template <int kE, bool kShift>
__device__ __forceinline__ bool inside(int64_t k, int64_t cols) { return !kShift || (k >= 0 && k + kE <= cols); }
template <int kE, class T>
__device__ __forceinline__ void load_each(const T* p, int64_t k, int64_t cols, float (&f)[kE]) {
#pragma unroll
  for (int j = 0; j < kE; ++j) f[j] = k + j >= 0 && k + j < cols ? to_f32(p[k + j]) : 0.0f;
}
// the vector at p, element k of the row
template <int kE, bool kShift, class T>
__device__ __forceinline__ void load_at(const T* p, int k, int cols, float (&f)[kE]) {
  if (inside<kE, kShift>(k, cols)) load_vec<kE>(p, f);
  else load_each<kE>(p - k, k, cols, f);
}
// kE values from shared memory, element `at` of a vector that starts on 16 bytes: out of the two aligned vectors that hold them, the words
// picked by the distance.
template <int kE, class T>
__device__ __forceinline__ void load_across(const T* from, int at, float (&f)[kE]) {
  static_assert(kE * sizeof(T) == 16, "");
  const int s = at % kE, q = s * (int)sizeof(T) / 4;  // elements, and words, into the first
  const uint4* v = reinterpret_cast<const uint4*>(from) + at / kE;
  const uint4 lo = v[0], hi = v[s ? 1 : 0];
  uint32_t x[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
  for (int i = 0; i < 6; ++i) x[i] = q & 2 ? x[i + 2] : x[i];
#pragma unroll
  for (int i = 0; i < 5; ++i) x[i] = q & 1 ? x[i + 1] : x[i];
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(x[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) unpack2<T>(__funnelshift_r(x[i], x[i + 1], (s & 1) * 16), f[2 * i], f[2 * i + 1]);
  }
}
// the norm's weights, which do not start where a row does: element by element for kShift. (Out of two aligned vectors, the words picked
// by the distance: no faster, 4096 x 1001 bf16 12.3 us to 11.8.)
template <int kE, bool kShift>
__device__ __forceinline__ void load_weight(const RowArgs& p, int64_t k, float (&f)[kE]) {
  if constexpr (!kShift) load_vec_any<kE>(p.weight, k, p.weight_dtype, f);
  else if (p.weight_dtype == AQD_F32) load_each<kE>(static_cast<const float*>(p.weight), k, p.cols, f);
  else if (p.weight_dtype == AQD_F16) load_each<kE>(static_cast<const __half*>(p.weight), k, p.cols, f);
  else load_each<kE>(static_cast<const __nv_bfloat16*>(p.weight), k, p.cols, f);
}
template <int kE, bool kShift, class T>
__device__ __forceinline__ void store_sum(const RowArgs& p, int64_t row, int k, const float (&f)[kE]) {
  if (inside<kE, kShift>(k, p.cols)) store_vec<kE>(static_cast<T*>(p.sum) + row * p.ld_sum + k, f);
  else {
#pragma unroll
    for (int j = 0; j < kE; ++j)
      if (k + j >= 0 && k + j < p.cols) store_vec<1>(static_cast<T*>(p.sum) + row * p.ld_sum + k + j, reinterpret_cast<const float(&)[1]>(f[j]));
  }
}

// Both activations are g times a logistic function: (1 + tanh z) / 2 = 1 / (1 + e^-2z), which loses nothing for z << 0 as 1 + tanh z
// does. The exponential and the reciprocal are the fast hardware functions': together within 2^-21 of their size for |z| <= 8, far inside
// half a code's step. (1 + e^-z infinite gives 0.)
__device__ __forceinline__ float activate(float g, int act) {
  const float z = act == AQD_ACT_SILU ? g : 1.5957691216f * fmaf(0.044715f * g * g, g, g);  // 2 sqrt(2 / pi)
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-1.4426950409f * z));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return g * r;
}

__host__ __device__ constexpr bool is_norm(RowOp op) { return op == kRowNorm || op == kRowNormSmall; }

// The sum of a row's squares, under the norm. Squares are exact to 2^-150, so their mean plus eps is as good as float32's from 2^-126 on. Where
// eps is below that (0, mostly; kRowNormSmall) the mean of a row of small values may be too, and `low` has the squares of 2^100 h, in
// range for every row that small. (4096 x 4096 bf16 27.9 us, 25.7 without; 1000 x 32768 f32, over clusters of two blocks an SM instead of three, 111 and 94.
// The two sums in one kernel for every eps would spill there; the second one in a pass ahead, read in a rare branch of these kernels: 8192 x 1024 bf16
// 22.3 us for every eps, 13.4 now.)
template <RowOp kOp>
struct Squares {
  float sum = 0.0f, low = 0.0f;
  __device__ __forceinline__ void add(float h) {
    if constexpr (is_norm(kOp)) sum = fmaf(h, h, sum);
    if constexpr (kOp == kRowNormSmall) low = fmaf(h * 0x1p100f, h * 0x1p100f, low);
  }
  __device__ __forceinline__ void join(const Squares& o) {
    if constexpr (is_norm(kOp)) sum += o.sum;
    if constexpr (kOp == kRowNormSmall) low += o.low;
  }
  __device__ __forceinline__ void join_lanes() {
    if constexpr (is_norm(kOp))
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if constexpr (kOp == kRowNormSmall)
      for (int o = 16; o > 0; o >>= 1) low += __shfl_xor_sync(0xffffffffu, low, o);
  }
};

// A row's codes: u * inv rounded; its scale, under the norm with the factor 1 / rms.
template <RowOp kOp>
__device__ __forceinline__ void row_scale(const RowArgs& p, int cols, float a, const Squares<kOp>& s, float& inv, float& scale) {
  inv = 0.0f;
  scale = 0.0f;
  float rrms = 1.0f, up = 1.0f;
  if constexpr (is_norm(kOp)) rrms = rsqrtf(s.sum / (float)cols + p.eps);
  if constexpr (kOp == kRowNormSmall) {
    if (s.sum / (float)cols + p.eps < kMinNormal) {  // 2^100 / rms(2^100 h), the power in two parts that stay in range
      rrms = rsqrtf(s.low / (float)cols + p.eps * 0x1p100f * 0x1p100f) * 0x1p60f;
      up = 0x1p40f;
    }
  }
  if (!(a < INFINITY) || !(s.sum < INFINITY)) scale = NAN;
  else if (a >= kTiny) {
    inv = 127.0f / a;
    scale = a / 127.0f * rrms * up;
  }
}

// The codes and values of kE adjacent u (which they replace), all finite or inv and u 0.
template <int kE, bool kShift>
__device__ __forceinline__ void write_codes(const RowArgs& p, int64_t row, int64_t k, float inv, float scale, float (&u)[kE]) {
  uint32_t q[kE];
#pragma unroll
  for (int j = 0; j < kE; ++j) {
    const float t = fmaf(u[j], inv, kRound);
    q[j] = __float_as_uint(t);
    u[j] = (t - kRound) * scale;
  }
  if (!inside<kE, kShift>(k, p.cols)) {
#pragma unroll
    for (int j = 0; j < kE; ++j) {
      if (k + j < 0 || k + j >= p.cols) continue;
      if (p.codes) p.codes[row * p.ld_codes + k + j] = (int8_t)q[j];
      if (p.values) store_any(p.values, row * p.ld_values + k + j, p.values_dtype, u[j]);
    }
    return;
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

// Statistics of a block's threads, in a fixed order: lanes, then warps.
template <RowOp kOp>
__device__ __forceinline__ void block_stats(uint32_t& top, Squares<kOp>& ss) {
  __shared__ float ssum[32], slow[32];
  __shared__ uint32_t smax[32];
  const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  top = __reduce_max_sync(0xffffffffu, top);
  ss.join_lanes();
  if (lane == 0) {
    if constexpr (is_norm(kOp)) ssum[threadIdx.x >> 5] = ss.sum;
    if constexpr (kOp == kRowNormSmall) slow[threadIdx.x >> 5] = ss.low;
    smax[threadIdx.x >> 5] = top;
  }
  __syncthreads();
  top = __reduce_max_sync(0xffffffffu, lane < warps ? smax[lane] : 0u);
  if constexpr (is_norm(kOp)) ss.sum = lane < warps ? ssum[lane] : 0.0f;
  if constexpr (kOp == kRowNormSmall) ss.low = lane < warps ? slow[lane] : 0.0f;
  ss.join_lanes();
}

// kWarpRow: a warp per row, else a block; kV vectors of kE elements a thread (32 values of 32 bits take a block of at most 512).
// kShift: rows start inside a vector, at the same element of it in every tensor but the weights.
template <class T, RowOp kOp, int kE, int kV, bool kWarpRow, bool kShift>
__global__ void __launch_bounds__(kWarpRow ? 256 : (kV * kE >= 32 ? 512 : 1024)) rows_kernel(const RowArgs p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t row = kWarpRow ? (int64_t)blockIdx.x * (blockDim.x >> 5) + warp : (int64_t)blockIdx.x;
  if (kWarpRow && row >= p.rows) return;
  const T* a = static_cast<const T*>(p.a) + row * p.lda;
  const T* b = static_cast<const T*>(p.b) + row * p.ldb;
  const int thread = kWarpRow ? lane : (int)threadIdx.x, step = (kWarpRow ? 32 : (int)blockDim.x) * kE;
  const int first = thread * kE - (kShift ? (int)((reinterpret_cast<uintptr_t>(a) & 15) / sizeof(T)) : 0);
  float u[kV][kE];
  Squares<kOp> ss;
  uint32_t top = 0;  // |u| as its bits: they order as the magnitudes do, a NaN above all
  if constexpr (kOp == kRowPlain) {
#pragma unroll
    for (int i = 0; i < kV; ++i)
      if (first + i * step < p.cols) load_at<kE, kShift>(a + first + i * step, first + i * step, p.cols, u[i]);
  } else {
    float v[kV][kE];
#pragma unroll
    for (int i = 0; i < kV; ++i)
      if (first + i * step < p.cols) {
        load_at<kE, kShift>(a + first + i * step, first + i * step, p.cols, u[i]);
        if (kOp == kRowGated || p.b) load_at<kE, kShift>(b + first + i * step, first + i * step, p.cols, v[i]);
      }
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const int k = first + i * step;
      if (k >= p.cols) break;
      if constexpr (is_norm(kOp)) {
        if (p.b) {
#pragma unroll
          for (int j = 0; j < kE; ++j) u[i][j] += v[i][j];
        }
        if (p.sum) store_sum<kE, kShift, T>(p, row, k, u[i]);
        float w[kE];
        load_weight<kE, kShift>(p, k, w);
#pragma unroll
        for (int j = 0; j < kE; ++j) {
          ss.add(u[i][j]);
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
  if constexpr (kWarpRow) {
    top = __reduce_max_sync(0xffffffffu, top);
    ss.join_lanes();
  } else {
    block_stats(top, ss);
  }
  float inv, scale;
  row_scale(p, p.cols, __uint_as_float(top), ss, inv, scale);
  if ((kShift ? thread : first) == 0) p.scales[row] = scale;
  if (isnan(scale)) {
#pragma unroll
    for (int i = 0; i < kV; ++i)
#pragma unroll
      for (int j = 0; j < kE; ++j) u[i][j] = 0.0f;
  }
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const int k = first + i * step;
    if (k >= p.cols) break;
    write_codes<kE, kShift>(p, row, k, inv, scale, u[i]);
  }
}

// kE values u_k of the row (under the norm without the factor 1 / rms), and h_k.
template <class T, RowOp kOp, int kE>
__device__ __forceinline__ void units(const RowArgs& p, int64_t row, int64_t k, float (&u)[kE], float (&h)[kE]) {
  load_vec<kE>(static_cast<const T*>(p.a) + row * p.lda + k, u);
  if constexpr (kOp != kRowPlain) {
    float v[kE];
    if (kOp == kRowGated || p.b) load_vec<kE>(static_cast<const T*>(p.b) + row * p.ldb + k, v);
    if constexpr (is_norm(kOp)) {
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
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int64_t row = blockIdx.x;
  Squares<kOp> ss;
  float u[kE], h[kE];
  uint32_t top = 0;
  for (int64_t k = (int64_t)threadIdx.x * kE; k < p.cols; k += 512 * kE) {
    units<T, kOp, kE>(p, row, k, u, h);
#pragma unroll
    for (int j = 0; j < kE; ++j) {
      if constexpr (is_norm(kOp)) ss.add(h[j]);
      top = max(top, __float_as_uint(fabsf(u[j])));
    }
  }
  block_stats(top, ss);
  float inv, scale;
  row_scale(p, p.cols, __uint_as_float(top), ss, inv, scale);
  if (threadIdx.x == 0) p.scales[row] = scale;
  for (int64_t k = (int64_t)threadIdx.x * kE; k < p.cols; k += 512 * kE) {
    units<T, kOp, kE>(p, row, k, u, h);
    if (is_norm(kOp) && p.sum) store_vec<kE>(static_cast<T*>(p.sum) + row * p.ld_sum + k, h);
    if (isnan(scale)) {
#pragma unroll
      for (int j = 0; j < kE; ++j) u[j] = 0.0f;
    }
    write_codes<kE, false>(p, row, k, inv, scale, u);
  }
}

// How the rows lie for rows_held_kernel: whole vectors; whole but for their ends (they start at the same element of a vector
// in every tensor but the weights); so the outputs alone, and the inputs anyhow; or all anyhow.
enum Lie { kWhole, kShifted, kLoose, kAnyhow };

// One block per row, which waits in shared memory: all of it is on its way at once, and few registers let several blocks share an SM. A
// thread copies, and later reads, its own vectors, and u takes the place of the two inputs that it came from (a single
// input of 16 bits is read twice instead). kLoose, kAnyhow: whole vectors of the aligned memory that holds the rows, their edges element by
// element, and u in a place of its own; the threads then take the outputs' vectors, or the row's elements, in turn.
// kSplit (of kWhole): a cluster of `splits` blocks per row, `part` columns each, which join their statistics.
template <class T, RowOp kOp, Lie kLie, bool kSplit>
__global__ void __launch_bounds__(512, (kLie == kShifted && is_norm(kOp)) || kLie == kLoose || (kSplit && kOp == kRowNormSmall) ? 2 : 3)
rows_held_kernel(const RowArgs call, const int bytes, const int splits, const int part) {
  extern __shared__ __align__(16) uint8_t smem[];  // a, then b where there are two (`bytes` each), then u (kLoose, kAnyhow)
  constexpr int kE = 16 / sizeof(T);
  __shared__ uint4 joined[kSplit ? 8 : 1];  // every block's maximum and squares
  RowArgs p = call;
  if constexpr (kSplit) {  // from here on a row is this block's part of it
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // (waited for before the first store into another block)
    const int64_t k0 = (int64_t)blockIdx.x * part;
    p.cols = min(part, call.cols - (int)k0);
    p.a = static_cast<const T*>(p.a) + k0;
    if (p.b) p.b = static_cast<const T*>(p.b) + k0;
    if (p.sum) p.sum = static_cast<T*>(p.sum) + k0;
    if (p.weight) p.weight = static_cast<const uint8_t*>(p.weight) + k0 * (p.weight_dtype == AQD_F32 ? 4 : 2);
    if (p.codes) p.codes += k0;
    if (p.values) p.values = static_cast<uint8_t*>(p.values) + k0 * (p.values_dtype == AQD_F32 ? 4 : 2);
  }
  constexpr bool kVec = kLie != kAnyhow, kOwn = kLie == kWhole || kLie == kShifted, kShift = kLie == kShifted || kLie == kLoose;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int64_t row = kSplit ? blockIdx.y : blockIdx.x;
  const bool two = kOp == kRowGated || (is_norm(kOp) && p.b);
  const T* ab[2] = {static_cast<const T*>(p.a) + row * p.lda, static_cast<const T*>(p.b) + row * p.ldb};
  int off[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (i == 1 && !two) break;
    uint8_t* to = smem + i * bytes;
    int v0 = 0, v1 = p.cols / kE;
    if constexpr (kLie != kWhole) {
      off[i] = (int)((reinterpret_cast<uintptr_t>(ab[i]) & 15) / sizeof(T));
      v0 = off[i] > 0;
      v1 = (off[i] + p.cols) / kE;
    }
    if constexpr (!kOwn) {
      // the edges, an element a thread: the first kE - off, and those from vector v1 on
      const int t = threadIdx.x, k = t < 32 ? t : v1 * kE - off[i] + t - 32;
      if (t < 32 ? v0 > 0 && k < kE - off[i] && k < p.cols : t < 32 + kE && k >= 0 && k < p.cols)
        reinterpret_cast<T*>(to)[off[i] + k] = ab[i][k];
      for (int v = v0 + (int)threadIdx.x; v < v1; v += blockDim.x) tc::cp_async<16>(tc::smem_u32(to + v * 16), ab[i] + v * kE - off[i], true);
    } else {
      for (int v = threadIdx.x; v * kE - off[i] < p.cols; v += blockDim.x) {
        if (!kShift || (v >= v0 && v < v1)) {
          tc::cp_async<16>(tc::smem_u32(to + v * 16), ab[i] + v * kE - off[i], true);
        } else {  // cut by the row's ends: what is not the row's is 0
          float f[kE];
          load_each<kE>(ab[i], v * kE - off[i], p.cols, f);
          store_vec<kE>(reinterpret_cast<T*>(to) + v * kE, f);
        }
      }
    }
  }
  tc::cp_async_commit();
  tc::cp_async_wait<0>();
  if (!kOwn) __syncthreads();
  Squares<kOp> ss;
  uint32_t top = 0;
  constexpr int kU = kVec ? kE : 1;
  const bool again = kOwn && sizeof(T) == 2 && !two;  // u is computed twice
  float* us = reinterpret_cast<float*>(smem + (two ? 2 : 1) * bytes);
  int out = kShift ? off[0] : 0;  // the outputs' first element's place in its vector
  if constexpr (kLie == kLoose) {
    if (p.codes) out = (int)(reinterpret_cast<uintptr_t>(p.codes + row * p.ld_codes) % kE);
    else {
      const int size = p.values_dtype == AQD_F32 ? 4 : 2;
      out = (int)(((reinterpret_cast<uintptr_t>(p.values) / size) + row * p.ld_values) % kE);
    }
  }
  // kU values from element k of an input on
  auto input = [&](int i, int k, float (&f)[kU]) {
    const T* from = reinterpret_cast<const T*>(smem + i * bytes);
    if constexpr (kLie != kLoose) load_vec<kU>(from + off[i] + k, f);
    else if (inside<kU, true>(k, p.cols)) load_across<kU>(from, off[i] + k, f);
    else load_each<kU>(from + off[i], k, p.cols, f);
  };
  // kU values from element k on: u and, under the norm, h
  auto units_of = [&](int k, float (&u)[kU], float (&h)[kU]) {
    input(0, k, u);
    if constexpr (kOp != kRowPlain) {
      float v[kU];
      if (two) input(1, k, v);
      if constexpr (is_norm(kOp)) {
        if (two) {
#pragma unroll
          for (int j = 0; j < kU; ++j) u[j] += v[j];
        }
        load_weight<kU, kShift>(p, k, v);
#pragma unroll
        for (int j = 0; j < kU; ++j) { h[j] = u[j]; u[j] *= v[j]; }
      } else {
#pragma unroll
        for (int j = 0; j < kU; ++j) u[j] = activate(u[j], p.act) * v[j];
      }
    }
  };
  const int first = (int)threadIdx.x * kU - out, step = (int)blockDim.x * kU;
  for (int k = first; k < p.cols; k += step) {
    float u[kU], h[kU];
    units_of(k, u, h);
    if (is_norm(kOp) && p.sum) store_sum<kU, kShift, T>(p, row, k, h);
#pragma unroll
    for (int j = 0; j < kU; ++j) {
      if constexpr (is_norm(kOp)) ss.add(h[j]);
      top = max(top, __float_as_uint(fabsf(u[j])));
    }
    if constexpr (!kOwn) store_vec<kU>(us + k + out, u);
    else if (!again) {
      uint4* at = reinterpret_cast<uint4*>(smem) + (k + out) / kE;
      at[0] = make_uint4(__float_as_uint(u[0]), __float_as_uint(u[1]), __float_as_uint(u[2]), __float_as_uint(u[3]));
      if constexpr (kE == 8)
        *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(at) + bytes) = make_uint4(__float_as_uint(u[4]), __float_as_uint(u[5]), __float_as_uint(u[6]), __float_as_uint(u[7]));
    }
  }
  block_stats(top, ss);
  if constexpr (kSplit) {
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    if ((int)threadIdx.x < splits) {
      const uint32_t to = tc::mapa_shared(tc::smem_u32(&joined[blockIdx.x]), threadIdx.x);
      asm volatile("st.shared::cluster.v2.u32 [%0], {%1, %2};" ::"r"(to), "r"(top), "r"(__float_as_uint(ss.sum)) : "memory");
      if constexpr (kOp == kRowNormSmall) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to + 8), "r"(__float_as_uint(ss.low)) : "memory");
    }
    tc::cluster_sync();
    ss = Squares<kOp>();
    for (int i = 0; i < splits; ++i) {  // in the blocks' order
      top = max(top, joined[i].x);
      Squares<kOp> other;
      other.sum = __uint_as_float(joined[i].y);
      if constexpr (kOp == kRowNormSmall) other.low = __uint_as_float(joined[i].z);
      ss.join(other);
    }
  }
  float inv, scale;
  row_scale(p, call.cols, __uint_as_float(top), ss, inv, scale);
  if (threadIdx.x == 0 && (!kSplit || blockIdx.x == 0)) p.scales[row] = scale;
  for (int k = first; k < p.cols; k += step) {
    float u[kU], h[kU];
    if constexpr (!kOwn) load_vec<kU>(us + k + out, u);
    else if (again) units_of(k, u, h);
    else {
      const uint4* at = reinterpret_cast<const uint4*>(smem) + (k + out) / kE;
      load_vec<4>(reinterpret_cast<const float*>(at), *reinterpret_cast<float(*)[4]>(&u[0]));
      if constexpr (kE == 8)
        load_vec<4>(reinterpret_cast<const float*>(reinterpret_cast<const uint8_t*>(at) + bytes), *reinterpret_cast<float(*)[4]>(&u[kE / 2]));
    }
    if (isnan(scale)) {
#pragma unroll
      for (int j = 0; j < kU; ++j) u[j] = 0.0f;
    }
    write_codes<kU, kShift>(p, row, k, inv, scale, u);
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

template <class T, RowOp kOp, Lie kLie, bool kSplit>
static cudaError_t start_held(const RowArgs& a, cudaStream_t stream, int splits = 1) {
  const int kE = 16 / (int)sizeof(T);
  const int part = kSplit ? (a.cols / kE + splits - 1) / splits * kE : a.cols, bytes = (part + 2 * kE - 2) / kE * 16;
  const int smem = (kOp == kRowGated || a.b ? 2 : 1) * bytes + (kLie < kLoose ? 0 : bytes / 16 * kE * 4);
  void (*kernel)(RowArgs, int, int, int) = rows_held_kernel<T, kOp, kLie, kSplit>;
  // (a block has 48 KB without asking, the kernel's own arrays among them: 128 to 320 bytes)
  if (smem > 40 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kHeldBytes);
    if (e != cudaSuccess) return e;
  }
  const int units = kLie != kAnyhow ? bytes / 16 : a.cols;
  // Three vectors a thread; four or five where that lets more blocks share an SM: of kLoose, for its registers (3000 x 3333 f16, gated, four
  // 20.3 us, three 22.2, two 24.8), and of a cluster, whose parts are shorter (3000 x 10240 f32, gated, five 58, four 63, three 74; 1000 x
  // 16384 f32, the norm, five 51, four 48).
  constexpr int kEach = kLie == kLoose ? 4 : !kSplit ? 3 : kOp == kRowGated ? 5 : 4;
  int threads = (units + kEach - 1) / kEach;
  threads = threads < 64 ? 64 : (threads > 512 ? 512 : (threads + 31) / 32 * 32);
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)splits;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  if constexpr (!kSplit) {
    cfg.gridDim = dim3((unsigned)a.rows);
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, bytes, 1, part);
  } else {
    cfg.numAttrs = 2;
    constexpr int64_t most = 65535;  // the grid's second dimension: the rows in pieces
    for (int64_t m = 0; m < a.rows; m += most) {
      RowArgs p = a;
      p.rows = a.rows - m < most ? a.rows - m : most;
      p.a = static_cast<const T*>(a.a) + m * a.lda;
      if (p.b) p.b = static_cast<const T*>(a.b) + m * a.ldb;
      if (p.sum) p.sum = static_cast<T*>(a.sum) + m * a.ld_sum;
      if (p.codes) p.codes += m * a.ld_codes;
      if (p.values) p.values = static_cast<uint8_t*>(a.values) + m * a.ld_values * (a.values_dtype == AQD_F32 ? 4 : 2);
      p.scales += m;
      cfg.gridDim = dim3((unsigned)splits, (unsigned)p.rows);
      const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p, bytes, splits, part);
      if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
  }
}
// Whether a row fits its share of an SM's shared memory.
template <class T>
static bool held(const RowArgs& a, Lie lie) {
  const int64_t kE = 16 / (int)sizeof(T), bytes = ((int64_t)a.cols + 2 * kE - 2) / kE * 16;
  return (a.b ? 2 : 1) * bytes + (lie < kLoose ? 0 : bytes / 16 * kE * 4) <= kHeldBytes;
}

static bool whole(const void* p, int64_t ld, int size, int bytes) {
  return p == nullptr || ((reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) == 0 && (ld * size) % bytes == 0);
}
static int size_of(int dtype) { return dtype == AQD_F32 ? 4 : 2; }

// Rows in vectors. A warp per row with up to 4 vectors a lane, where the rows fill the GPU that way; else a block, in registers with one
// vector a thread (two, of 32-bit values or for few rows); longer rows in shared memory. (4096 rows of 4096 bf16, the norm: one
// vector a thread 26 us, two 30, four 35; 4096 x 12288 f16, gated: four 85 us, three 74, read twice 69, in shared memory 56.)
template <class T, RowOp kOp, bool kShift>
static cudaError_t run_vectors(const RowArgs& a, cudaStream_t stream) {
  constexpr int kE = 16 / sizeof(T);
  const unsigned rows = (unsigned)a.rows;
  auto block = [](int64_t n, int v) { return (unsigned)(((n + v - 1) / v + 31) / 32 * 32); };  // threads for n vectors, v each
  if constexpr (kShift) {
    // (4096 x 1001 bf16, the norm: 11.7 us, an element at a time 14.2; 500 x 5001 f16: in shared memory 7.5, in registers 8.8, an element
    // at a time 11.2; 2000 x 7777 bf16: 43.8, 52.4, 55; 100 x 3001: in registers 3.3, in shared memory 4.4.)
    const int64_t n = ((int64_t)a.cols + 2 * kE - 2) / kE;
    if (n <= (rows > 304 ? 256 : 1024)) return start(rows_kernel<T, kOp, kE, 1, false, true>, rows, block(n, 1), a, stream);
  } else {
    const int64_t n = a.cols / kE;
    if (n <= 32) return start(rows_kernel<T, kOp, kE, 1, true, false>, (rows + 7) / 8, 256, a, stream);
    if (n <= 64 && rows > 608) return start(rows_kernel<T, kOp, kE, 2, true, false>, (rows + 7) / 8, 256, a, stream);
    if (n <= 128 && rows > 608) return start(rows_kernel<T, kOp, kE, 4, true, false>, (rows + 7) / 8, 256, a, stream);
    if (n <= 1024) return start(rows_kernel<T, kOp, kE, 1, false, false>, rows, block(n, 1), a, stream);
    if (n <= 2048 && (kE == 4 || rows <= 304)) return start(rows_kernel<T, kOp, kE, 2, false, false>, rows, block(n, 2), a, stream);
  }
  return start_held<T, kOp, kShift ? kShifted : kWhole, false>(a, stream);
}

template <class T, RowOp kOp>
static cudaError_t run(const RowArgs& a, cudaStream_t stream) {
  constexpr int kE = 16 / sizeof(T);
  const int ts = (int)sizeof(T), vs = size_of(a.values_dtype), wbytes = kE * size_of(a.weight_dtype) > 16 ? 16 : kE * size_of(a.weight_dtype);
  const bool vec = a.cols % kE == 0 && whole(a.a, a.lda, ts, 16) && whole(a.b, a.ldb, ts, 16) && whole(a.sum, a.ld_sum, ts, 16) &&
                   whole(a.codes, a.ld_codes, 1, kE) && whole(a.values, a.ld_values, vs, kE * vs > 16 ? 16 : kE * vs) &&
                   whole(a.weight, 0, 1, wbytes);
  const unsigned rows = (unsigned)a.rows;
  auto block = [](int64_t n, int v) { return (unsigned)(((n + v - 1) / v + 31) / 32 * 32); };  // threads for n elements, v each
  if (vec) {
    if (a.cols <= 1024 * kE || held<T>(a, kWhole)) return run_vectors<T, kOp, false>(a, stream);
    // Longer rows in the shared memory of a cluster; for few rows of more blocks than they need. (1500 x 32768 f32, gated: 97 us, read twice
    // 138; 1000 x 131072 bf16, gated, 171 and 229; 300 x 131072 bf16, the norm, 69 and 102; one row of 32768 f32, gated, 3.3 and 11.8.)
    const int64_t room = kHeldBytes / 16 / (a.b ? 2 : 1) - 2, n = a.cols / kE;
    int64_t splits = (n + room - 1) / room;
    if (splits <= 8) {
      if (splits < 304 / rows) splits = 304 / rows < 8 ? 304 / rows : 8;
      return start_held<T, kOp, kWhole, true>(a, stream, (int)splits);
    }
    return start(rows_long_kernel<T, kOp, kE>, rows, 512, a, stream);
  }
  // Whether every tensor's rows start at the same element of their vectors. (Up to 64 vectors the ends are too many of them: 4096 x 257
  // bf16, the norm, 6.4 us, an element at a time 5.9; 4096 x 513 8.9 and 9.3.)
  auto alike = [&](const void* p, int64_t ld, int size, const void* q, int64_t ldq, int sizeq) {
    return p == nullptr || q == nullptr ||
           ((reinterpret_cast<uintptr_t>(p) / size - reinterpret_cast<uintptr_t>(q) / sizeq) % kE == 0 && (ld - ldq) % kE == 0);
  };
  const bool outputs = alike(a.sum, a.ld_sum, ts, a.codes, a.ld_codes, 1) && alike(a.values, a.ld_values, vs, a.codes, a.ld_codes, 1) &&
                       alike(a.sum, a.ld_sum, ts, a.values, a.ld_values, vs);
  const bool all = outputs && alike(a.b, a.ldb, ts, a.a, a.lda, ts) && alike(a.codes, a.ld_codes, 1, a.a, a.lda, ts) &&
                   alike(a.values, a.ld_values, vs, a.a, a.lda, ts);
  if (all && a.cols > 64 * kE && held<T>(a, kShifted)) return run_vectors<T, kOp, true>(a, stream);
  // The outputs' rows alike, the inputs' not (the two halves of rows of an odd width): 3000 x 3333 f16, gated, 20.3 us, an element at a time 32;
  // 1000 x 2049 bf16 6.8 and 11.5; 5000 x 777 13.6 and 11.6.
  if (outputs && a.cols > 2048 && held<T>(a, kLoose)) return start_held<T, kOp, kLoose, false>(a, stream);
  // Rows at any address: an element at a time, neighbours by neighbours. (4096 x 1001 bf16, the norm: eight 14.2 us, in shared memory
  // 29; 2000 x 7777: 68 and 55; 5000 x 777, gated: eight 15.5, four 11.7.)
  if (a.cols <= 256 && rows > 608) return start(rows_kernel<T, kOp, 1, 8, true, false>, (rows + 7) / 8, 256, a, stream);
  if (a.cols <= (kOp == kRowGated ? 2048 : 768)) return start(rows_kernel<T, kOp, 1, 4, false, false>, rows, block(a.cols, 4), a, stream);
  if (kOp != kRowGated && a.cols <= 6144) return start(rows_kernel<T, kOp, 1, 8, false, false>, rows, block(a.cols, 8), a, stream);
  if (held<T>(a, kAnyhow)) return start_held<T, kOp, kAnyhow, false>(a, stream);
  return start(rows_long_kernel<T, kOp, 1>, rows, 512, a, stream);
}
template <class T>
static cudaError_t run_op(RowOp op, const RowArgs& a, cudaStream_t stream) {
  if (op == kRowPlain) return run<T, kRowPlain>(a, stream);
  if constexpr (!std::is_same<T, __half>::value) {  // (no square of a binary16 value or sum is that small)
    if (op == kRowNorm && a.eps < kMinNormal) return run<T, kRowNormSmall>(a, stream);
  }
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
