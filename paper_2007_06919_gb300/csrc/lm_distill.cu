// lm_distill.cu -- distillation from a teacher's top logits: the loss of each token, its normalizer, and the gradient.
//
// Bound by memory: the logits are read once and the gradient written once. A token's logits stay in registers between the
// normalizer's sum and the gradient: 16-byte vectors, eight a thread at most, spread over the threads of up to eight blocks of a
// cluster, which join their (maximum, sum) through distributed shared memory. Tokens of a larger vocabulary than that holds
// (262,144 logits of 16 bits, 131,072 of 32) are read a second time for the gradient.
//
// Exponentials are taken to base 2 (one multiply-add and one ex2.approx, within 2 units of 2^-23 of its value): with c = log2(e) / tau,
// q_v = 2^(x_v c - lse2). A row may start at any element: its first and last vectors are read and
// written element by element where they hold others'.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/aqd.h"
#include "common.cuh"
#include "kernels.h"
#include "tc_ptx.cuh"

namespace aqd {
namespace distill {

constexpr int kMaxThreads = 512, kMaxTop = 1024, kMaxSplits = 8;
constexpr int kHold = 8;  // vectors of a thread that stay in registers
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float load_f32(const float* p) { return *p; }
__device__ __forceinline__ float load_f32(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ float load_f32(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_f32(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f32(__half* p, float v) { *p = __float2half_rn(v); }
__device__ __forceinline__ void store_f32(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// A 16-byte vector of T as float32 and back; -infinity in T's bits, in every place.
template <class T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int kE = 4;
  static constexpr uint32_t kLow = 0xff800000u;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[4]) {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <>
struct Vec<__half> {
  static constexpr int kE = 8;
  static constexpr uint32_t kLow = 0xfc00fc00u;
  static __device__ __forceinline__ void two(uint32_t w, float& a, float& b) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x; b = f.y;
  }
  static __device__ __forceinline__ uint32_t one(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
    two(v.x, f[0], f[1]); two(v.y, f[2], f[3]); two(v.z, f[4], f[5]); two(v.w, f[6], f[7]);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    return make_uint4(one(f[0], f[1]), one(f[2], f[3]), one(f[4], f[5]), one(f[6], f[7]));
  }
};
template <>
struct Vec<__nv_bfloat16> {
  static constexpr int kE = 8;
  static constexpr uint32_t kLow = 0xff80ff80u;
  static __device__ __forceinline__ void two(uint32_t w, float& a, float& b) {
    a = __uint_as_float(w << 16); b = __uint_as_float(w & 0xffff0000u);
  }
  static __device__ __forceinline__ uint32_t one(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
    two(v.x, f[0], f[1]); two(v.y, f[2], f[3]); two(v.z, f[4], f[5]); two(v.w, f[6], f[7]);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    return make_uint4(one(f[0], f[1]), one(f[2], f[3]), one(f[4], f[5]), one(f[6], f[7]));
  }
};

// Vector v of a row: elements [v kE - off, v kE - off + kE) of it, off the row's first element's place in its 16 bytes.
template <class T>
__device__ __forceinline__ uint4 load_vec(const T* x, int64_t first, int vocab) {
  constexpr int kE = Vec<T>::kE;
  if (first >= 0 && first + kE <= vocab) return __ldcs(reinterpret_cast<const uint4*>(x + first));
  float f[kE];
#pragma unroll
  for (int e = 0; e < kE; ++e) f[e] = first + e >= 0 && first + e < vocab ? load_f32(x + first + e) : -INFINITY;
  return Vec<T>::pack(f);
}
template <class T>
__device__ __forceinline__ void store_vec(T* g, int64_t first, int vocab, bool whole, const float (&f)[Vec<T>::kE]) {
  constexpr int kE = Vec<T>::kE;
  if (whole && first >= 0 && first + kE <= vocab) {
    __stcs(reinterpret_cast<uint4*>(g + first), Vec<T>::pack(f));
    return;
  }
#pragma unroll
  for (int e = 0; e < kE; ++e)
    if (first + e >= 0 && first + e < vocab) store_f32(g + first + e, f[e]);
}

// The maximum m and the sum s of 2^(z - m) of a share of a softmax's terms; an empty share is (-inf, 0).
struct Soft {
  float m, s;
};
__device__ __forceinline__ Soft join(Soft a, Soft b) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) return {m, a.s + b.s};  // nothing yet (or NaN sums, which stay)
  return {m, a.s * ex2(a.m - m) + b.s * ex2(b.m - m)};
}
__device__ Soft block_join(Soft v, Soft* sh) {  // (in a fixed order: lanes, then warps)
  for (int o = 16; o > 0; o >>= 1)
    v = join(v, Soft{__shfl_xor_sync(0xffffffffu, v.m, o), __shfl_xor_sync(0xffffffffu, v.s, o)});
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  const int warps = blockDim.x >> 5, lane = threadIdx.x & 31;
  v = lane < warps ? sh[lane] : Soft{-INFINITY, 0.0f};
  for (int o = 8; o > 0; o >>= 1)
    v = join(v, Soft{__shfl_xor_sync(0xffffffffu, v.m, o), __shfl_xor_sync(0xffffffffu, v.s, o)});
  return v;  // (of lane 0 .. 15: 16 warps at most)
}
template <int kE>
__device__ __forceinline__ Soft add(Soft a, const float (&f)[kE], float c) {
  float top = f[0];
#pragma unroll
  for (int e = 1; e < kE; ++e) top = fmaxf(top, f[e]);
  const float m = fmaxf(a.m, top * c);
  const float zero = m == -INFINITY ? 0.0f : m;  // (nothing but -inf so far: every term below is 0)
  float s = a.s * ex2(a.m - zero);
#pragma unroll
  for (int e = 0; e < kE; ++e) s += ex2(fmaf(f[e], c, -zero));
  return {m, s};
}

// A token per cluster of `splits` blocks, each a range of its vectors. kRegs: the range stays in registers.
template <class T, bool kRegs>
__global__ void __launch_bounds__(kMaxThreads, 2) distill_kernel(const DistillArgs p, const int splits) {
  __shared__ int sidx[kMaxTop];
  __shared__ float sp[kMaxTop], slz[kMaxTop];
  __shared__ Soft ssoft[kMaxThreads / 32], sranks[kMaxSplits];
  __shared__ float ssum[kMaxThreads / 32];
  constexpr int kE = Vec<T>::kE;
  const int threads = blockDim.x;
  const int64_t row = blockIdx.x / (unsigned)splits;
  const int rank = (int)(blockIdx.x - (unsigned)row * (unsigned)splits);
  tc::grid_dep_wait();
  const T* x = static_cast<const T*>(p.logits) + row * p.ld_logits;
  T* g = p.grad ? static_cast<T*>(p.grad) + row * p.ld_grad : nullptr;
  const int off = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
  const bool whole = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(g)) & 15) == 0;
  const int vecs = (int)(((int64_t)p.vocab + off + kE - 1) / kE), per = (vecs + splits - 1) / splits;
  const int v0 = rank * per, v1 = min(v0 + per, vecs);
  const float rt = 1.0f / p.tau, c = kLog2e * rt;
  const float w = p.row_weight ? p.row_weight[row] : 1.0f;
  const bool sums = !p.lse_in && (w != 0.0f || p.lse);  // the normalizer is computed here
  uint4 raw[kRegs ? kHold : 1];
  if constexpr (kRegs) {
    if (sums || (g && w != 0.0f)) {
#pragma unroll
      for (int j = 0; j < kHold; ++j) {
        const int v = v0 + (int)threadIdx.x + j * threads;
        raw[j] = v < v1 ? load_vec(x, (int64_t)v * kE - off, p.vocab) : make_uint4(Vec<T>::kLow, Vec<T>::kLow, Vec<T>::kLow, Vec<T>::kLow);
      }
    }
  }
  // the kept places, in base 2; an empty one has index -1
  Soft t{-INFINITY, 0.0f};
  for (int j = threadIdx.x; j < p.top; j += threads) {
    const int64_t i = p.index[row * p.top + j];
    const float z = p.teacher[row * p.top + j] * c;
    const bool in = i >= 0 && i < p.vocab && z != -INFINITY;
    sidx[j] = in ? (int)i : -1;
    sp[j] = z;
    slz[j] = in ? load_f32(x + i) * c : 0.0f;
    if (in) {
      const float one[1] = {z};
      t = add<1>(t, one, 1.0f);
    }
  }
  t = block_join(t, ssoft);
  t = Soft{__shfl_sync(0xffffffffu, t.m, 0), __shfl_sync(0xffffffffu, t.s, 0)};
  const bool live = w != 0.0f && (t.m != -INFINITY || t.s != 0.0f);
  float lse2 = 0.0f;
  if (p.lse_in) lse2 = p.lse_in[row] * kLog2e;
  Soft s{-INFINITY, 0.0f};
  if (sums) {
    if constexpr (kRegs) {
#pragma unroll
      for (int j = 0; j < kHold; ++j) {
        if (v0 + j * threads >= v1) break;
        float f[kE];
        Vec<T>::unpack(raw[j], f);
        s = add<kE>(s, f, c);
      }
    } else {
      for (int v = v0 + (int)threadIdx.x; v < v1; v += threads) {
        float f[kE];
        Vec<T>::unpack(load_vec(x, (int64_t)v * kE - off, p.vocab), f);
        s = add<kE>(s, f, c);
      }
    }
    s = block_join(s, ssoft);
  }
  if (splits > 1) {  // (also: no block writes a gradient in place before all have read their kept places' logits)
    if (threadIdx.x < (unsigned)splits) {
      const uint32_t to = tc::mapa_shared(tc::smem_u32(&sranks[rank]), threadIdx.x);
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(s.m), "f"(s.s) : "memory");
    }
    tc::cluster_sync();
    s = sranks[0];
    for (int r = 1; r < splits; ++r) s = join(s, sranks[r]);
  } else {
    s = Soft{__shfl_sync(0xffffffffu, s.m, 0), __shfl_sync(0xffffffffu, s.s, 0)};
    __syncthreads();
  }
  if (sums) {
    lse2 = s.m == -INFINITY && s.s == 0.0f ? -INFINITY : s.m + log2f(s.s);
    if (p.lse && rank == 0 && threadIdx.x == 0) p.lse[row] = lse2 * kLn2;
  }
  float f0 = 0.0f;
  if (live) {
    const float lt = t.m + log2f(t.s);
    float loss = 0.0f;
    for (int j = threadIdx.x; j < p.top; j += threads) {
      const float lp = sp[j] - lt, pj = sidx[j] >= 0 ? exp2f(lp) : 0.0f;
      if (pj != 0.0f) loss += pj * (lp - (slz[j] - lse2));
      sp[j] = pj;
    }
    if (p.loss && rank == 0) {
      for (int o = 16; o > 0; o >>= 1) loss += __shfl_xor_sync(0xffffffffu, loss, o);
      if ((threadIdx.x & 31) == 0) ssum[threadIdx.x >> 5] = loss;
      __syncthreads();
      if (threadIdx.x == 0) {
        loss = 0.0f;
        for (int i = 0; i < threads / 32; ++i) loss += ssum[i];
        p.loss[row] = w * (loss * kLn2);
      }
    }
    f0 = w * rt;
  } else if (p.loss && rank == 0 && threadIdx.x == 0) {
    p.loss[row] = 0.0f;
  }
  if (!g) return;
  if constexpr (kRegs) {
#pragma unroll
    for (int j = 0; j < kHold; ++j) {
      const int v = v0 + (int)threadIdx.x + j * threads;
      if (v >= v1) break;
      float f[kE];
      Vec<T>::unpack(raw[j], f);
#pragma unroll
      for (int e = 0; e < kE; ++e) f[e] = live ? f0 * ex2(fmaf(f[e], c, -lse2)) : 0.0f;
      store_vec(g, (int64_t)v * kE - off, p.vocab, whole, f);
    }
  } else {
    for (int v = v0 + (int)threadIdx.x; v < v1; v += threads) {
      float f[kE];
      if (live) Vec<T>::unpack(load_vec(x, (int64_t)v * kE - off, p.vocab), f);
#pragma unroll
      for (int e = 0; e < kE; ++e) f[e] = live ? f0 * ex2(fmaf(f[e], c, -lse2)) : 0.0f;
      store_vec(g, (int64_t)v * kE - off, p.vocab, whole, f);
    }
  }
  if (!live) return;
  __syncthreads();
  // the kept places of this block's range (one listed several times takes the sum of its shares, every time alike)
  for (int j = threadIdx.x; j < p.top; j += threads) {
    const int i = sidx[j];
    const int v = (int)(((int64_t)i + off) / kE);
    if (i < 0 || v < v0 || v >= v1) continue;
    float pj = 0.0f;
    for (int l = 0; l < p.top; ++l) pj += sidx[l] == i ? sp[l] : 0.0f;
    store_f32(g + i, f0 * (ex2(slz[j] - lse2) - pj));
  }
}

template <class T>
static cudaError_t run(const DistillArgs& a, cudaStream_t stream) {
  constexpr int kE = Vec<T>::kE;
  const int64_t vecs = ((int64_t)a.vocab + 2 * kE - 2) / kE;  // at most
  int64_t splits = (vecs + kHold * kMaxThreads - 1) / (kHold * kMaxThreads);
  const bool regs = splits <= kMaxSplits;
  if (!regs) splits = kMaxSplits;
  // few tokens: more blocks a token, down to a vector a thread
  const int64_t room = 304 / a.tokens, wide = vecs / kMaxThreads;
  if (splits < room && splits < wide) splits = room < wide ? room : wide;
  if (splits > kMaxSplits) splits = kMaxSplits;
  // about four vectors a thread where they are that few
  int64_t threads = ((vecs + splits - 1) / splits + 3) / 4;
  threads = threads < 64 ? 64 : (threads > kMaxThreads ? kMaxThreads : (threads + 31) / 32 * 32);
  // (a grid holds 2^31 - 1 blocks: the tokens in pieces)
  const int64_t most = 2147483647LL / splits;
  for (int64_t m = 0; m < a.tokens; m += most) {
    DistillArgs p = a;
    p.tokens = a.tokens - m < most ? a.tokens - m : most;
    p.logits = static_cast<const T*>(a.logits) + m * a.ld_logits;
    p.index += m * a.top;
    p.teacher += m * a.top;
    if (p.row_weight) p.row_weight += m;
    if (p.grad) p.grad = static_cast<T*>(a.grad) + m * a.ld_grad;
    if (p.loss) p.loss += m;
    if (p.lse) p.lse += m;
    if (p.lse_in) p.lse_in += m;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.tokens * splits));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)splits;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = splits > 1 ? 2 : 1;
    const cudaError_t e = regs ? cudaLaunchKernelEx(&cfg, distill_kernel<T, true>, p, (int)splits)
                               : cudaLaunchKernelEx(&cfg, distill_kernel<T, false>, p, (int)splits);
    if (e != cudaSuccess) return e;
  }
  return cudaGetLastError();
}

}  // namespace distill

int launch_distill(const DistillArgs& a, cudaStream_t stream, std::string* err) {
  const cudaError_t e = a.dtype == AQD_F32   ? distill::run<float>(a, stream)
                        : a.dtype == AQD_F16 ? distill::run<__half>(a, stream)
                                             : distill::run<__nv_bfloat16>(a, stream);
  if (e != cudaSuccess) { *err = std::string("distillation launch: ") + cudaGetErrorString(e); return AQD_ERR_CUDA; }
  return 0;
}

}  // namespace aqd
