// lm_distill.cu -- distillation from a teacher's top logits: the loss of each token, its normalizer, and the gradient.
//
// The logits are read once and the gradient written once. Between the normalizer's sum and the gradient a token's
// logits stay in shared memory, spread over the blocks of a cluster (up to 48 KB each, so that several blocks share an SM and
// one's copies overlap another's sums and barriers), which join their (maximum, sum) through distributed shared memory. Every thread
// reads only what it copied itself (cp.async), so the copies need no barrier. Tokens of a larger vocabulary than eight blocks
// hold (1.6 MB of logits) are read a second time for the gradient. (2048 x 131072 bf16, loss and gradient: logits in registers 336 us,
// in shared memory 219, 4.9 TB/s; a cluster for several tokens, the next one's copies under way: 358, an SM
// then holds too few warps for the sums and exponentials.) Bound by memory and, nearly as much, by the instructions of the two passes and of
// each block's joins (70% of the issue slots): hence pairs of float32, and blocks that leave early where there is no gradient.
//
// q_v = exp(z_v - m) / s with z = x / tau: z_v - m is one multiply-add, rounded once, so that logits of any size
// (a row of the type's lowest value too) keep their differences; then a multiplication by log2(e) and ex2.approx (within 2 units of 2^-23).
// A row may start at any element: its first and last vectors are read and written element by element where they hold others'.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <climits>
#include <cstdint>

#include "../../include/aqd.h"
#include "common.cuh"
#include "kernels.h"
#include "tc_ptx.cuh"

namespace aqd {
namespace distill {

constexpr int kMaxThreads = 256, kMaxTop = 1024, kMaxSplits = 8;
constexpr int kMaxWarps = kMaxThreads / 32;
constexpr int kSlice = 48 * 1024, kMaxSlice = 200 * 1024;  // bytes of a block's logits: wanted, at most
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float load_f32(const float* p) { return *p; }
__device__ __forceinline__ float load_f32(const __half* p) { return __half2float(*p); }
__device__ __forceinline__ float load_f32(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_f32(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_f32(__half* p, float v) { *p = __float2half_rn(v); }
__device__ __forceinline__ void store_f32(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
// exp(x): 2^(x log2 e); the product's rounding, 2^-24 |x log2 e|, is relative to the result, so small where the result counts
__device__ __forceinline__ float ex(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x * kLog2e));
  return y;
}

// Two float32 at a time: half the instructions, which bound the passes over a row.
__device__ __forceinline__ uint64_t two_of(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void one_each(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// exp(x rt - zero) of two values
__device__ __forceinline__ uint64_t ex_two(float a, float b, float rt, float zero) {
  one_each(mul2(fma2(two_of(a, b), two_of(rt, rt), two_of(-zero, -zero)), two_of(kLog2e, kLog2e)), a, b);
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
  return two_of(a, b);
}

// A 16-byte vector of T as float32 and back.
template <class T>
struct Vec;
template <>
struct Vec<float> {
  static constexpr int kE = 4;
  static __device__ __forceinline__ void unpack(const uint4& v, float (&f)[4]) {
    f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ float top(const uint4& v, float m) {
    return fmaxf(fmaxf(fmaxf(m, __uint_as_float(v.x)), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <>
struct Vec<__half> {
  static constexpr int kE = 8;
  static __device__ __forceinline__ void two(uint32_t w, float& a, float& b) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    a = f.x; b = f.y;
  }
  // the larger of m and v's values (a NaN counts only where nothing else is there)
  static __device__ __forceinline__ float top(const uint4& v, float m) {
    const __half2* h = reinterpret_cast<const __half2*>(&v);
    const __half2 t = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(m, fmaxf(__low2float(t), __high2float(t)));
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
  static __device__ __forceinline__ void two(uint32_t w, float& a, float& b) {
    a = __uint_as_float(w << 16); b = __uint_as_float(w & 0xffff0000u);
  }
  static __device__ __forceinline__ float top(const uint4& v, float m) {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
    const __nv_bfloat162 t = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    return fmaxf(m, fmaxf(__low2float(t), __high2float(t)));
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

// Vector v of a row is the 16 bytes v of the aligned memory that holds it: elements [v kE - off, v kE - off + kE) of the row, off its first
// element's place in its 16 bytes. The row's first and last vectors may hold others' elements: these two are
// read (others' as -infinity) and written element by element.
template <class T>
__device__ __noinline__ uint4 load_edge(const T* x, int64_t first, int vocab) {
  constexpr int kE = Vec<T>::kE;
  float f[kE];
#pragma unroll
  for (int e = 0; e < kE; ++e) f[e] = first + e >= 0 && first + e < vocab ? load_f32(x + first + e) : -INFINITY;
  return Vec<T>::pack(f);
}
template <class T>
__device__ __forceinline__ void store_edge(T* g, int64_t first, int vocab, const float (&f)[Vec<T>::kE]) {
#pragma unroll
  for (int e = 0; e < Vec<T>::kE; ++e)
    if (first + e >= 0 && first + e < vocab) store_f32(g + first + e, f[e]);
}

// The maximum m and the sum s of exp(z - m) of a share of a softmax's terms; an empty share is (-inf, 0).
struct alignas(8) Soft {
  float m, s;
};
__device__ __forceinline__ Soft join(Soft a, Soft b) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) return {m, a.s + b.s};  // nothing yet (or NaN sums, which stay)
  return {m, a.s * ex(a.m - m) + b.s * ex(b.m - m)};
}
// Floats as integers of the same order, and back (a NaN above or below all).
__device__ __forceinline__ int ordered(float f) {
  const int i = __float_as_int(f);
  return i ^ ((i >> 31) & 0x7fffffff);
}
// A warp's shares, every lane gets the same: the largest maximum, the sums scaled to it, then added in a fixed order.
__device__ __forceinline__ Soft lanes_join(Soft v) {
  const int top = __reduce_max_sync(0xffffffffu, ordered(v.m));
  const float m = __int_as_float(top ^ ((top >> 31) & 0x7fffffff));
  v.s *= ex(v.m - (m == -INFINITY ? 0.0f : m));
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v.s += __shfl_xor_sync(0xffffffffu, v.s, o);
  return {m, v.s};
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// A share and one more term z.
__device__ __forceinline__ Soft add(Soft a, float z) {
  const float m = fmaxf(a.m, z), zero = m == -INFINITY ? 0.0f : m;
  return {m, a.s * ex(a.m - zero) + ex(z - zero)};
}
// sum exp(x rt - zero) over a vector
template <class T>
__device__ __forceinline__ float terms(const uint4& v, float rt, float zero) {
  constexpr int kE = Vec<T>::kE;
  float f[kE];
  Vec<T>::unpack(v, f);
  uint64_t sum[kE / 2];
#pragma unroll
  for (int e = 0; e < kE / 2; ++e) sum[e] = ex_two(f[2 * e], f[2 * e + 1], rt, zero);
#pragma unroll
  for (int d = kE / 4; d > 0; d >>= 1)
#pragma unroll
    for (int e = 0; e < d; ++e) sum[e] = add2(sum[e], sum[e + d]);
  one_each(sum[0], f[0], f[1]);
  return f[0] + f[1];
}

// A token per `splits` blocks, each a range of its vectors. kStay: the range stays in shared memory. together: the blocks are a cluster and
// join their sums, or write the gradient in place; else (the gradient from a given normalizer) each goes its own way.
template <class T, bool kStay>
__global__ void __launch_bounds__(kMaxThreads, kStay ? 6 : 4) distill_kernel(const DistillArgs p, const int splits, const int per, const bool together) {
  extern __shared__ __align__(16) uint8_t smem[];  // the kept places' logits, teacher logits, indices and shares, then the range
  __shared__ Soft swt[kMaxWarps], sws[kMaxSplits * kMaxWarps];  // the warps' shares: of the kept places, of the logits (all blocks')
  constexpr int kE = Vec<T>::kE;
  const int threads = blockDim.x, tops = (p.top + 3) & ~3;
  float* slz = reinterpret_cast<float*>(smem);
  float* sp = slz + tops;
  int* sidx = reinterpret_cast<int*>(sp + tops);
  float* share = reinterpret_cast<float*>(sidx + tops);
  const uint4* held = reinterpret_cast<const uint4*>(share + tops);
  const int64_t row = blockIdx.y;
  const int rank = (int)blockIdx.x;
  if (together) cluster_arrive();  // (waited for before the first store into another block: all have started)
  tc::grid_dep_wait();
  const T* x = static_cast<const T*>(p.logits) + row * p.ld_logits;
  T* g = p.grad ? static_cast<T*>(p.grad) + row * p.ld_grad : nullptr;
  const int off = (int)((reinterpret_cast<uintptr_t>(x) & 15) / sizeof(T));
  const bool whole = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(g)) & 15) == 0;
  const int vecs = (int)(((int64_t)p.vocab + off + kE - 1) / kE);
  const int v0 = rank * per, v1 = min(v0 + per, vecs);
  const int in0 = off > 0, in1 = (int)(((int64_t)p.vocab + off) / kE);  // the vectors that the row fills
  const uint4* xv = reinterpret_cast<const uint4*>(x - off);
  const float rt = 1.0f / p.tau;
  const float w = p.row_weight ? p.row_weight[row] : 1.0f;
  const bool sums = !p.lse_in && (p.lse || w != 0.0f);  // the normalizer is computed here
  if constexpr (kStay) {
    if (sums || (g && w != 0.0f)) {
      uint32_t to = tc::smem_u32(held + threadIdx.x);
      const uint4* from = xv + v0 + (int)threadIdx.x;
      int v = v0 + (int)threadIdx.x;
      if (v < in0 && v < v1) {
        const_cast<uint4*>(held)[v - v0] = load_edge(x, (int64_t)v * kE - off, p.vocab);
        v += threads, from += threads, to += threads * 16;
      }
      const int end = min(v1, in1);
#pragma unroll 4
      for (; v < end; v += threads, from += threads, to += threads * 16) tc::cp_async<16>(to, from, true);
      if (v < v1) const_cast<uint4*>(held)[v - v0] = load_edge(x, (int64_t)v * kE - off, p.vocab);
    }
    tc::cp_async_commit();
  }
  // the kept places; an empty one has index -1
  Soft t{-INFINITY, 0.0f};
  const bool joins = g || rank == 0;  // (the loss alone: the first block of a cluster has it)
  for (int j = threadIdx.x; joins && j < p.top; j += threads) {
    const int64_t i = p.index[row * p.top + j];
    const float z = p.teacher[row * p.top + j] * rt;
    const bool in = i >= 0 && i < p.vocab && z != -INFINITY;
    sidx[j] = in ? (int)i : -1;
    sp[j] = z;
    slz[j] = in ? load_f32(x + i) : 0.0f;
    if (in) t = add(t, z);
  }
  Soft s{-INFINITY, 0.0f};
  if constexpr (kStay) tc::cp_async_wait<0>();
  if (sums) {
    // a few vectors at a time: their maximum, then their terms
    constexpr int kU = 4;
    auto read = [&](int v) -> uint4 {
      if constexpr (kStay) return held[v - v0];
      return v >= in0 && v < in1 ? __ldcs(xv + v) : load_edge(x, (int64_t)v * kE - off, p.vocab);
    };
    int v = v0 + (int)threadIdx.x;
    for (; v + (kU - 1) * threads < v1; v += kU * threads) {
      uint4 raw[kU];
#pragma unroll
      for (int u = 0; u < kU; ++u) raw[u] = read(v + u * threads);
      float top = -INFINITY;
#pragma unroll
      for (int u = 0; u < kU; ++u) top = Vec<T>::top(raw[u], top);
      const float m = fmaxf(s.m, top * rt), zero = m == -INFINITY ? 0.0f : m;  // (nothing but -inf so far: every term is 0)
      s = Soft{m, s.s * ex(s.m - zero)};
#pragma unroll
      for (int u = 0; u < kU; ++u) s.s += terms<T>(raw[u], rt, zero);
    }
    for (; v < v1; v += threads) {
      const uint4 raw = read(v);
      const float m = fmaxf(s.m, Vec<T>::top(raw, -INFINITY) * rt), zero = m == -INFINITY ? 0.0f : m;
      s = Soft{m, s.s * ex(s.m - zero) + terms<T>(raw, rt, zero)};
    }
  }
  // Every warp's share to every block of the cluster, then one barrier. (Also: no gradient is written in place before all
  // blocks have read their kept places' logits.)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = threads >> 5;
  if (joins && warp * 32 < p.top) t = lanes_join(t);
  if (sums) s = lanes_join(s);
  if (lane == 0) swt[warp] = t;
  if (together) {
    cluster_wait();
    if (lane < (g ? splits : 1)) {
      const uint32_t to = tc::mapa_shared(tc::smem_u32(&sws[rank * warps + warp]), (uint32_t)lane);
      asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(s.m), "f"(s.s) : "memory");
    }
    cluster_arrive();
    if (!joins) return;
    cluster_wait();
  } else {
    if (lane == 0) sws[warp] = s;
    __syncthreads();
  }
  if (!g && warp != 0) return;
  t = lanes_join(lane < warps ? swt[lane] : Soft{-INFINITY, 0.0f});
  if (sums) {
    s = lane < splits * warps ? sws[lane] : Soft{-INFINITY, 0.0f};
    if (lane + 32 < splits * warps) s = join(s, sws[lane + 32]);
    s = lanes_join(s);
  }
  const bool live = w != 0.0f && (t.m != -INFINITY || t.s != 0.0f);
  if (sums && p.lse && rank == 0 && threadIdx.x == 0) p.lse[row] = s.m == -INFINITY && s.s == 0.0f ? -INFINITY : s.m + logf(s.s);
  if (p.lse_in) s = Soft{p.lse_in[row], 1.0f};
  const float f0 = w * rt;
  if (p.loss && rank == 0 && warp == 0) {
    float loss = 0.0f;
    if (live) {
      const float lt = logf(t.s), ls = logf(s.s);
      for (int j = lane; j < p.top; j += 32) {
        const float lp = (sp[j] - t.m) - lt, pj = sidx[j] >= 0 ? ex(sp[j] - t.m) / t.s : 0.0f;
        if (pj != 0.0f) loss += pj * (lp - (fmaf(slz[j], rt, -s.m) - ls));
      }
      for (int o = 16; o > 0; o >>= 1) loss += __shfl_xor_sync(0xffffffffu, loss, o);
      loss *= w;
    }
    if (lane == 0) p.loss[row] = loss;
  }
  if (!g) return;
  for (int j = threadIdx.x; j < p.top; j += threads) share[j] = sidx[j] >= 0 ? ex(sp[j] - t.m) / t.s : 0.0f;
  const float fs = isnan(t.s) ? NAN : f0 / s.s;  // (p a NaN: its sum, which q is multiplied by, is one too)
  uint4* gv = reinterpret_cast<uint4*>(g - off);
  auto slopes = [&](int v, bool inside, float (&f)[kE]) {
    Vec<T>::unpack(kStay ? held[v - v0] : inside ? __ldcs(xv + v) : load_edge(x, (int64_t)v * kE - off, p.vocab), f);
#pragma unroll
    for (int e = 0; e < kE; e += 2) one_each(mul2(ex_two(f[e], f[e + 1], rt, s.m), two_of(fs, fs)), f[e], f[e + 1]);
  };
  int v = v0 + (int)threadIdx.x;
  if (live && whole) {
    if (v < in0 && v < v1) {
      float f[kE];
      slopes(v, false, f);
      store_edge(g, (int64_t)v * kE - off, p.vocab, f);
      v += threads;
    }
    const int end = min(v1, in1);
#pragma unroll 2
    for (; v < end; v += threads) {
      float f[kE];
      slopes(v, true, f);
      __stcs(gv + v, Vec<T>::pack(f));
    }
  }
  for (; v < v1; v += threads) {  // the row's last vector; all, where the gradient lies otherwise than the logits, or is 0
    float f[kE];
    if (live) slopes(v, v >= in0 && v < in1, f);
    else {
#pragma unroll
      for (int e = 0; e < kE; ++e) f[e] = 0.0f;
    }
    if (whole && v >= in0 && v < in1) __stcs(gv + v, Vec<T>::pack(f));
    else store_edge(g, (int64_t)v * kE - off, p.vocab, f);
  }
  if (!live) return;
  __syncthreads();
  // the kept places of this block's range (one listed several times takes the sum of its shares, every time alike)
  for (int j = threadIdx.x; j < p.top; j += threads) {
    const int i = sidx[j], v = (int)(((int64_t)i + off) / kE);
    if (i < 0 || v < v0 || v >= v1) continue;
    float pj = 0.0f;
    for (int l = 0; l < p.top; ++l) pj += sidx[l] == i ? share[l] : 0.0f;
    store_f32(g + i, fs * ex(fmaf(slz[j], rt, -s.m)) - f0 * pj);
  }
}

template <class T>
static cudaError_t run(const DistillArgs& a, cudaStream_t stream) {
  constexpr int kE = Vec<T>::kE;
  // a row's vectors, at most: one more where rows start between vectors
  const bool aligned = (reinterpret_cast<uintptr_t>(a.logits) & 15) == 0 && a.ld_logits % kE == 0;
  const int64_t vecs = ((int64_t)a.vocab + (aligned ? kE - 1 : 2 * kE - 2)) / kE;
  const int64_t bytes = vecs * 16;
  int64_t splits = (bytes + kSlice - 1) / kSlice;
  // few tokens: more blocks a token, down to a vector a thread
  const int64_t room = 608 / a.tokens, wide = vecs / kMaxThreads;
  if (splits < room && splits < wide) splits = room < wide ? room : wide;
  if (splits > kMaxSplits) splits = kMaxSplits;
  const int64_t per = (vecs + splits - 1) / splits;
  const bool stay = per * 16 <= kMaxSlice;
  // about four vectors a thread where they are that few
  int64_t threads = (per + 3) / 4;
  threads = threads < 64 ? 64 : (threads > kMaxThreads ? kMaxThreads : (threads + 31) / 32 * 32);
  const size_t smem = (size_t)((a.top + 3) / 4 * 4) * 16 + (stay ? (size_t)per * 16 : 0);
  // (the gradient alone of 1024 x 131072 f32: 164 us, 6.6 TB/s, as clusters 205; of 2000 x 50257 bf16 71 and 79)
  const bool together = splits > 1 && (!a.lse_in || a.grad == a.logits);
  void (*kernel)(DistillArgs, int, int, bool) = stay ? distill_kernel<T, true> : distill_kernel<T, false>;
  if (smem > 40 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSlice + kMaxTop * 16);
    if (e != cudaSuccess) return e;
  }
  constexpr int64_t most = 65535;  // the grid's second dimension: the tokens in pieces
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
    cfg.gridDim = dim3((unsigned)splits, (unsigned)p.tokens);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)splits;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = together ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p, (int)splits, (int)per, together);
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
