// lm_heads.cu -- rows of heads before attention: norms of queries and keys with the position rotation, and the 4-bit cache's
// quantizer, in one pass; the cache's values read back.
//
// A row is one token's vector of one head. Some lanes of a warp hold it in registers, each with two vectors that the rotation pairs (i and
// i + rot / 2), or that hold its pairs themselves (interleaved), so norm, rotation and codes take one read and one write, and what crosses
// lanes is a sum of squares and a row's lowest and highest value. Bound by memory.
//
// The angle of position p at frequency f is p f / 2 pi turns, of which the whole ones do not count: with u = frac(f / 2 pi) 2^64 rounded to
// an integer, p u mod 2^64 is the fraction, exact but for |p| 2^-64 of a turn (and the 2^-53 of u's own product), whatever the position. A block's
// sines and cosines are computed once, for all heads.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/aqd.h"
#include "common.cuh"
#include "kernels.h"
#include "tc_ptx.cuh"

namespace aqd {
namespace headrows {

constexpr int kThreads = 256;

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <class T, int V>
struct alignas(sizeof(T) * V) Vec {
  T x[V];
};
template <int V, class T>
__device__ __forceinline__ void load(const T* p, float (&f)[V]) {
  const Vec<T, V> v = *reinterpret_cast<const Vec<T, V>*>(p);
#pragma unroll
  for (int i = 0; i < V; ++i) f[i] = to_f32(v.x[i]);
}
template <int V, class T>
__device__ __forceinline__ void store(T* p, const float (&f)[V]) {
  Vec<T, V> v;
#pragma unroll
  for (int i = 0; i < V; ++i) v.x[i] = from_f32<T>(f[i]);
  *reinterpret_cast<Vec<T, V>*>(p) = v;
}
// weights, V at a time (V = 8 float32: two vectors)
template <int V>
__device__ __forceinline__ void load_weight(const void* p, int k, int dtype, float (&f)[V]) {
  if (dtype == AQD_F32) {
    if constexpr (V == 8) {
      float a[4], b[4];
      load<4>(static_cast<const float*>(p) + k, a);
      load<4>(static_cast<const float*>(p) + k + 4, b);
#pragma unroll
      for (int i = 0; i < 4; ++i) { f[i] = a[i]; f[i + 4] = b[i]; }
    } else {
      load<V>(static_cast<const float*>(p) + k, f);
    }
  } else if (dtype == AQD_F16) {
    load<V>(static_cast<const __half*>(p) + k, f);
  } else {
    load<V>(static_cast<const __nv_bfloat16*>(p) + k, f);
  }
}
__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// A row's lowest value and step, as the cache keeps them; NaN for both where a value is none or the span is out of range.
struct RowStep {
  float low, step, inv;
  uint32_t word;
  __device__ __forceinline__ RowStep(float lo, float hi) {
    const __nv_bfloat16 l = __float2bfloat16_rd(lo);
    low = __bfloat162float(l);
    __nv_bfloat16 s = __float2bfloat16_ru(__fdiv_rn(__fsub_rn(hi, low), 15.0f));
    step = __bfloat162float(s);
    if (hi == low) s = __float2bfloat16_rn(0.0f);
    else if (step < 0x1p-126f) s = __float2bfloat16_rn(0x1p-126f);
    step = __bfloat162float(s);
    const bool fine = fabsf(low) < INFINITY && step < INFINITY;
    inv = fine && step > 0.0f ? __frcp_rn(step) : 0.0f;
    word = fine ? (uint32_t)__bfloat16_as_ushort(l) | (uint32_t)__bfloat16_as_ushort(s) << 16 : 0x7fc07fc0u;
    if (!fine) low = step = 0.0f;
  }
  // (x - low) / step to the nearest, ties to even. d * inv is off by 2^-23 of it, so only its integer can be wrong, by one, next to a tie;
  // what is left of d under it decides, exactly (16-bit values meet exact ties often).
  __device__ __forceinline__ uint32_t code(float x) const {
    const float d = __fsub_rn(x, low);
    float n = __fadd_rn(__fmaf_rn(d, inv, 12582912.0f), -12582912.0f);
    const float r = __fmaf_rn(-n, step, d), h = 0.5f * step;
    if (fabsf(r) >= h) {
      const bool odd = ((int)n & 1) != 0;
      if (r > h || (r == h && odd)) n += 1.0f;
      else if (r < -h || (r == -h && odd)) n -= 1.0f;
    }
    return inv > 0.0f ? (uint32_t)(int)n & 15u : 0u;
  }
};

// The block of 16 places of a slot, and the slot's row in it.
__device__ __forceinline__ uint8_t* place(const CacheGeom& c, int64_t slot, int head, int& row) {
  const int64_t page = slot >> c.page_shift;
  const int in = (int)(slot & ((1 << c.page_shift) - 1));
  row = in & 15;
  return c.data + (((page * c.kv_heads + head) << (c.page_shift - 4)) + (in >> 4)) * (16 * ((int64_t)c.dim + 8));
}
__device__ __forceinline__ bool in_cache(const CacheGeom& c, int64_t slot) { return slot >= 0 && (slot >> c.page_shift) < c.pages; }

// V: elements of a vector (8 of 16 bits, 4 of 32; 1 for rows at any address or with any rot), kC: pairs of vectors a lane. lanes: those of a
// row, a power of two, 32 for V = 1. A block takes `per` tokens, all rows of them.
template <class T, int V, int kC, bool kCache>
__global__ void __launch_bounds__(kThreads) heads_kernel(const QkArgs p, const int per, const int lanes, const uint64_t rows_magic) {
  extern __shared__ float2 turns[];  // [per][rot / 2]: cosine, sine
  __shared__ uint8_t bytes[V == 1 && kCache ? kThreads / 32 * 256 : 1];
  tc::grid_dep_wait();
  const int64_t t0 = (int64_t)blockIdx.x * per;
  const int here = (int)(p.tokens - t0 < per ? p.tokens - t0 : per), half = p.rot >> 1;
  for (int i = threadIdx.x; i < here * half; i += kThreads) {
    const int t = half == 0 ? 0 : i / half, f = i - t * half;
    double turn = (double)p.inv_freq[f] * 0.15915494309189535;
    turn -= floor(turn);
    const uint64_t u = __double2ull_rn(turn * 18446744073709551616.0);  // (a turn rounded up to 1 wraps in the product alike)
    const uint64_t frac = (uint64_t)p.positions[t0 + t] * u;
    float s, c;
    sincospif((float)(int32_t)(uint32_t)((frac + 0x80000000ull) >> 32) * 0x1p-31f, &s, &c);
    turns[i] = make_float2(c, s);
  }
  __syncthreads();
  const int each = p.heads + p.kv_heads * (kCache ? 2 : 1), rows = here * each;  // rows of a token: queries, keys, values
  const int lane = threadIdx.x & (lanes - 1), group = threadIdx.x / lanes, groups = kThreads / lanes;
  for (int r0 = 0; r0 < rows; r0 += groups) {
    const int r = r0 + group;
    const bool live = r < rows;
    const int t = fast_div(live ? r : 0, rows_magic), h = (live ? r : 0) - t * each;
    const int64_t token = t0 + t;
    const bool is_q = h < p.heads, is_v = kCache && h >= p.heads + p.kv_heads;
    const int kh = is_v ? h - p.heads - p.kv_heads : h - p.heads;
    const T* x = is_q ? static_cast<const T*>(p.q) + token * p.ldq + h * p.ldqh
               : is_v ? static_cast<const T*>(p.v) + token * p.ldv + kh * p.ldvh
                      : static_cast<const T*>(p.k) + token * p.ldk + kh * p.ldkh;
    float a[kC][V], b[kC][V];
    int ia[kC], ib[kC];
    float ss = 0.0f;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      const int i = lane + c * 32;  // (lanes is 32 where there are several)
      if (p.interleaved || i * V >= half) {
        ia[c] = 2 * i * V;
        ib[c] = ia[c] + V;
      } else {
        ia[c] = i * V;
        ib[c] = ia[c] + half;
      }
      const bool in = live && 2 * i * V < p.dim;
#pragma unroll
      for (int j = 0; j < V; ++j) a[c][j] = b[c][j] = 0.0f;
      if (in) {
        load<V>(x + ia[c], a[c]);
        load<V>(x + ib[c], b[c]);
      } else {
        ia[c] = -1;
      }
#pragma unroll
      for (int j = 0; j < V; ++j) ss = fmaf(a[c][j], a[c][j], fmaf(b[c][j], b[c][j], ss));
    }
    const void* w = is_v ? nullptr : is_q ? p.q_weight : p.k_weight;
    for (int o = lanes >> 1; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    if (w) {
      const float rms = rsqrtf(ss / (float)p.dim + p.eps);
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        if (ia[c] < 0) continue;
        float wa[V], wb[V];
        load_weight<V>(w, ia[c], p.weight_dtype, wa);
        load_weight<V>(w, ib[c], p.weight_dtype, wb);
#pragma unroll
        for (int j = 0; j < V; ++j) {
          a[c][j] = a[c][j] * rms * wa[j];
          b[c][j] = b[c][j] * rms * wb[j];
        }
      }
    }
    if (!is_v) {
      const float2* turn = turns + t * half;
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        if (ia[c] < 0) continue;
        if (V > 1 && p.interleaved) {  // pairs within each vector
#pragma unroll
          for (int j = 0; j + 1 < V; j += 2) {
            if (ia[c] < p.rot) {
              const float2 cs = turn[(ia[c] + j) >> 1];
              const float u = a[c][j], v = a[c][j + 1];
              a[c][j] = u * cs.x - v * cs.y;
              a[c][j + 1] = v * cs.x + u * cs.y;
            }
            if (ib[c] < p.rot) {
              const float2 cs = turn[(ib[c] + j) >> 1];
              const float u = b[c][j], v = b[c][j + 1];
              b[c][j] = u * cs.x - v * cs.y;
              b[c][j + 1] = v * cs.x + u * cs.y;
            }
          }
        } else {
          const int f = (lane + c * 32) * V;  // pairs between the two
          if (f < half) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
              const float2 cs = turn[f + j];
              const float u = a[c][j], v = b[c][j];
              a[c][j] = u * cs.x - v * cs.y;
              b[c][j] = v * cs.x + u * cs.y;
            }
          }
        }
      }
      T* y = is_q ? static_cast<T*>(p.q_out) + token * p.ldqo + h * p.ldqoh
                  : (p.k_out ? static_cast<T*>(p.k_out) + token * p.ldko + kh * p.ldkoh : nullptr);
      if (y) {
#pragma unroll
        for (int c = 0; c < kC; ++c) {
          if (ia[c] < 0) continue;
          store<V>(y + ia[c], a[c]);
          store<V>(y + ib[c], b[c]);
        }
      }
    }
    if constexpr (kCache) {
      float lo = INFINITY, hi = -INFINITY;
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        if (ia[c] < 0) continue;
#pragma unroll
        for (int j = 0; j < V; ++j) {
          a[c][j] = to_f32(from_f32<T>(a[c][j]));  // codes are of the rounded values, whether these are stored or not
          b[c][j] = to_f32(from_f32<T>(b[c][j]));
          lo = min_nan(lo, min_nan(a[c][j], b[c][j]));
          hi = max_nan(hi, max_nan(a[c][j], b[c][j]));
        }
      }
      for (int o = lanes >> 1; o > 0; o >>= 1) {
        lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
      }
      const int64_t slot = live && !is_q ? p.slots[token] : -1;
      const bool kept = in_cache(p.cache, slot);
      const RowStep rs(lo, hi);
      int row = 0;
      uint8_t* blk = kept ? place(p.cache, slot, kh, row) : nullptr;
      uint8_t* codes = kept ? blk + (is_v ? 8 * p.dim : 0) + row * (p.dim >> 1) : nullptr;
      if (kept && lane == 0) *reinterpret_cast<uint32_t*>(blk + 16 * p.dim + (is_v ? 64 : 0) + 4 * row) = rs.word;
      if constexpr (V > 1) {
        if (kept && ia[0] >= 0) {
          uint32_t wa = 0, wb = 0;
#pragma unroll
          for (int j = 0; j < V; ++j) {
            wa |= rs.code(a[0][j]) << (4 * j);
            wb |= rs.code(b[0][j]) << (4 * j);
          }
          if constexpr (V == 8) {
            *reinterpret_cast<uint32_t*>(codes + (ia[0] >> 1)) = wa;
            *reinterpret_cast<uint32_t*>(codes + (ib[0] >> 1)) = wb;
          } else {
            *reinterpret_cast<uint16_t*>(codes + (ia[0] >> 1)) = (uint16_t)wa;
            *reinterpret_cast<uint16_t*>(codes + (ib[0] >> 1)) = (uint16_t)wb;
          }
        }
      } else {  // a warp per row: codes meet their neighbours in shared memory
        uint8_t* line = bytes + (threadIdx.x >> 5) * 256;
        __syncwarp();
#pragma unroll
        for (int c = 0; c < kC; ++c) {
          if (ia[c] < 0) continue;
          line[ia[c]] = (uint8_t)rs.code(a[c][0]);
          line[ib[c]] = (uint8_t)rs.code(b[c][0]);
        }
        __syncwarp();
        if (kept && lane * 8 < p.dim) {
          uint32_t w8 = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j) w8 |= (uint32_t)line[lane * 8 + j] << (4 * j);
          *reinterpret_cast<uint32_t*>(codes + 4 * lane) = w8;
        }
      }
    }
  }
}

// A lane per word of 8 codes; `lanes` (a power of two, at least dim / 8) to a row. Rows: [token][key or value][head].
template <class T, bool kVec>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const CacheReadArgs p, const int lanes, const uint64_t rows_magic) {
  tc::grid_dep_wait();
  const CacheGeom& g = p.cache;
  const int lane = threadIdx.x & (lanes - 1), groups = kThreads / lanes, each = 2 * g.kv_heads;
  const int64_t rows = p.tokens * each;
  if (lane * 8 >= g.dim) return;
  for (int64_t r = (int64_t)blockIdx.x * groups + threadIdx.x / lanes; r < rows; r += (int64_t)gridDim.x * groups) {
    const int64_t token = rows < (1ll << 31) ? fast_div((int)r, rows_magic) : r / each;
    int h = (int)(r - token * each);
    const bool is_v = h >= g.kv_heads;
    if (is_v) h -= g.kv_heads;
    T* y = is_v ? static_cast<T*>(p.v) : static_cast<T*>(p.k);
    if (!y) continue;
    y += token * (is_v ? p.ldv : p.ldk) + h * (is_v ? p.ldvh : p.ldkh) + lane * 8;
    const int64_t slot = p.slots[token];
    uint32_t w = 0, ls = 0;
    if (in_cache(g, slot)) {
      int row;
      const uint8_t* blk = place(g, slot, h, row);
      w = *reinterpret_cast<const uint32_t*>(blk + (is_v ? 8 * g.dim : 0) + row * (g.dim >> 1) + 4 * lane);
      ls = *reinterpret_cast<const uint32_t*>(blk + 16 * g.dim + (is_v ? 64 : 0) + 4 * row);
    }
    const float low = __uint_as_float(ls << 16), step = __uint_as_float(ls & 0xffff0000u);
    float f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = fmaf((float)(w >> (4 * j) & 15u), step, low);
    if constexpr (kVec) {
      if constexpr (sizeof(T) == 4) {
        const float lo4[4] = {f[0], f[1], f[2], f[3]}, hi4[4] = {f[4], f[5], f[6], f[7]};
        store<4>(y, lo4);
        store<4>(y + 4, hi4);
      } else {
        store<8>(y, f);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = from_f32<T>(f[j]);
    }
  }
}

static bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
static int pow2_at_least(int n) {
  int v = 1;
  while (v < n) v *= 2;
  return v;
}

template <class T, int V, int kC>
static cudaError_t run_heads(const QkArgs& a, cudaStream_t stream) {
  const int each = a.heads + a.kv_heads * (a.cache.data ? 2 : 1);
  const int lanes = V == 1 ? 32 : pow2_at_least(a.dim / (2 * V)), groups = kThreads / lanes;
  // tokens of a block: one while that leaves SMs without a block; else enough for four rows to a group of lanes, of which the table of
  // turns takes 16 KB at most
  int per = 1;
  while (per * 2 * each <= 8 * groups && a.tokens / (per * 2) >= 4 * 152 && per * 2 * (a.rot / 2) * 8 <= 16384) per *= 2;
  const int64_t blocks = (a.tokens + per - 1) / per;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)per * (a.rot / 2) * sizeof(float2);
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  const uint64_t magic = div_magic(each);
  if (a.cache.data) return cudaLaunchKernelEx(&cfg, heads_kernel<T, V, kC, true>, a, per, lanes, magic);
  return cudaLaunchKernelEx(&cfg, heads_kernel<T, V, kC, false>, a, per, lanes, magic);
}

template <class T>
static cudaError_t run_heads_type(const QkArgs& a, cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  bool vec = a.dim % (2 * V) == 0 && a.dim / (2 * V) <= 32 && (a.interleaved ? a.rot % V == 0 : a.rot % (2 * V) == 0);
  if (a.heads > 0) vec = vec && on16(a.q) && on16(a.q_out) && (a.ldq | a.ldqh | a.ldqo | a.ldqoh) % V == 0;
  vec = vec && on16(a.k) && (a.ldk | a.ldkh) % V == 0 && on16(a.q_weight) && on16(a.k_weight);
  if (a.k_out) vec = vec && on16(a.k_out) && (a.ldko | a.ldkoh) % V == 0;
  if (a.cache.data) vec = vec && on16(a.v) && (a.ldv | a.ldvh) % V == 0;
  return vec ? run_heads<T, V, 1>(a, stream) : run_heads<T, 1, 8>(a, stream);
}

template <class T>
static cudaError_t run_read(const CacheReadArgs& a, cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = on16(a.k) && on16(a.v) && (a.ldk | a.ldkh | a.ldv | a.ldvh) % V == 0;
  const int lanes = pow2_at_least(a.cache.dim / 8), groups = kThreads / lanes;
  const int64_t rows = a.tokens * 2 * a.cache.kv_heads, blocks = (rows + groups - 1) / groups;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(blocks < (1 << 30) ? blocks : (1 << 30)));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  const uint64_t magic = div_magic(2 * a.cache.kv_heads);
  if (vec) return cudaLaunchKernelEx(&cfg, cache_read_kernel<T, true>, a, lanes, magic);
  return cudaLaunchKernelEx(&cfg, cache_read_kernel<T, false>, a, lanes, magic);
}

}  // namespace headrows

int launch_heads(const QkArgs& a, cudaStream_t stream, std::string* err) {
  const cudaError_t e = a.dtype == AQD_F32 ? headrows::run_heads_type<float>(a, stream)
                      : a.dtype == AQD_F16 ? headrows::run_heads_type<__half>(a, stream)
                                           : headrows::run_heads_type<__nv_bfloat16>(a, stream);
  if (e == cudaSuccess) return 0;
  *err = std::string("rows of heads: ") + cudaGetErrorString(e);
  return 3;
}

int launch_cache_read(const CacheReadArgs& a, cudaStream_t stream, std::string* err) {
  const cudaError_t e = a.dtype == AQD_F32 ? headrows::run_read<float>(a, stream)
                      : a.dtype == AQD_F16 ? headrows::run_read<__half>(a, stream)
                                           : headrows::run_read<__nv_bfloat16>(a, stream);
  if (e == cudaSuccess) return 0;
  *err = std::string("cache read: ") + cudaGetErrorString(e);
  return 3;
}

}  // namespace aqd
