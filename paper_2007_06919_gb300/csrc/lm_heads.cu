// lm_heads.cu -- rows of heads before attention: norms of queries and keys with the position rotation, and the 4-bit cache's
// quantizer, in one pass; the cache's values read back.
//
// A row is one token's vector of one head. Some lanes of a warp hold it in registers, each with two vectors that the rotation pairs (i and
// i + rot / 2), or that hold its pairs themselves (interleaved), so norm, rotation and codes take one read and one write, and what crosses
// lanes is a sum of squares and a row's lowest and highest value. Bound by memory, if the instructions for a value stay below about eight: a
// warp takes a token's heads in turn (rows_kernel), its lanes keep their places in the row, and with them the products of weights, cosines and sines;
// float32 goes in pairs; 16-bit minima and maxima stay packed; codes come out of the bits of one multiply-add.
//   8192 tokens of 40 heads of 128 in bfloat16: 32.6 us, 168 MB at 5.1 TB/s (47 with a row at a time, its indexes, weights and turns looked up for
//   each); with keys and values to the cache 41.6, 177 MB. 16,384 tokens' 16 rows to codes: 20.1 us, 85 MB at 4.2 TB/s (46), and back 13.8 (34).
// What holds them back is bytes on their way: 90 registers leave 20 warps an SM, with two rows' loads each and the next two's lines asked for without a
// register (38.4 us, and 47.3, with 24 warps and none asked for ahead; 36.8 with all of a token's asked for at once; 39 with 16 warps). Four rows at once
// (75 registers for codes, fewer warps) 21.7, weights and turns in shared memory 52 to 78.
// Rows at any address, and rotations of any even length, take heads_kernel, a value at a time: the 8192 tokens at odd addresses 129 us (1.3 TB/s); 777 tokens
// of 14 + 2 heads of 64 in float32 7.1, where rows_kernel takes 4.7.
//
// The angle of position p at frequency f is p f / 2 pi turns, of which the whole ones do not count: with u = frac(f / 2 pi) 2^64 cut to
// an integer, p u mod 2^64 is the fraction, exact but for |p| (1 + |f|) 2^-64 of a turn, whatever the position. A block's sines and cosines are computed
// once, for all heads.
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
namespace headrows {

constexpr int kThreads = 128;

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

__device__ __forceinline__ void prefetch(const void* p) { asm volatile("prefetch.global.L1 [%0];" ::"l"(p)); }

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

// Norms whose mean of squares and eps lie outside [2^-100, infinity): below, squares (each off by up to 2^-150) and products with weights lose bits that count in the
// result; above, the sum is infinite. The row is taken times a power of two that brings the larger of its largest value and the root of that mean to [1, 4)
// (a subnormal value to 2^-23 at least), and eps times its square. So rows of any finite values come out as ordinary ones do; one of zeros with eps = 0 is
// 0 / 0, and what holds a NaN or an infinity stays as it is.
__device__ __forceinline__ bool off_range(float mean_eps) { return __float_as_uint(mean_eps) - 0x0d800000u >= 0x7f800000u - 0x0d800000u; }
// 1 / sqrt of a mean within it
__device__ __forceinline__ float root(float mean_eps) {
  float r;
  asm("rsqrt.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(mean_eps));
  return r;
}
// That power for a row whose largest magnitude is `top`; 1 for rows that stay as they are.
__device__ __forceinline__ float into_range(float mean_eps, float top) {
  if (!off_range(mean_eps) || isnan(mean_eps) || !(top > 0.0f && top < INFINITY)) return 1.0f;
  const int e = 254 - (int)(__float_as_uint(mean_eps < INFINITY ? fmaxf(top, sqrtf(mean_eps)) : top) >> 23);
  return __uint_as_float((uint32_t)(e < 1 ? 1 : e > 253 ? 253 : e) << 23);
}

// The quotient a / b from inv, 1 / b to about a step: what a first one leaves over corrects it. Exact where the quotient is a float32 (16-bit rows meet
// codes exactly halfway between two often, and those have to stay there).
__device__ __forceinline__ float quotient(float a, float b, float inv) {
  const float q = __fmul_rn(a, inv);
  return __fmaf_rn(__fmaf_rn(-q, b, a), inv, q);
}
// A row's lowest value and step, as the cache keeps them; NaN for both where a value is none or the span is out of range.
struct RowStep {
  float low, step, inv;
  uint32_t word;
  __device__ __forceinline__ RowStep(float lo, float hi) {
    // bfloat16 is a float32's upper half: cut towards zero, or with the magnitude raised to the next
    const uint32_t b = __float_as_uint(lo);
    const uint32_t l = (b + (uint32_t)((int32_t)b >> 31 & 0xffff)) & 0xffff0000u;
    low = __uint_as_float(l);
    const float span = __fsub_rn(hi, low);
    uint32_t s = __float_as_uint(quotient(span, 15.0f, 1.0f / 15.0f)) + 0xffffu & 0xffff0000u;
    // The span and the quotient are rounded, each maybe down to 15 steps and to a step: the next step then, if 15 of these are less than the span and what
    // its rounding left over (12 bits against a number beside them: the difference is exact).
    const float back = __fsub_rn(span, hi), over = __fsub_rn(__fsub_rn(hi, __fsub_rn(span, back)), __fadd_rn(low, back));
    if (__fmaf_rn(15.0f, __uint_as_float(s), -span) < over) s += 0x10000u;
    s = hi == low ? 0u : s < 0x00800000u ? 0x00800000u : s;
    const bool fine = fabsf(low) < INFINITY && span < INFINITY;
    word = fine ? l >> 16 | s : 0x7fc07fc0u;
    step = fine ? __uint_as_float(s) : 0.0f;
    if (!fine) low = 0.0f;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(step));
    if (step == 0.0f) inv = 0.0f;
  }
  // (x - low) / step to the nearest, ties to even: the low bits under 1.5 2^23
  __device__ __forceinline__ uint32_t code(float x) const {
    return inv > 0.0f ? __float_as_uint(__fadd_rn(quotient(__fsub_rn(x, low), step, inv), 12582912.0f)) & 15u : 0u;
  }
};

// frac(f / 2 pi) 2^64: f is an integer of 24 bits times a power of two, so it is that integer times 2^64 / 2 pi, shifted (whole turns fall out at
// the top; what is cut at the bottom, and of the constant, is below (1 + |f|) 2^-64 of a turn).
__device__ __forceinline__ uint64_t turn_rate(float f) {
  constexpr uint64_t kPerTurn = 0x28be60db9391054aull;  // floor(2^64 / 2 pi)
  const uint32_t b = __float_as_uint(f), exponent = b >> 23 & 255u;
  const uint64_t m = (b & 0x7fffffu) | (exponent ? 0x800000u : 0u);
  const int e = (int)(exponent ? exponent : 1u) - 150;
  const uint64_t lo = m * kPerTurn, hi = __umul64hi(m, kPerTurn);
  uint64_t u;
  if (e >= 0) u = e < 64 ? lo << e : 0;
  else if (e > -64) u = lo >> -e | hi << (64 + e);
  else u = e > -128 ? hi >> (-64 - e) : 0;
  return b >> 31 ? 0 - u : u;
}
// Cosine and sine of position p at that rate: whole turns leave the product by themselves.
__device__ __forceinline__ float2 turn_of(uint64_t rate, int64_t p) {
  const uint64_t frac = (uint64_t)p * rate;
  float s, c;
  sincospif((float)(int32_t)(uint32_t)((frac + 0x80000000ull) >> 32) * 0x1p-31f, &s, &c);
  return make_float2(c, s);
}

// The block of 16 places of a slot, and the slot's row in it.
__device__ __forceinline__ uint8_t* place(const CacheGeom& c, int64_t slot, int head, int& row) {
  const int64_t page = slot >> c.page_shift;
  const int in = (int)(slot & ((1 << c.page_shift) - 1));
  row = in & 15;
  return c.data + (((page * c.kv_heads + head) << (c.page_shift - 4)) + (in >> 4)) * (16 * ((int64_t)c.dim + 8));
}
__device__ __forceinline__ bool in_cache(const CacheGeom& c, int64_t slot) { return slot >= 0 && (slot >> c.page_shift) < c.pages; }

// A warp per row, a value at a time: kC pairs of values a lane (rows of up to 64 kC values). A block takes `per` tokens, all rows of them.
template <class T, bool kCache>
__global__ void __launch_bounds__(kThreads) heads_kernel(const QkArgs p, const int per, const uint64_t rows_magic) {
  constexpr int kC = 8;
  extern __shared__ float2 turns[];  // [per][rot / 2]: cosine, sine
  __shared__ uint8_t bytes[kCache ? kThreads / 32 * 256 : 1];
  tc::grid_dep_wait();
  const int64_t t0 = (int64_t)blockIdx.x * per;
  const int here = (int)(p.tokens - t0 < per ? p.tokens - t0 : per), half = p.rot >> 1;
  for (int i = threadIdx.x; i < here * half; i += kThreads) {
    const int t = i / half, f = i - t * half;
    turns[i] = turn_of(turn_rate(p.inv_freq[f]), p.positions[t0 + t]);
  }
  __syncthreads();
  const int each = p.heads + p.kv_heads * (kCache ? 2 : 1), rows = here * each;  // rows of a token: queries, keys, values
  const int lane = threadIdx.x & 31;
  for (int r = threadIdx.x >> 5; r < rows; r += kThreads / 32) {
    const int t = fast_div(r, rows_magic), h = r - t * each;
    const int64_t token = t0 + t;
    const bool is_q = h < p.heads, is_v = kCache && h >= p.heads + p.kv_heads;
    const int kh = is_v ? h - p.heads - p.kv_heads : h - p.heads;
    const T* x = is_q ? static_cast<const T*>(p.q) + token * p.ldq + h * p.ldqh
               : is_v ? static_cast<const T*>(p.v) + token * p.ldv + kh * p.ldvh
                      : static_cast<const T*>(p.k) + token * p.ldk + kh * p.ldkh;
    float a[kC], b[kC];
    int ia[kC], ib[kC];
    float ss = 0.0f;
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      const int i = lane + c * 32;
      const bool between = !p.interleaved && i < half;
      ia[c] = between ? i : 2 * i;
      ib[c] = between ? i + half : 2 * i + 1;
      a[c] = b[c] = 0.0f;
      if (2 * i < p.dim) {
        a[c] = to_f32(x[ia[c]]);
        b[c] = to_f32(x[ib[c]]);
      } else {
        ia[c] = -1;
      }
      ss = fmaf(a[c], a[c], fmaf(b[c], b[c], ss));
    }
    const void* w = is_v ? nullptr : is_q ? p.q_weight : p.k_weight;
    if (w) {
      for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      float mean = ss / (float)p.dim + p.eps;
      if (off_range(mean)) {  // (every lane has the same sum)
        float top = 0.0f;
#pragma unroll
        for (int c = 0; c < kC; ++c) top = fmaxf(top, fmaxf(fabsf(a[c]), fabsf(b[c])));
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float s = into_range(mean, top);
        ss = 0.0f;
#pragma unroll
        for (int c = 0; c < kC; ++c) {
          a[c] *= s;
          b[c] *= s;
          ss = fmaf(a[c], a[c], fmaf(b[c], b[c], ss));
        }
        for (int o = 16; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        mean = ss / (float)p.dim + p.eps * s * s;
      }
      const float rms = rsqrtf(mean);
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        if (ia[c] < 0) continue;
        float wa[1], wb[1];
        load_weight<1>(w, ia[c], p.weight_dtype, wa);
        load_weight<1>(w, ib[c], p.weight_dtype, wb);
        a[c] = a[c] * rms * wa[0];
        b[c] = b[c] * rms * wb[0];
      }
    }
    if (!is_v) {
      T* y = is_q ? static_cast<T*>(p.q_out) + token * p.ldqo + h * p.ldqoh
                  : (p.k_out ? static_cast<T*>(p.k_out) + token * p.ldko + kh * p.ldkoh : nullptr);
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        if (ia[c] < 0) continue;
        const int f = lane + c * 32;
        if (f < half) {
          const float2 cs = turns[t * half + f];
          const float u = a[c], v = b[c];
          a[c] = u * cs.x - v * cs.y;
          b[c] = v * cs.x + u * cs.y;
        }
        if (y) {
          y[ia[c]] = from_f32<T>(a[c]);
          y[ib[c]] = from_f32<T>(b[c]);
        }
      }
    }
    if constexpr (kCache) {
      if (is_q) continue;
      float lo = INFINITY, hi = -INFINITY;
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        if (ia[c] < 0) continue;
        a[c] = to_f32(from_f32<T>(a[c]));  // codes are of the rounded values, whether these are stored or not
        b[c] = to_f32(from_f32<T>(b[c]));
        lo = min_nan(lo, min_nan(a[c], b[c]));
        hi = max_nan(hi, max_nan(a[c], b[c]));
      }
      for (int o = 16; o > 0; o >>= 1) {
        lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
      }
      const int64_t slot = p.slots[token];
      if (!in_cache(p.cache, slot)) continue;
      const RowStep rs(lo, hi);
      int row;
      uint8_t* blk = place(p.cache, slot, kh, row);
      if (lane == 0) *reinterpret_cast<uint32_t*>(blk + 16 * p.dim + (is_v ? 64 : 0) + 4 * row) = rs.word;
      // codes meet their neighbours in shared memory
      uint8_t* line = bytes + (threadIdx.x >> 5) * 256;
      __syncwarp();
#pragma unroll
      for (int c = 0; c < kC; ++c) {
        if (ia[c] < 0) continue;
        line[ia[c]] = (uint8_t)rs.code(a[c]);
        line[ib[c]] = (uint8_t)rs.code(b[c]);
      }
      __syncwarp();
      if (lane * 8 < p.dim) {
        uint32_t w8 = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) w8 |= (uint32_t)line[lane * 8 + j] << (4 * j);
        *reinterpret_cast<uint32_t*>(blk + (is_v ? 8 * p.dim : 0) + row * (p.dim >> 1) + 4 * lane) = w8;
      }
    }
  }
}

// ---------------------------------------------------------------- rows at 16-byte addresses

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

// 16 bytes of a row as pairs of float32, and back
template <class T> __device__ __forceinline__ void to_pairs(const uint4& v, uint64_t (&x)[8 / sizeof(T)]);
template <> __device__ __forceinline__ void to_pairs<float>(const uint4& v, uint64_t (&x)[2]) {
  x[0] = two_of(__uint_as_float(v.x), __uint_as_float(v.y));
  x[1] = two_of(__uint_as_float(v.z), __uint_as_float(v.w));
}
__device__ __forceinline__ uint64_t half_pair(uint32_t w) {
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
  return two_of(f.x, f.y);
}
__device__ __forceinline__ uint64_t bfloat_pair(uint32_t w) { return two_of(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
template <> __device__ __forceinline__ void to_pairs<__half>(const uint4& v, uint64_t (&x)[4]) {
  x[0] = half_pair(v.x); x[1] = half_pair(v.y); x[2] = half_pair(v.z); x[3] = half_pair(v.w);
}
template <> __device__ __forceinline__ void to_pairs<__nv_bfloat16>(const uint4& v, uint64_t (&x)[4]) {
  x[0] = bfloat_pair(v.x); x[1] = bfloat_pair(v.y); x[2] = bfloat_pair(v.z); x[3] = bfloat_pair(v.w);
}
template <class T> __device__ __forceinline__ uint32_t word_of(uint64_t p);
template <> __device__ __forceinline__ uint32_t word_of<__half>(uint64_t p) {
  float a, b;
  one_each(p, a, b);
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t word_of<__nv_bfloat16>(uint64_t p) {
  float a, b;
  one_each(p, a, b);
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <class T>
__device__ __forceinline__ uint4 from_pairs(const uint64_t (&x)[8 / sizeof(T)]) {
  if constexpr (sizeof(T) == 4) {
    float a, b, c, d;
    one_each(x[0], a, b);
    one_each(x[1], c, d);
    return make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
  } else {
    return make_uint4(word_of<T>(x[0]), word_of<T>(x[1]), word_of<T>(x[2]), word_of<T>(x[3]));
  }
}

// Lowest and highest value of a row, of which each of `lanes` lanes has two vectors; a NaN wins.
template <class T>
__device__ __forceinline__ void extremes(const uint4& a, const uint4& b, int lanes, bool in, float& lo, float& hi) {
  if constexpr (sizeof(T) == 4) {
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    lo = in ? __uint_as_float(w[0]) : INFINITY;
    hi = in ? __uint_as_float(w[0]) : -INFINITY;
    if (in) {
#pragma unroll
      for (int i = 1; i < 8; ++i) {
        lo = min_nan(lo, __uint_as_float(w[i]));
        hi = max_nan(hi, __uint_as_float(w[i]));
      }
    }
    for (int o = lanes >> 1; o > 0; o >>= 1) {
      lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
  } else {
    using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
    auto as2 = [](uint32_t w) { return *reinterpret_cast<T2*>(&w); };
    auto bits = [](T2 h) { return *reinterpret_cast<uint32_t*>(&h); };
    const T2 l2 = __hmin2_nan(__hmin2_nan(__hmin2_nan(as2(a.x), as2(a.y)), __hmin2_nan(as2(a.z), as2(a.w))),
                              __hmin2_nan(__hmin2_nan(as2(b.x), as2(b.y)), __hmin2_nan(as2(b.z), as2(b.w))));
    const T2 h2 = __hmax2_nan(__hmax2_nan(__hmax2_nan(as2(a.x), as2(a.y)), __hmax2_nan(as2(a.z), as2(a.w))),
                              __hmax2_nan(__hmax2_nan(as2(b.x), as2(b.y)), __hmax2_nan(as2(b.z), as2(b.w))));
    // the lowest in the low half, the highest with its sign turned in the high half: one minimum for both
    const uint32_t lw = bits(l2), hw = bits(h2);
    T2 both = __hmin2_nan(as2(__byte_perm(lw, hw, 0x5410) ^ 0x80000000u), as2(__byte_perm(lw, hw, 0x7632) ^ 0x80000000u));
    constexpr uint32_t inf = std::is_same<T, __half>::value ? 0x7c007c00u : 0x7f807f80u;
    if (!in) both = as2(inf);
    for (int o = lanes >> 1; o > 0; o >>= 1) both = __hmin2_nan(both, as2(__shfl_xor_sync(0xffffffffu, bits(both), o)));
    lo = to_f32(both.x);
    hi = -to_f32(both.y);
  }
}

// Codes of the kN values of 16 bytes, the first in the lowest bits.
template <class T>
__device__ __forceinline__ uint32_t codes_of(const RowStep& rs, const uint4& v) {
  constexpr int kPairs = 8 / sizeof(T);
  uint64_t x[kPairs];
  to_pairs<T>(v, x);
  const uint64_t low = two_of(-rs.low, -rs.low), inv = two_of(rs.inv, rs.inv), magic = two_of(12582912.0f, 12582912.0f), step = two_of(-rs.step, -rs.step);
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < kPairs; ++i) {
    const uint64_t d = add2(x[i], low), q = mul2(d, inv), t = add2(fma2(fma2(q, step, d), inv, q), magic);
    float ta, tb;
    one_each(t, ta, tb);
    w += __float_as_uint(ta) * (1u << (8 * i)) + __float_as_uint(tb) * (16u << (8 * i));  // (what is not the code adds up to a constant)
  }
  constexpr uint32_t kRest = 0x4b400000u + (0x4b400000u << 4) + (0x4b400000u << 8);
  return rs.inv > 0.0f ? w - kRest : 0u;
}

template <bool k>
struct Bool {
  static constexpr bool value = k;
};

// A warp, or several, to a token: the lanes of a row keep their places in it while the warp goes through the heads. lanes: a power of two, those past the
// row's end idle. `share` warps (1, 2 or 4) take a token's rows in turn. kPlain: keys and values to the cache as they are.
template <class T, bool kCache, bool kInter, bool kPlain>
__global__ void __launch_bounds__(kThreads, kPlain ? 8 : 5) rows_kernel(const QkArgs p, const int share, const int lanes, const int lanes_log2) {
  constexpr int V = 16 / sizeof(T), kPairs = V / 2;
  extern __shared__ float2 turns[];  // [tokens of the block][rot / 2]: cosine, sine
  tc::grid_dep_wait();
  const int per = kThreads / 32 / share, warp = threadIdx.x >> 5, half = p.rot >> 1;
  const int64_t t0 = (int64_t)blockIdx.x * per;
  const int here = (int)(p.tokens - t0 < per ? p.tokens - t0 : per);
  const int t = warp / share;
  const int64_t token = t0 + (t < here ? t : 0);
  const int lane = threadIdx.x & (lanes - 1), group = (threadIdx.x & 31) >> lanes_log2, groups = 32 >> lanes_log2;
  const int first = (warp % share) * groups, step = share * groups;
  // this lane's two vectors
  const bool in = 2 * lane * V < p.dim, between = !kInter && lane * V < half;  // (pairs between the two)
  // (with no pairs to keep, adjacent vectors are in adjacent lanes all the same: an access takes whole sectors)
  const int ia = kPlain || between ? lane * V : 2 * lane * V, ib = kPlain ? ia + (p.dim >> 1) : between ? ia + half : ia + V;
  const bool turn_a = kInter ? ia < p.rot : between, turn_b = kInter ? ib < p.rot : between;
  const int64_t slot = kCache ? p.slots[token] : -1;
  const bool kept = kCache && in_cache(p.cache, slot);
  int row = 0;
  uint8_t* blk = kept ? place(p.cache, slot, 0, row) : nullptr;
  const int64_t head_bytes = ((int64_t)1 << (p.cache.page_shift - 4)) * 16 * (p.cache.dim + 8);
  // rows to come begin their way, a lane to a line of 128 bytes; the first ones while sines and cosines are made
  auto begin = [&](const T* x, int64_t ldh, int h0, int n, int count) {
    if (lane * (int)(128 / sizeof(T)) < p.dim) {
#pragma unroll
      for (int k = 0; k < count; ++k)
        if (h0 + group + k * step < n) prefetch(x + (h0 + group + k * step) * ldh + lane * (int)(128 / sizeof(T)));
    }
  };
  if constexpr (!kPlain) {
    begin(static_cast<const T*>(p.q) + token * p.ldq, p.ldqh, first, p.heads, kCache ? 1 : 2);
    begin(static_cast<const T*>(p.k) + token * p.ldk, p.ldkh, first, p.kv_heads, kCache ? 1 : 2);
  }
  if constexpr (!kPlain) {
    if (half > 0) {
      // a thread keeps to one frequency, where there are as many threads
      const int wide = half < kThreads ? half : kThreads, f0 = threadIdx.x % wide, each = kThreads / wide;
      for (int f = f0; f < half; f += wide) {
        const uint64_t rate = turn_rate(p.inv_freq[f]);
        for (int s = threadIdx.x / wide; s < here && (int)threadIdx.x < wide * each; s += each) turns[s * half + f] = turn_of(rate, p.positions[t0 + s]);
      }
    }
    __syncthreads();
  }
  if (t >= here) return;

  auto to_cache = [&](int head, bool live, bool values, const uint4& a, const uint4& b) {
    float lo, hi;
    extremes<T>(a, b, lanes, in, lo, hi);
    if (!kept || !live) return;
    const RowStep rs(lo, hi);
    uint8_t* y = blk + head * head_bytes;
    if (lane == 0) *reinterpret_cast<uint32_t*>(y + 16 * p.dim + (values ? 64 : 0) + 4 * row) = rs.word;
    if (!in) return;
    y += (values ? 8 * p.dim : 0) + row * (p.dim >> 1);
    const uint32_t wa = codes_of<T>(rs, a), wb = codes_of<T>(rs, b);
    if constexpr (V == 8) {
      *reinterpret_cast<uint32_t*>(y + (ia >> 1)) = wa;
      *reinterpret_cast<uint32_t*>(y + (ib >> 1)) = wb;
    } else {
      *reinterpret_cast<uint16_t*>(y + (ia >> 1)) = (uint16_t)wa;
      *reinterpret_cast<uint16_t*>(y + (ib >> 1)) = (uint16_t)wb;
    }
  };
  // two rows' vectors at once: their loads are on the way together
  auto fetch = [&](auto& a, auto& b, const T* x, int64_t ldh, int h, int n) {
#pragma unroll
    for (int k = 0; k < (int)(sizeof(a) / sizeof(uint4)); ++k) {
      a[k] = b[k] = make_uint4(0, 0, 0, 0);
      if (in && h + k * step < n) {
        const T* y = x + (int64_t)(h + k * step) * ldh;
        a[k] = *reinterpret_cast<const uint4*>(y + ia);
        b[k] = *reinterpret_cast<const uint4*>(y + ib);
      }
    }
  };
  const float per_value = 1.0f / (float)p.dim;
  // rows of queries or keys: norm, turn, out, and keys to the cache
  auto run = [&](auto cached, const T* x, int64_t ldh, int n, const void* weight, T* y, int64_t ldyh) {
    constexpr bool kCached = decltype(cached)::value;
    // out = in * own + partner * other, and times 1 / rms at the end
    uint64_t own_a[kPairs], own_b[kPairs], other_a[kPairs], other_b[kPairs];
    const bool plain = kPlain || (!weight && half == 0);
    if (!plain && in) {
      float wa[V], wb[V];
#pragma unroll
      for (int j = 0; j < V; ++j) wa[j] = wb[j] = 1.0f;
      if (weight) {
        load_weight<V>(weight, ia, p.weight_dtype, wa);
        load_weight<V>(weight, ib, p.weight_dtype, wb);
      }
      const float2* tt = turns + t * half;
#pragma unroll
      for (int j = 0; j < V; j += 2) {
        float2 c0 = make_float2(1.0f, 0.0f), c1 = c0, d0 = c0, d1 = c0;
        if constexpr (kInter) {
          if (turn_a) c0 = c1 = tt[(ia + j) >> 1];
          if (turn_b) d0 = d1 = tt[(ib + j) >> 1];
          other_a[j / 2] = two_of(-wa[j + 1] * c0.y, wa[j] * c0.y);
          other_b[j / 2] = two_of(-wb[j + 1] * d0.y, wb[j] * d0.y);
        } else {
          if (between) {
            c0 = d0 = tt[ia + j];
            c1 = d1 = tt[ia + j + 1];
          }
          other_a[j / 2] = two_of(-wb[j] * c0.y, -wb[j + 1] * c1.y);
          other_b[j / 2] = two_of(wa[j] * c0.y, wa[j + 1] * c1.y);
        }
        own_a[j / 2] = two_of(wa[j] * c0.x, wa[j + 1] * c1.x);
        own_b[j / 2] = two_of(wb[j] * d0.x, wb[j + 1] * d1.x);
      }
    }
    constexpr int kAtOnce = kCached && !kPlain ? 1 : 2;  // (with the codes' numbers, two rows would not fit the registers of five blocks an SM)
    for (int h0 = first; h0 < n; h0 += kAtOnce * step) {
      uint4 va[kAtOnce], vb[kAtOnce];
      fetch(va, vb, x, ldh, h0 + group, n);
      if constexpr (!kPlain) begin(x, ldh, h0 + kAtOnce * step, n, kAtOnce);
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        if (h0 + k * step >= n) break;
        const int h = h0 + group + k * step;
        uint4 a = va[k], b = vb[k];
        if (!plain) {
          uint64_t u[kPairs], v[kPairs];
          to_pairs<T>(a, u);
          to_pairs<T>(b, v);
          uint64_t f = two_of(1.0f, 1.0f);
          if (weight) {
            auto squares = [&] {
              uint64_t s0 = 0, s1 = 0;
#pragma unroll
              for (int i = 0; i < kPairs; ++i) {
                s0 = fma2(u[i], u[i], s0);
                s1 = fma2(v[i], v[i], s1);
              }
              float ss, s2;
              one_each(add2(s0, s1), ss, s2);
              ss += s2;
              for (int o = lanes >> 1; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
              return ss;
            };
            const float mean = fmaf(squares(), per_value, p.eps);
            float rms = root(mean);
            if (__any_sync(0xffffffffu, off_range(mean))) {
              float top = 0.0f;
#pragma unroll
              for (int i = 0; i < kPairs; ++i) {
                float c, d;
                one_each(u[i], c, d);
                top = fmaxf(top, fmaxf(fabsf(c), fabsf(d)));
                one_each(v[i], c, d);
                top = fmaxf(top, fmaxf(fabsf(c), fabsf(d)));
              }
              for (int o = lanes >> 1; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
              const float s = into_range(mean, top);  // (1 for the other rows of the warp: theirs come out as before)
              const uint64_t by = two_of(s, s);
#pragma unroll
              for (int i = 0; i < kPairs; ++i) {
                u[i] = mul2(u[i], by);
                v[i] = mul2(v[i], by);
              }
              rms = rsqrtf(fmaf(squares(), per_value, p.eps * s * s));
            }
            f = two_of(rms, rms);
          }
          uint64_t ya[kPairs], yb[kPairs];
#pragma unroll
          for (int i = 0; i < kPairs; ++i) {
            ya[i] = mul2(u[i], own_a[i]);
            yb[i] = mul2(v[i], own_b[i]);
            // (a place that does not turn has no partner, whose infinity would reach it)
            if constexpr (kInter) {
              float c, d;
              one_each(u[i], c, d);
              if (turn_a) ya[i] = fma2(two_of(d, c), other_a[i], ya[i]);
              one_each(v[i], c, d);
              if (turn_b) yb[i] = fma2(two_of(d, c), other_b[i], yb[i]);
            } else if (between) {
              ya[i] = fma2(v[i], other_a[i], ya[i]);
              yb[i] = fma2(u[i], other_b[i], yb[i]);
            }
            ya[i] = mul2(ya[i], f);
            yb[i] = mul2(yb[i], f);
          }
          a = from_pairs<T>(ya);
          b = from_pairs<T>(yb);
        }
        if (y && in && h < n) {
          T* z = y + (int64_t)h * ldyh;
          *reinterpret_cast<uint4*>(z + ia) = a;
          *reinterpret_cast<uint4*>(z + ib) = b;
        }
        if constexpr (kCached) to_cache(h, h < n, false, a, b);  // codes are of the rounded values, whether these are stored or not
      }
    }
  };
  if (!kPlain && p.heads > 0) run(Bool<false>(), static_cast<const T*>(p.q) + token * p.ldq, p.ldqh, p.heads, p.q_weight, static_cast<T*>(p.q_out) + token * p.ldqo, p.ldqoh);
  run(Bool<kCache>(), static_cast<const T*>(p.k) + token * p.ldk, p.ldkh, p.kv_heads, p.k_weight, p.k_out ? static_cast<T*>(p.k_out) + token * p.ldko : nullptr, p.ldkoh);
  if constexpr (kCache) {
    const T* x = static_cast<const T*>(p.v) + token * p.ldv;
    for (int h0 = first; h0 < p.kv_heads; h0 += 2 * step) {
      uint4 a[2], b[2];
      fetch(a, b, x, p.ldvh, h0 + group, p.kv_heads);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (h0 + k * step >= p.kv_heads) break;
        const int h = h0 + group + k * step;
        to_cache(h, h < p.kv_heads, true, a[k], b[k]);
      }
    }
  }
}

// `share` warps to a token, as above; a lane takes two words of 8 codes of a row, half a row apart (its values' stores are whole sectors with its neighbours':
// 16,384 tokens of 8 heads of 128 back to bfloat16 in 13.8 us, 19 with 16 codes together), `lanes` lanes a row, keys' rows and then values'.
template <class T, bool kVec>
__global__ void __launch_bounds__(kThreads) cache_read_kernel(const CacheReadArgs p, const int share, const int lanes, const int lanes_log2) {
  tc::grid_dep_wait();
  const CacheGeom& c = p.cache;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & (lanes - 1), groups = 32 >> lanes_log2, wide = c.dim >> 4;
  const int64_t token = ((int64_t)blockIdx.x * (kThreads / 32) + warp) / share;
  if (token >= p.tokens || lane >= wide) return;
  const int64_t slot = p.slots[token], head_bytes = ((int64_t)1 << (c.page_shift - 4)) * 16 * (c.dim + 8);
  int row = 0;
  const uint8_t* blk = in_cache(c, slot) ? place(c, slot, 0, row) : nullptr;
  const int step = share * groups;
  for (int r0 = (warp % share) * groups + ((threadIdx.x & 31) >> lanes_log2); r0 < 2 * c.kv_heads; r0 += 4 * step) {
    // four rows' loads on the way together
    uint2 words[4];
    uint32_t steps[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int r = r0 + k * step;
      const bool is_v = r >= c.kv_heads;
      words[k] = make_uint2(0, 0);
      steps[k] = 0;
      if (blk && r < 2 * c.kv_heads) {
        const uint8_t* x = blk + (is_v ? r - c.kv_heads : r) * head_bytes;
        const uint32_t* w = reinterpret_cast<const uint32_t*>(x + (is_v ? 8 * c.dim : 0) + row * (c.dim >> 1)) + lane;
        words[k] = make_uint2(w[0], w[wide]);
        steps[k] = *reinterpret_cast<const uint32_t*>(x + 16 * c.dim + (is_v ? 64 : 0) + 4 * row);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int r = r0 + k * step;
      const bool is_v = r >= c.kv_heads;
      T* y = is_v ? static_cast<T*>(p.v) : static_cast<T*>(p.k);
      if (r >= 2 * c.kv_heads || !y) continue;
      y += token * (is_v ? p.ldv : p.ldk) + (is_v ? r - c.kv_heads : r) * (is_v ? p.ldvh : p.ldkh) + lane * 8;
      const float low = __uint_as_float(steps[k] << 16), size = __uint_as_float(steps[k] & 0xffff0000u);
      const uint64_t low2 = two_of(low, low), step2 = two_of(size, size), less = two_of(-8388608.0f, -8388608.0f);
#pragma unroll
      for (int h = 0; h < 2; ++h, y += c.dim >> 1) {
        const uint32_t w = h ? words[k].y : words[k].x;
        uint64_t f[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {  // (a code under the exponent of 2^23 is 2^23 + n)
          const uint32_t u = w >> (8 * j);
          f[j] = fma2(add2(two_of(__uint_as_float((u & 15u) | 0x4b000000u), __uint_as_float((u >> 4 & 15u) | 0x4b000000u)), less), step2, low2);
        }
        if constexpr (kVec) {
          constexpr int kPairs = 8 / sizeof(T);
#pragma unroll
          for (int i = 0; i < 4; i += kPairs) {
            uint64_t v[kPairs];
#pragma unroll
            for (int e = 0; e < kPairs; ++e) v[e] = f[i + e];
            *reinterpret_cast<uint4*>(y + 2 * i) = from_pairs<T>(v);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float a, b;
            one_each(f[j], a, b);
            y[2 * j] = from_f32<T>(a);
            y[2 * j + 1] = from_f32<T>(b);
          }
        }
      }
    }
  }
}

static bool on16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
static int pow2_at_least(int n) {
  int v = 1;
  while (v < n) v *= 2;
  return v;
}

static void config(cudaLaunchConfig_t& cfg, cudaLaunchAttribute* at, int64_t blocks, size_t smem, cudaStream_t stream) {
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
}
// Warps to a token: more while all of them are on the GPU at once (`blocks` an SM) and have rows for their groups of lanes. (40 heads of 128 and a cache, us with
// one, two and four warps a token: 512 tokens 9.1, 7.1, 6.9; 1024 tokens 10.4, 8.7, 11.8; 2048 tokens 12.9, 14.4, 17.6; 4096 tokens 24.4, 25.1, 34.4.)
static int share_of(int64_t tokens, int rows, int groups, int blocks) {
  int share = 1;
  while (share < kThreads / 32 && 2 * share * tokens <= 152 * (kThreads / 32) * blocks && share * groups < rows) share *= 2;
  return share;
}

template <class T>
static cudaError_t run_heads_type(const QkArgs& a, cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  bool vec = a.dim % (2 * V) == 0 && a.dim / (2 * V) <= 32 && (a.interleaved ? a.rot % V == 0 : a.rot % (2 * V) == 0);
  if (a.heads > 0) vec = vec && on16(a.q) && on16(a.q_out) && (a.ldq | a.ldqh | a.ldqo | a.ldqoh) % V == 0;
  vec = vec && on16(a.k) && (a.ldk | a.ldkh) % V == 0 && on16(a.q_weight) && on16(a.k_weight);
  if (a.k_out) vec = vec && on16(a.k_out) && (a.ldko | a.ldkoh) % V == 0;
  if (a.cache.data) vec = vec && on16(a.v) && (a.ldv | a.ldvh) % V == 0;
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute at[1];
  if (vec) {
    const int lanes = pow2_at_least(a.dim / (2 * V)), log2 = __builtin_ctz(lanes);
    const bool plain = a.cache.data && a.heads == 0 && !a.k_weight && a.rot == 0 && !a.k_out;
    const int blocks = plain ? 8 : 5;  // an SM, as the kernels are built for
    const int share = share_of(a.tokens, a.heads > a.kv_heads ? a.heads : a.kv_heads, 32 / lanes, blocks), per = kThreads / 32 / share;
    config(cfg, at, (a.tokens + per - 1) / per, (size_t)per * (a.rot / 2) * sizeof(float2), stream);
    if (plain) return cudaLaunchKernelEx(&cfg, rows_kernel<T, true, false, true>, a, share, lanes, log2);
    if (a.cache.data)
      return a.interleaved ? cudaLaunchKernelEx(&cfg, rows_kernel<T, true, true, false>, a, share, lanes, log2)
                           : cudaLaunchKernelEx(&cfg, rows_kernel<T, true, false, false>, a, share, lanes, log2);
    return a.interleaved ? cudaLaunchKernelEx(&cfg, rows_kernel<T, false, true, false>, a, share, lanes, log2)
                         : cudaLaunchKernelEx(&cfg, rows_kernel<T, false, false, false>, a, share, lanes, log2);
  }
  // a block's tokens: one while that leaves SMs without a block, else enough for four rows a warp, as far as their cosines and sines fit in 32 KB
  const int each = a.heads + a.kv_heads * (a.cache.data ? 2 : 1);
  int per = 1;
  while (per * 2 * each <= 32 && a.tokens / (per * 2) >= 4 * 152 && per * 2 * (a.rot / 2) * sizeof(float2) <= 32768) per *= 2;
  config(cfg, at, (a.tokens + per - 1) / per, (size_t)per * (a.rot / 2) * sizeof(float2), stream);
  if (a.cache.data) return cudaLaunchKernelEx(&cfg, heads_kernel<T, true>, a, per, div_magic(each));
  return cudaLaunchKernelEx(&cfg, heads_kernel<T, false>, a, per, div_magic(each));
}

template <class T>
static cudaError_t run_read(const CacheReadArgs& a, cudaStream_t stream) {
  constexpr int V = 16 / sizeof(T);
  const bool vec = on16(a.k) && on16(a.v) && (a.ldk | a.ldkh | a.ldv | a.ldvh) % V == 0;
  const int lanes = pow2_at_least(a.cache.dim / 16), log2 = __builtin_ctz(lanes);
  const int share = share_of(a.tokens, 2 * a.cache.kv_heads, 32 / lanes, 5);
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute at[1];
  config(cfg, at, (a.tokens * share + kThreads / 32 - 1) / (kThreads / 32), 0, stream);
  if (vec) return cudaLaunchKernelEx(&cfg, cache_read_kernel<T, true>, a, share, lanes, log2);
  return cudaLaunchKernelEx(&cfg, cache_read_kernel<T, false>, a, share, lanes, log2);
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
