// lm_prompt.cu -- attention over whole sequences packed one after another, causal or not, with grouped heads.
//
// One pass over the keys with a running maximum m and sum l of each row: with m' = max(m, max_t s_t), o' = o 2^(c (m - m')) +
// sum_t 2^(c (s_t - m')) v_t and l' likewise, c = scale log2(e). Scores and weights stay in registers: the
// accumulator of one product has the layout of the next one's first operand.
//
// This kernel takes 64 query rows of one head, four warps of 16, and keys in tiles of 64 (or 32) through two stages of shared memory. It serves what the
// tensor-memory kernels do not: strides of zero, which no tensor map holds, and more jobs than a grid's second axis. Bound by mma.sync, whose rate is a
// fraction of theirs: 8192 tokens of 32 heads of 192 3,730 us (221 TFLOP/s; 511 there), of 256 4,193 (262; 639). Prompts of less than
// a tile's 128 rows come near: 100 of 64 tokens, 32 heads of 256, 112 us (99 there).
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "../../include/aqd.h"
#include "common.cuh"
#include "kernels.h"
#include "lm_prompt.cuh"
#include "tc_ptx.cuh"

namespace aqd {
namespace prompt {

using namespace tc;

constexpr int kWarps = 4, kThreads = kWarps * 32, kRows = 64;
// keys of a tile: 64 of a head's 256 values would spill
__host__ __device__ constexpr int keys_of(int dim) { return dim == 256 ? 32 : 64; }
template <class T>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (std::is_same<T, __half>::value)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// 16 bytes `c` of row r of a tile of D 16-bit values a row: chunks of 128 bytes swap their 16-byte parts by the row
template <int D>
__device__ __forceinline__ uint32_t at(uint32_t base, int r, int c) {
  return base + r * (D * 2) + ((c & ~7) | ((c ^ r) & 7)) * 16;
}

// The rows of a warp, from row `first` on, that a hidden value reached. (A call, with copies: heads of 256 have no registers left for it.)
template <class T, int D>
static __device__ __noinline__ void take_rows_again(const PromptArgs p, const Job jb, int head, int first) {
  const int end = first + 16 < jb.queries ? first + 16 : jb.queries, seen = seen_by(jb, (jb.tile + 1) * kRows - 1 < jb.queries ? (jb.tile + 1) * kRows - 1 : jb.queries - 1);
  const int keys = (seen + keys_of(D) - 1) / keys_of(D) * keys_of(D);  // that the block's products took
  const T* v = static_cast<const T*>(p.v) + (int64_t)jb.kv_start * p.ldv + (int64_t)(head / (p.heads / p.kv_heads)) * p.ldvh;
  const int last = last_not_finite<T, D>(seen_by(jb, first), keys < jb.keys ? keys : jb.keys, [&](int t, int i) { return reinterpret_cast<const uint4*>(v + t * p.ldv)[i]; });
  __syncwarp();  // (the rows' first outputs come before)
  for (int at = first; at < end && seen_by(jb, at) <= last; ++at) attend_again<T, D>(p, jb, head, at);
}
// (Blocks an SM: heads of 64 three, 4096 tokens of 8 heads 94 us, 111 with four and 122 with five; of 128 two by shared memory, three by registers would spill.)
template <class T, int D>
__global__ void __launch_bounds__(kThreads, D == 64 ? 3 : D == 128 ? 2 : 0) prompt_kernel(const __grid_constant__ PromptArgs p) {
  constexpr int kKeys = keys_of(D), kTile = kKeys * D * 2, kChunks = D / 8;
  extern __shared__ __align__(128) uint8_t smem[];  // queries, two stages of keys and values
  __shared__ Job job;
  __shared__ uint64_t red[kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  grid_dep_wait();
  if (!find_job(p, kRows, blockIdx.x, &job, red)) return;
  const Job jb = job;
  const int head = blockIdx.y, kvh = head / (p.heads / p.kv_heads);
  const uint32_t sq = smem_u32(smem), sk = sq + kRows * D * 2;
  const int row0 = jb.tile * kRows, shift = jb.keys - jb.queries;  // row r sees keys 0 .. r + shift
  const T* q = static_cast<const T*>(p.q) + (int64_t)(jb.start + row0) * p.ldq + (int64_t)head * p.ldqh;
  const T* k = static_cast<const T*>(p.k) + (int64_t)jb.kv_start * p.ldk + (int64_t)kvh * p.ldkh;
  const T* v = static_cast<const T*>(p.v) + (int64_t)jb.kv_start * p.ldv + (int64_t)kvh * p.ldvh;
  const int rows = jb.queries - row0 < kRows ? jb.queries - row0 : kRows;
  int64_t see = p.causal ? (int64_t)row0 + rows + shift : jb.keys;
  see = see < 0 ? 0 : see > jb.keys ? jb.keys : see;
  const int tiles = (int)((see + kKeys - 1) / kKeys);

  auto load_tile = [&](uint32_t dst, const T* src, int64_t ld, int first, int end, int n) {
    for (int i = threadIdx.x; i < n * kChunks; i += kThreads) {
      const int r = i / kChunks, c = i - r * kChunks;
      const bool in = first + r < end;
      cp_async<16>(at<D>(dst, r, c), src + (in ? (int64_t)(first + r) * ld + c * 8 : 0), in);
    }
  };
  load_tile(sq, q, p.ldq, 0, rows, kRows);
  if (tiles > 0) load_tile(sk, k, p.ldk, 0, jb.keys, kKeys);
  cp_async_commit();
  if (tiles > 0) load_tile(sk + kTile, v, p.ldv, 0, jb.keys, kKeys);
  cp_async_commit();

  float o[D / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < D / 8; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c) o[i][c] = 0.0f;
  const float c2 = factor(p.scale);
  const int r0 = row0 + warp * 16 + (lane >> 2);  // this lane's rows: r0 and r0 + 8
  for (int t = 0; t < tiles; ++t) {
    const uint32_t kt = sk + (t & 1) * 2 * kTile, vt = kt + kTile;
    cp_async_wait<1>();
    __syncthreads();  // keys are there; the other stage's readers are through
    if (t + 1 < tiles) {
      const uint32_t next = sk + ((t + 1) & 1) * 2 * kTile;
      load_tile(next, k, p.ldk, (t + 1) * kKeys, jb.keys, kKeys);
      cp_async_commit();
      load_tile(next + kTile, v, p.ldv, (t + 1) * kKeys, jb.keys, kKeys);
      cp_async_commit();
    } else {
      cp_async_commit();
      cp_async_commit();
    }
    float s[kKeys / 8][4];
#pragma unroll
    for (int i = 0; i < kKeys / 8; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) s[i][c] = 0.0f;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      uint32_t a[4];
      ldsm(a, at<D>(sq, warp * 16 + (lane & 15), kk * 2 + (lane >> 4)));
#pragma unroll
      for (int n = 0; n < kKeys / 16; ++n) {
        uint32_t b[4];
        ldsm(b, at<D>(kt, n * 16 + (lane & 7) + (lane >> 4) * 8, kk * 2 + ((lane >> 3) & 1)));
        mma<T>(s[2 * n], a, b[0], b[1]);
        mma<T>(s[2 * n + 1], a, b[2], b[3]);
      }
    }
    // places that a row does not see
    if ((t + 1) * kKeys > jb.keys || (p.causal && (t + 1) * kKeys > row0 + shift + 1)) {
#pragma unroll
      for (int n = 0; n < kKeys / 8; ++n)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int key = t * kKeys + n * 8 + (lane & 3) * 2 + (c & 1), row = r0 + (c >> 1) * 8;
          if (key >= jb.keys || (p.causal && key > row + shift)) s[n][c] = -INFINITY;
        }
    }
    uint32_t pw[kKeys / 8][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float top = -INFINITY;
#pragma unroll
      for (int n = 0; n < kKeys / 8; ++n) top = fmaxf(top, fmaxf(s[n][2 * h], s[n][2 * h + 1]));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      top = fmaxf(m[h], top);
      const float ref = top == -INFINITY ? 0.0f : top, f = ex2((m[h] - ref) * c2);
      m[h] = top;
      l[h] *= f;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) { o[i][2 * h] *= f; o[i][2 * h + 1] *= f; }
#pragma unroll
      for (int n = 0; n < kKeys / 8; ++n) {
        const float a = ex2((s[n][2 * h] - ref) * c2), b = ex2((s[n][2 * h + 1] - ref) * c2);
        l[h] += a + b;
        pw[n][h] = pack(a, b, (T*)nullptr);
      }
    }
    cp_async_wait<2>();
    __syncthreads();  // values are there
#pragma unroll
    for (int n = 0; n < kKeys / 16; ++n) {
      const uint32_t a[4] = {pw[2 * n][0], pw[2 * n][1], pw[2 * n + 1][0], pw[2 * n + 1][1]};
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        uint32_t b[4];
        ldsm_t(b, at<D>(vt, n * 16 + (lane & 15), i * 2 + (lane >> 4)));
        mma<T>(o[2 * i], a, b[0], b[1]);
        mma<T>(o[2 * i + 1], a, b[2], b[3]);
      }
    }
  }
  cp_async_wait<0>();
  float zero = 0.0f;  // (a sum of outputs times 0: NaN where one is not finite)
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
    const int r = warp * 16 + (lane >> 2) + 8 * h;
    if (r >= rows) continue;
    const float inv = m[h] == -INFINITY && l[h] == 0.0f ? 0.0f : 1.0f / l[h];
    const int64_t token = jb.start + row0 + r;
    T* y = static_cast<T*>(p.out) + token * p.ldo + (int64_t)head * p.ldoh + (lane & 3) * 2;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) {
      *reinterpret_cast<uint32_t*>(y + 8 * i) = pack(o[i][2 * h] * inv, o[i][2 * h + 1] * inv, (T*)nullptr);
      zero = fmaf(o[i][2 * h], 0.0f, fmaf(o[i][2 * h + 1], 0.0f, zero));
    }
    if (p.lse && (lane & 3) == 0) p.lse[token * p.heads + head] = fmaf(m[h], c2, log2f(l[h])) * kLn2;
  }
  if (p.causal && __any_sync(0xffffffffu, isnan(zero))) take_rows_again<T, D>(p, job, head, job.tile * kRows + warp * 16);
}

template <class T, int D>
static cudaError_t run(const PromptArgs& a, cudaStream_t stream) {
  constexpr int smem = (kRows + 4 * keys_of(D)) * D * 2;
  cudaError_t e = cudaFuncSetAttribute(prompt_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(a.tokens / kRows + a.seqs), (unsigned)a.heads);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, prompt_kernel<T, D>, a);
}
template <class T>
static cudaError_t run_type(const PromptArgs& a, cudaStream_t stream) {
  switch (a.dim) {
    case 64: return run<T, 64>(a, stream);
    case 128: return run<T, 128>(a, stream);
    case 192: return run<T, 192>(a, stream);
    default: return run<T, 256>(a, stream);
  }
}

}  // namespace prompt

int launch_prompt(const PromptArgs& a, cudaStream_t stream, std::string* err) {
  if (prompt_tc_takes(a)) return launch_prompt_tc(a, stream, err);
  const cudaError_t e = a.dtype == AQD_F16 ? prompt::run_type<__half>(a, stream) : prompt::run_type<__nv_bfloat16>(a, stream);
  if (e == cudaSuccess) return 0;
  *err = std::string("prompt attention: ") + cudaGetErrorString(e);
  return 3;
}

}  // namespace aqd
