// lm_linear.cu -- product of int8 codes with a scale per token and per output channel: the weights' layout, the kernel for
// few tokens, one that takes any shape, stride and alignment without a workspace, and the choice among them and the
// tensor-core kernel for many tokens. Every one computes the same exact sums. Sizes below are tokens x n x K.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "../../include/aqd.h"
#include "common.cuh"
#include "kernels.h"
#include "tc_ptx.cuh"

namespace aqd {
namespace lin {

// Rows of k codes plus 128, as bytes (what the conversion to F16 starts from), padded with code 0 to whole chunks of
// 128; and the header's first word, the most chunks in a row that any row of weights lets an FP32 accumulator sum exactly:
// those of every window of that length have sum |w| * 128 <= 2^24. (8 chunks always do.) One warp per row, eight chunks' loads at a
// time, in words where all rows start on one.
template <bool kWords>
__global__ void __launch_bounds__(128) prepare_kernel(const int8_t* __restrict__ codes, int64_t ld, int32_t n, int32_t k,
                                                      int64_t pitch, uint8_t* __restrict__ out) {
  __shared__ uint16_t sums[4][1024];  // sum |w| of each chunk (at most 128 * 128)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int chunks = (int)(pitch / 128);
  int most = chunks;
  for (int64_t row = (int64_t)blockIdx.x * 4 + warp; row < n; row += (int64_t)gridDim.x * 4) {
    const int8_t* from = codes + row * ld;
    uint32_t* to = reinterpret_cast<uint32_t*>(out + kLinHeader + row * pitch) + lane;
    for (int c0 = 0; c0 < chunks; c0 += 8) {
      uint32_t w[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const int i = (c0 + c) * 128 + lane * 4;
        w[c] = 0;
        if (kWords && i + 4 <= k) w[c] = __ldg(reinterpret_cast<const uint32_t*>(from + i));
        else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (i + j < k) w[c] |= (uint32_t)(uint8_t)from[i + j] << (8 * j);
        }
      }
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        if (c0 + c >= chunks) break;
        to[(c0 + c) * 32] = w[c] ^ 0x80808080u;
        const uint32_t s = __reduce_add_sync(0xffffffffu, __dp4a(__vabs4(w[c]), 0x01010101u, 0u));  // (|-128| is 128 there)
        if (lane == 0) sums[warp][c0 + c] = (uint16_t)s;
      }
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

// Tokens at any address without a workspace: 32 tokens x 64 channels per block of 256 threads, 8 outputs a thread, four products per __dp4a.
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

// ---------------------------------------------------------------- few tokens

__device__ __forceinline__ uint4 ld_weights(const uint8_t* p) {  // read once: past L1
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.L2::128B.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// Four codes with 128 added, as bytes, to F16: a byte u under the exponent byte 0x64 is 1024 + u, and 1024 + u - 1152 the code.
__device__ __forceinline__ void bytes_to_f16(uint32_t u, uint32_t& lo, uint32_t& hi) {
  const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(0x64806480u));
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(0x64806480u));
}
__device__ __forceinline__ void piece_to_f16(const uint4& v, uint32_t flip, uint32_t (&f)[8]) {
  bytes_to_f16(v.x ^ flip, f[0], f[1]);
  bytes_to_f16(v.y ^ flip, f[2], f[3]);
  bytes_to_f16(v.z ^ flip, f[4], f[5]);
  bytes_to_f16(v.w ^ flip, f[6], f[7]);
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Tokens' codes from rows at any address to rows that start on 16 bytes, 4 codes a thread.
__global__ void __launch_bounds__(256) align_kernel(const int8_t* __restrict__ x, int64_t ldx, int32_t k, uint32_t* __restrict__ out, int64_t pitch) {
  tc::grid_dep_wait();
  const int i = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (i >= k) return;
  x += blockIdx.y * ldx + i;
  uint32_t v = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (i + j < k) v |= (uint32_t)(uint8_t)x[j] << (8 * j);
  out[(blockIdx.y * pitch + i) / 4] = v;
}

constexpr int kSmallWarps = 8;

constexpr int small_bytes(int g, int r, int depth) {
  const int ring = kSmallWarps * depth * (2 * r + g) * 512, part = kSmallWarps * g * 8 * (16 * r + 1) * 4;
  return ring > part ? ring : part;
}

// Up to 8 kG tokens: bound by the weights' bytes. A block takes 16 kR channels and all tokens, and its warps take 64-K pieces
// of the rows in turn, as operands of mma.sync. The order of K within a piece is free, so a lane's 16 adjacent codes
// of a row are its fragments of four MMAs: each lane copies the bytes that it will itself multiply into its own places of a ring in
// shared memory (kDepth pieces ahead, no barrier between lanes) and turns them into F16 in registers. Sums are exact in FP32 over
// 1024 K, then add up in int32 (kLong: a warp has more than that), across warps in shared memory.
// (Measured: 1 x 4096 x 4096 5.7 us; 1 x 12288 x 4096 11.3, 4.4 TB/s; 24 x 12288 x 4096 14.8, 3.4 TB/s. At two row tiles and 18.2 us for that
// one: loads straight into registers, a round of them at a time, 23.3; weights by bulk copies, the tokens' loads then waited for
// at each stage, 33; tokens as F16 once per block and K split over a cluster, 20.)
template <int kG, int kR, int kDepth, bool kLong>
__global__ void __launch_bounds__(kSmallWarps * 32, kG * kR == 16 ? 1 : 2) linear_ring_kernel(const LinArgs p) {
  extern __shared__ __align__(16) uint8_t smem[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int64_t pitch = ((int64_t)p.k + 127) / 128 * 128;
  const int n0 = blockIdx.x * 16 * kR;
  const int64_t m0 = (int64_t)blockIdx.y * (8 * kG);
  constexpr int kPieces = 2 * kR + kG;
  const uint32_t ring = tc::smem_u32(smem) + (uint32_t)warp * (kDepth * kPieces * 512) + (uint32_t)lane * 16;
  tc::grid_dep_wait();
  const uint8_t* w = p.w + kLinHeader + (int64_t)(n0 + g) * pitch + t * 16;
  const int8_t* x = p.x + (m0 + g) * p.ldx + t * 16;
  const int rows = p.n - n0 - g, tokens = (int)min((int64_t)(8 * kG), p.m - m0) - g;
  const int blocks = (p.k + 63) / 64;
  const int mine = (blocks - warp + kSmallWarps - 1) / kSmallWarps;  // this warp's blocks: warp, warp + 8, ...
  auto fetch = [&](int i) {
    if (i < mine) {
      const int k = (warp + i * kSmallWarps) * 64;
      const uint32_t to = ring + (uint32_t)(i % kDepth) * (kPieces * 512);
      // (rows and tokens past the last, and codes past a row's end: zeros, from an address that is not read)
#pragma unroll
      for (int r = 0; r < 2 * kR; ++r) {
        const bool in = r * 8 < rows;
        asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;"
                     ::"r"(to + r * 512), "l"(in ? w + (r * 8 * pitch + k) : p.w), "r"(in ? 16 : 0) : "memory");
      }
      const int left = p.k - k - t * 16, bytes = left < 0 ? 0 : (left < 16 ? left : 16);
#pragma unroll
      for (int j = 0; j < kG; ++j) {
        const bool in = j * 8 < tokens && bytes > 0;
        asm volatile("cp.async.ca.shared.global [%0], [%1], 16, %2;"
                     ::"r"(to + (2 * kR + j) * 512), "l"(in ? x + (j * 8 * p.ldx + k) : p.x), "r"(in ? bytes : 0) : "memory");
      }
    }
    tc::cp_async_commit();
  };
#pragma unroll
  for (int i = 0; i < kDepth - 1; ++i) fetch(i);
  int sum[kR][kG][4];
  float d[kR][kG][4] = {};
  if constexpr (kLong) {
#pragma unroll
    for (int r = 0; r < kR; ++r)
#pragma unroll
      for (int j = 0; j < kG; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) sum[r][j][q] = 0;
  }
  for (int i = 0; i < mine; ++i) {
    tc::cp_async_wait<kDepth - 2>();
    const uint32_t from = ring + (uint32_t)(i % kDepth) * (kPieces * 512);
    if constexpr (kR < 3) {  // the weights wait in registers
      uint32_t wf[2 * kR][8];
#pragma unroll
      for (int r = 0; r < 2 * kR; ++r) piece_to_f16(lds128(from + r * 512), 0u, wf[r]);
#pragma unroll
      for (int j = 0; j < kG; ++j) {
        uint32_t xf[8];
        piece_to_f16(lds128(from + (2 * kR + j) * 512), 0x80808080u, xf);
#pragma unroll
        for (int r = 0; r < kR; ++r)
#pragma unroll
          for (int q = 0; q < 8; q += 2)
            mma_16816(d[r][j], wf[2 * r][q], wf[2 * r + 1][q], wf[2 * r][q + 1], wf[2 * r + 1][q + 1], xf[q], xf[q + 1]);
      }
    } else {  // the tokens do
      uint32_t xf[kG][8];
#pragma unroll
      for (int j = 0; j < kG; ++j) piece_to_f16(lds128(from + (2 * kR + j) * 512), 0x80808080u, xf[j]);
#pragma unroll
      for (int r = 0; r < kR; ++r) {
        uint32_t lo[8], hi[8];
        piece_to_f16(lds128(from + 2 * r * 512), 0u, lo);
        piece_to_f16(lds128(from + (2 * r + 1) * 512), 0u, hi);
#pragma unroll
        for (int q = 0; q < 8; q += 2)
#pragma unroll
          for (int j = 0; j < kG; ++j) mma_16816(d[r][j], lo[q], hi[q], lo[q + 1], hi[q + 1], xf[j][q], xf[j][q + 1]);
      }
    }
    fetch(i + kDepth - 1);
    if (kLong && (i & 15) == 15) {
#pragma unroll
      for (int r = 0; r < kR; ++r)
#pragma unroll
        for (int j = 0; j < kG; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q) { sum[r][j][q] += __float2int_rn(d[r][j][q]); d[r][j][q] = 0.0f; }
    }
  }
  __syncthreads();  // (every fetched stage has been waited for; the sums take the ring's place)
  int* part = reinterpret_cast<int*>(smem);
  constexpr int kRow = 16 * kR + 1, kPart = kG * 8 * kRow;
#pragma unroll
  for (int r = 0; r < kR; ++r)
#pragma unroll
    for (int i = 0; i < kG; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        part[warp * kPart + (i * 8 + 2 * t + (j & 1)) * kRow + r * 16 + g + (j >> 1) * 8] = (kLong ? sum[r][i][j] : 0) + __float2int_rn(d[r][i][j]);
  __syncthreads();
  for (int i = threadIdx.x; i < kG * 8 * 16 * kR; i += kSmallWarps * 32) {
    const int c = i % (16 * kR), m = i / (16 * kR);
    int s = 0;
#pragma unroll
    for (int v = 0; v < kSmallWarps; ++v) s += part[v * kPart + m * kRow + c];
    if (m0 + m < p.m && n0 + c < p.n) store_y(p, m0 + m, n0 + c, s);
  }
}

template <int kG, int kR, int kDepth, bool kLong>
static cudaError_t run_ring(const LinArgs& a, cudaStream_t stream) {
  constexpr int smem = small_bytes(kG, kR, kDepth);
  if constexpr (smem > 48 * 1024) {
    const cudaError_t e = cudaFuncSetAttribute(linear_ring_kernel<kG, kR, kDepth, kLong>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(((int64_t)a.n + 16 * kR - 1) / (16 * kR)), (unsigned)((a.m + 8 * kG - 1) / (8 * kG)));
  cfg.blockDim = dim3(kSmallWarps * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, linear_ring_kernel<kG, kR, kDepth, kLong>, a);
}

// Time of this kernel (us) with r row tiles a warp, for the launch that takes m tokens in groups of 8: a launch's fill and drain, and
// blocks per SM times a block's share of an SM, most of which grows with K. Fitted to n 1024 .. 16384, K 1024 .. 12288. More row tiles halve, or
// third, the work on the tokens' codes for each weight, and the blocks, so the best count follows from how the blocks fill the SMs (K 4096, 1, 2 and 3 row
// tiles: 24 tokens, n 2048 5.6, 7.6 and 8.8 us; n 6144 11.2, 11.1, 9.4; n 8192 13.9, 11.4, 14.3; n 12288 19.4, 16.6, 14.8; 16 tokens, n 12288 15.1, 13.2,
// 12.2; 64 tokens, n 2048 9.5 and 13.4, n 4096 17.9 and 13.6). 0: no such kernel (it would spill registers), or never the best (up to 8 tokens,
// n 12288 11.5 and 10.9, n 16384 13.5 and 15.0).
static int groups_of(int64_t m) { return m <= 8 ? 1 : m <= 16 ? 2 : m <= 24 ? 3 : m <= 32 ? 4 : 8; }
static float ring_time(const LinArgs& a, int r) {
  static constexpr float kTime[9][3][2] = {{}, {{3.1f, 1.45f}}, {{2.7f, 2.1f}, {2.2f, 3.65f}, {2.6f, 4.85f}}, {{2.6f, 2.85f}, {3.2f, 4.3f}, {2.9f, 5.8f}},
                                           {{2.6f, 3.3f}, {3.3f, 4.95f}}, {}, {}, {}, {{0.9f, 8.5f}, {1.3f, 12.3f}}};
  const int g = groups_of(a.m);
  const float *t = kTime[g][r - 1], grows = g == 8 ? 0.75f : 0.9f;
  if (t[1] == 0.0f || (a.k > 16 * 64 * kSmallWarps && (r == 3 || (r == 2 && (g == 3 || g == 4))))) return INFINITY;
  const float blocks = (float)(((int64_t)a.n + 16 * r - 1) / (16 * r)) * (float)((a.m + 8 * g - 1) / (8 * g));
  return t[0] + t[1] * ceilf(blocks / 152.0f) * (1.0f - grows + grows * (float)((a.k + 63) / 64) / 64.0f);
}
static int ring_tiles(const LinArgs& a) {  // the row tiles of the fastest
  const float t[3] = {ring_time(a, 1), ring_time(a, 2), ring_time(a, 3)};
  return t[2] < t[1] && t[2] < t[0] ? 3 : t[1] < t[0] ? 2 : 1;
}
static float ring_estimate(const LinArgs& a) { return ring_time(a, ring_tiles(a)); }

static int launch_ring(const LinArgs& a, cudaStream_t stream, std::string* err) {
  const bool longk = a.k > 16 * 64 * kSmallWarps;
  const int g = groups_of(a.m), r = ring_tiles(a);
  cudaError_t e;
  if (g == 1) e = longk ? run_ring<1, 1, 4, true>(a, stream) : run_ring<1, 1, 4, false>(a, stream);
  else if (g == 2 && r == 1) e = longk ? run_ring<2, 1, 4, true>(a, stream) : run_ring<2, 1, 4, false>(a, stream);
  else if (g == 2 && r == 2) e = longk ? run_ring<2, 2, 4, true>(a, stream) : run_ring<2, 2, 4, false>(a, stream);
  else if (g == 2) e = run_ring<2, 3, 3, false>(a, stream);
  else if (g == 3 && r == 1) e = longk ? run_ring<3, 1, 4, true>(a, stream) : run_ring<3, 1, 4, false>(a, stream);
  else if (g == 3 && r == 2) e = run_ring<3, 2, 3, false>(a, stream);
  else if (g == 3) e = run_ring<3, 3, 3, false>(a, stream);
  else if (g == 4 && r == 1) e = longk ? run_ring<4, 1, 4, true>(a, stream) : run_ring<4, 1, 4, false>(a, stream);
  else if (g == 4) e = run_ring<4, 2, 3, false>(a, stream);
  else if (r == 1) e = longk ? run_ring<8, 1, 3, true>(a, stream) : run_ring<8, 1, 3, false>(a, stream);
  else e = longk ? run_ring<8, 2, 3, true>(a, stream) : run_ring<8, 2, 3, false>(a, stream);
  if (e == cudaSuccess) e = cudaGetLastError();
  if (e != cudaSuccess) { *err = std::string("8-bit product launch: ") + cudaGetErrorString(e); return AQD_ERR_CUDA; }
  return 0;
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
  const bool words = ld % 4 == 0 && (reinterpret_cast<uintptr_t>(codes) & 3) == 0;
  void (*kernel)(const int8_t*, int64_t, int32_t, int32_t, int64_t, uint8_t*) = words ? lin::prepare_kernel<true> : lin::prepare_kernel<false>;
  kernel<<<n < 9728 ? (n + 3) / 4 : 2432, 128, 0, stream>>>(codes, ld, n, k, lin_pitch(k), out);
  return launched("weight preparation launch: ", err);
}

size_t linear_workspace_bytes(int64_t m, int32_t n, int32_t k) { return linear_tc_workspace_bytes(m, k); }

int launch_linear(const LinArgs& call, cudaStream_t stream, std::string* err) {
  LinArgs a = call;
  bool aligned = (a.m == 1 || a.ldx % 16 == 0) && (reinterpret_cast<uintptr_t>(a.x) & 15) == 0;
  const float tc = a.m > 16 || !aligned ? linear_tc_estimate(a) : INFINITY;
  // Few tokens at other addresses are copied to the workspace first (2 us; 16 tokens, n 4096, K 4100: the tensor cores, which take any address,
  // 17.1 us; up to 16 aligned tokens never need these).
  const int64_t pitch = ((int64_t)a.k + 15) / 16 * 16;
  if (!aligned && a.m <= 64 && a.ws && a.ws_bytes >= (size_t)(a.m * pitch) && (a.m <= 16 || lin::ring_estimate(a) + 2.0f < tc)) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((a.k + 1023) / 1024), (unsigned)a.m);
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, lin::align_kernel, a.x, a.ldx, a.k, reinterpret_cast<uint32_t*>(a.ws), pitch);
    if (e != cudaSuccess) { *err = std::string("8-bit product launch: ") + cudaGetErrorString(e); return AQD_ERR_CUDA; }
    a.x = reinterpret_cast<const int8_t*>(a.ws);
    a.ldx = pitch;
    return lin::launch_ring(a, stream, err);
  }
  if (aligned && a.m <= 16) return lin::launch_ring(a, stream, err);
  if (tc < INFINITY && (!aligned || tc < lin::ring_estimate(a))) return launch_linear_tc(a, stream, err);
  // the tokens in pieces of the grid's second dimension
  const int64_t most = 65535LL * (aligned ? 64 : lin::kTM);
  const size_t es = a.y_dtype == AQD_F32 || a.y_dtype == AQD_I32 ? 4 : 2;
  for (int64_t m = 0; m < a.m; m += most) {
    LinArgs p = a;
    p.m = a.m - m < most ? a.m - m : most;
    p.x += m * a.ldx;
    if (p.x_scale) p.x_scale += m;
    p.y = static_cast<uint8_t*>(p.y) + (size_t)m * a.ldy * es;
    int st = 0;
    if (aligned) st = lin::launch_ring(p, stream, err);
    else {
      const dim3 grid((unsigned)(((int64_t)p.n + lin::kTN - 1) / lin::kTN), (unsigned)((p.m + lin::kTM - 1) / lin::kTM));
      lin::linear_direct_kernel<<<grid, 256, 0, stream>>>(p);
      st = launched("8-bit product launch: ", err);
    }
    if (st) return st;
  }
  return 0;
}

}  // namespace aqd
