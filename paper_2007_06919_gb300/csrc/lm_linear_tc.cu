// lm_linear_tc.cu -- product of int8 codes on the tensor cores, for more than a handful of tokens.
//
// sm_103a has no integer tcgen05.mma. int8 values are exact in F16, their products (up to 2^14) and sums up to 2^24 exact
// in the FP32 accumulator, so kind::f16 computes integer sums, in segments of K short enough for the weights at hand
// (the prepared weights carry the length, from the largest sum of |w| over any run of K); segments add up in int32.
//
// CTA pairs take tiles of 256 output channels x up to 256 tokens, 128 K at a time. The weights stay one byte: TMA brings them into
// shared memory, 8 warps turn them into F16 in TMEM, where they are the A operand (channels along TMEM lanes, so a
// warp's store of one token's outputs is contiguous, and a channel's scale is one register). The tokens' codes, which every channel tile
// reads again, become F16 once per call, in the workspace (expand_kernel), and TMA brings them as the B operand. One thread of the pair issues
// the MMAs (cta_group::2).
// (Measured at 8192 tokens, n 12288, K 4096, with expand_kernel: 445 to 460 us for the first launches after a pause, 1790 to 1850 TFLOP/s; 490 us, 1680 TFLOP/s,
// from 50 ms on, when the power limit lowers the clock. A library bf16 product of that size 412 to 433 and 470. Both operands converted
// in the kernel 578 us at best, bound by the converting warps' issue slots and their stages' shared memory.)
//
// A pair computes whole tiles, in turn. The tiles' width in tokens follows the problem (plan): narrow tiles give few tokens to every pair, where
// splitting K and adding the shares up in the workspace cost more than it gave (512 tokens, n and K 4096, 34.9 us split, 21.9 with tiles of
// 128 tokens; 2048 tokens 63.8 and 53.3).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>
#include <mutex>
#include <type_traits>

#include "../../include/aqd.h"
#include "common.cuh"
#include "kernels.h"
#include "tc_ptx.cuh"

namespace aqd {
namespace lintc {

using namespace tc;

constexpr int kKC = 128;           // K per stage
constexpr int kMinRaw = 4, kMaxRaw = 8;  // stages of the weights' bytes
constexpr int kCvt = 4;            // stages of converted weights (TMEM: 64 columns each beside 256 accumulator columns)
constexpr int kMaxX = 8;           // stages of the tokens
// Warps: 8 read the accumulators and write outputs, 8 convert, in two sets that take stages in turn, and one thread each issues
// the two operands' copies and the MMAs. Registers move from the last two kinds to the first. The stages of both weight rings are a
// whole multiple of the sets, so that one set alone waits on a stage's barriers: a set that met a barrier two phases ahead would pass it.
constexpr int kEpi = 8, kSets = 2, kSetWarps = 4;
constexpr int kWarpCvt = kEpi, kWarpTmaW = kWarpCvt + kSets * kSetWarps, kWarpTmaX = kWarpTmaW + 1, kWarpMma = kWarpTmaW + 2;
constexpr int kThreads = (kWarpTmaW + 4) * 32;  // (an idle warp fills the issuing warps' warpgroup)
constexpr int kRegsLaunch = 65536 / kThreads / 8 * 8, kRegsEpi = 176, kRegsCvt = 40, kRegsIssue = 48;
static_assert(kEpi * kRegsEpi + kSets * kSetWarps * kRegsCvt + 4 * kRegsIssue <= kThreads / 32 * kRegsLaunch, "the launch's registers");
static_assert(kCvt % kSets == 0 && kMinRaw % kSets == 0 && kMaxRaw % kSets == 0, "one set for each stage of the weights");
constexpr int kEpiCols = kEpi / 4, kBlocks = 16 / kEpiCols;  // warps of a lane quarter; 16-token blocks of each
constexpr int kTmemA = 256;        // first column of the converted weights
constexpr int kRawW = 128 * kKC;   // bytes of a stage's weights
constexpr int kSmemLimit = 232448;

struct Params {
  LinArgs a;
  int32_t nt, tok_tiles;           // tokens per tile (multiple of 16), token tiles
  int32_t chunks;                  // K in pieces of kKC
  int32_t tiles, pairs;            // pair j computes tiles j, j + pairs, ...
  int32_t raw_stages, x_stages;    // (raw_stages: kMinRaw or kMaxRaw)
};
struct Maps {
  CUtensorMap w, x;
};

struct Barriers {
  uint64_t raw_full[kMaxRaw], raw_empty[kMaxRaw], cv_full[kCvt], cv_empty[kCvt], x_full[kMaxX], x_empty[kMaxX], d_full, d_empty, done;
  uint32_t tmem, seg;
  int abort_flag;
  alignas(16) float scales[2][256];  // the tokens' scales of a tile, and of the next
};

__device__ __forceinline__ bool mbar_test_cluster(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// Bounded wait of the MMA thread, for arrivals from both CTAs.
__device__ __forceinline__ bool wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  if (mbar_test_cluster(bar, parity)) return true;
  const uint64_t deadline = globaltimer() + kTimeoutNs;
  for (uint32_t spin = 1;; ++spin) {
    if (mbar_test_cluster(bar, parity)) return true;
    if ((spin & 63) == 0 && (*abort_flag || globaltimer() > deadline)) return false;
  }
}
// D (+)= A B, A in TMEM (128 lanes of each CTA, two F16 per column), B in shared memory
__device__ __forceinline__ void mma_f16_pair_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
// Four codes with 128 added, as bytes, to F16: a byte u under the exponent byte 0x64 is 1024 + u, and 1024 + u - 1152 the code.
__device__ __forceinline__ void bytes_to_f16(uint32_t u, uint32_t& lo, uint32_t& hi) {
  const uint32_t a = __byte_perm(u, 0x64646464u, 0x4140), b = __byte_perm(u, 0x64646464u, 0x4342);
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(0x64806480u));
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(0x64806480u));
}

__device__ __forceinline__ void put(float* y, float v) { *y = v; }
__device__ __forceinline__ void put(__half* y, float v) { *y = __float2half_rn(v); }
__device__ __forceinline__ void put(__nv_bfloat16* y, float v) { *y = __float2bfloat16_rn(v); }

// The outputs of one 16-token block of a lane's channel from its sums (int32, or their float32 bits); xs: the tokens' scales
// (shared memory, 16-byte aligned).
template <class T>
__device__ __forceinline__ void store_block(const LinArgs& a, int64_t m0, int n, const int (&acc)[16], bool ints, float ws, float bias, uint32_t xs) {
  T* y = static_cast<T*>(a.y) + m0 * a.ldy + n;
  const int left = (int)(a.m - m0 < 16 ? a.m - m0 : 16);
#pragma unroll
  for (int j0 = 0; j0 < 16; j0 += 4) {
    const uint4 s4 = lds128(xs + j0 * 4);
    const float s[4] = {__uint_as_float(s4.x), __uint_as_float(s4.y), __uint_as_float(s4.z), __uint_as_float(s4.w)};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float v = ints ? __int2float_rn(acc[j0 + j]) : __int_as_float(acc[j0 + j]);
      if (j0 + j < left) put(y, __fadd_rn(__fmul_rn(__fmul_rn(v, s[j]), ws), bias));
      y += a.ldy;
    }
  }
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
linear_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Params p) {
  extern __shared__ __align__(1024) uint8_t smem[];  // weights, tokens, Barriers
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1;
  const int rows_x = p.nt >> 1;                      // tokens of this CTA
  const uint32_t raw0 = smem_u32(smem), x0 = raw0 + (uint32_t)p.raw_stages * kRawW;
  const uint32_t x_half = (uint32_t)rows_x * kKC, x_bytes = 2 * x_half;  // 64 K of F16 a row and half (whole kilobytes: rows_x is a multiple of 8)
  Barriers& bar = *reinterpret_cast<Barriers*>(smem + p.raw_stages * kRawW + p.x_stages * x_bytes);
  volatile int* abort_flag = &bar.abort_flag;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kMaxRaw; ++i) {
      mbar_init(smem_u32(&bar.raw_full[i]), 1);
      mbar_init(smem_u32(&bar.raw_empty[i]), kSetWarps);
    }
    for (int i = 0; i < kCvt; ++i) {
      mbar_init(smem_u32(&bar.cv_full[i]), 2 * kSetWarps);
      mbar_init(smem_u32(&bar.cv_empty[i]), 1);
    }
    for (int i = 0; i < kMaxX; ++i) {
      mbar_init(smem_u32(&bar.x_full[i]), 1);
      mbar_init(smem_u32(&bar.x_empty[i]), 1);
    }
    mbar_init(smem_u32(&bar.d_full), 1);
    mbar_init(smem_u32(&bar.d_empty), 2 * kEpi);
    mbar_init(smem_u32(&bar.done), 1);
    bar.abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == kWarpMma) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&bar.tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  // (what follows the previous kernel's end: every read and write of global memory)
  grid_dep_wait();
  if (threadIdx.x == 0) bar.seg = *reinterpret_cast<const volatile uint32_t*>(p.a.w);
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = *const_cast<volatile uint32_t*>(&bar.tmem);
  // K in segments of `per` chunks, no longer than the weights allow
  const int nseg = (p.chunks + (int)bar.seg - 1) / (int)bar.seg, per = (p.chunks + nseg - 1) / nseg;

  if (warp >= kWarpTmaW) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    if (warp == kWarpTmaW && elect_one()) {
      uint32_t st = 0, ph = 0, issued = 0;
      bool ok = true;
      for (int tile = pair; ok && tile < p.tiles; tile += p.pairs) {
        const int yw = tile / p.tok_tiles * 256 + (int)rank * 128;
        for (int c = 0; c < p.chunks; ++c) {
          if (!mbar_wait(smem_u32(&bar.raw_empty[st]), ph ^ 1, abort_flag)) { ok = false; break; }
          const uint32_t full = smem_u32(&bar.raw_full[st]);
          mbar_arrive_expect_tx(full, kRawW);
          tma_load_2d(raw0 + st * kRawW, &maps.w, c * kKC, yw, full);
          ++issued;
          if (++st == (uint32_t)p.raw_stages) { st = 0; ph ^= 1; }
        }
      }
      if (!ok) {
        fail(abort_flag, p.a.status);
        // the copies in flight end before the block does (each of these waits is bounded too)
        int never = 0;
        for (uint32_t i = 0; i < (issued < (uint32_t)p.raw_stages ? issued : (uint32_t)p.raw_stages); ++i) {
          const uint32_t q = issued - 1 - i;
          mbar_wait(smem_u32(&bar.raw_full[q % p.raw_stages]), (q / p.raw_stages) & 1, &never);
        }
      }
    }
    if (warp == kWarpTmaX && elect_one()) {
      // both CTAs' copies complete on the leader's barrier
      const uint32_t full0 = mapa_shared(smem_u32(&bar.x_full[0]), 0);
      uint32_t st = 0, ph = 0, issued = 0;
      bool ok = true;
      for (int tile = pair; ok && tile < p.tiles; tile += p.pairs) {
        const int yx = tile % p.tok_tiles * p.nt + (int)rank * rows_x;
        for (int c = 0; c < p.chunks; ++c) {
          if (!mbar_wait(smem_u32(&bar.x_empty[st]), ph ^ 1, abort_flag)) { ok = false; break; }
          if (rank == 0) mbar_arrive_expect_tx(smem_u32(&bar.x_full[st]), 2 * x_bytes);
          const uint32_t dst = x0 + st * x_bytes;
          tma_load_2d_pair(dst, &maps.x, c * kKC, yx, full0 + st * 8);
          tma_load_2d_pair(dst + x_half, &maps.x, c * kKC + 64, yx, full0 + st * 8);
          ++issued;
          if (++st == (uint32_t)p.x_stages) { st = 0; ph ^= 1; }
        }
      }
      if (!ok) {
        fail(abort_flag, p.a.status);
        int never = 0;
        if (rank == 0)
          for (uint32_t i = 0; i < (issued < (uint32_t)p.x_stages ? issued : (uint32_t)p.x_stages); ++i) {
            const uint32_t q = issued - 1 - i;
            mbar_wait(smem_u32(&bar.x_full[q % p.x_stages]), (q / p.x_stages) & 1, &never);
          }
      }
    }
    if (warp == kWarpMma && rank == 0 && elect_one()) {
      const uint32_t idesc = idesc_e4m3(p.nt, 256);
      uint32_t st = 0, ph = 0, xst = 0, xph = 0, dph = 0;
      bool ok = true;
      for (int tile = pair; ok && tile < p.tiles; tile += p.pairs) {
        for (int c = 0; ok && c < p.chunks; c += per) {
          if (!wait_cluster(smem_u32(&bar.d_empty), dph ^ 1, abort_flag)) { ok = false; break; }
          dph ^= 1;
          tc_fence_after();
          const int end = c + per < p.chunks ? c + per : p.chunks;
          for (int i = c; i < end; ++i) {
            if (!wait_cluster(smem_u32(&bar.x_full[xst]), xph, abort_flag) || !wait_cluster(smem_u32(&bar.cv_full[st]), ph, abort_flag)) {
              ok = false;
              break;
            }
            tc_fence_after();
            const uint32_t a0 = tmem + kTmemA + st * 64, b0 = x0 + xst * x_bytes;
#pragma unroll
            for (int s = 0; s < 8; ++s)
              mma_f16_pair_ta(tmem, a0 + s * 8, sdesc_sw128(b0 + (s >> 2) * x_half + (s & 3) * 32), idesc, (i > c || s > 0) ? 1u : 0u);
            mma_commit_pair_both(smem_u32(&bar.cv_empty[st]));
            mma_commit_pair_both(smem_u32(&bar.x_empty[xst]));
            if (++st == kCvt) { st = 0; ph ^= 1; }
            if (++xst == (uint32_t)p.x_stages) { xst = 0; xph ^= 1; }
          }
          if (ok) mma_commit_pair_both(smem_u32(&bar.d_full));
        }
      }
      if (!ok) {
        fail(abort_flag, p.a.status);
        mma_commit_pair(smem_u32(&bar.done));  // MMAs in flight end before the block does (bounded)
        int never = 0;
        mbar_wait(smem_u32(&bar.done), 0, &never);
      }
    }
  } else if (warp >= kWarpCvt) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsCvt));
    const int q = warp & 3, set = (warp - kWarpCvt) / kSetWarps, row = q * 32 + lane;
    const uint32_t cv_full0 = mapa_shared(smem_u32(&bar.cv_full[0]), 0);
    const uint32_t to_tmem = tmem + ((uint32_t)(q * 32) << 16) + kTmemA;
    // a thread converts one row; piece c (16 codes) of a row lies at c ^ (row & 7) of its 128 bytes
    const uint32_t from = (uint32_t)row * 128 + (uint32_t)((row & 7) << 4);
    const int total = (p.tiles - pair + p.pairs - 1) / p.pairs * p.chunks;
    uint32_t rst = (uint32_t)set, rph = 0;
    for (int i = set; i < total; i += kSets) {
      const uint32_t cst = (uint32_t)i % kCvt, cph = ((uint32_t)i / kCvt) & 1;
      bool ok = mbar_wait_inline(smem_u32(&bar.raw_full[rst]), rph, abort_flag) &&
                mbar_wait_inline(smem_u32(&bar.cv_empty[cst]), cph ^ 1, abort_flag);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) { fail(abort_flag, p.a.status); break; }
      const uint32_t raw = raw0 + rst * kRawW;
      tc_fence_after();
      // (loads of four pieces, then their conversion: asm volatile keeps this order)
#pragma unroll
      for (int c0 = 0; c0 < 8; c0 += 4) {
        uint4 w[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) w[c] = lds128(raw + (from ^ ((c0 + c) << 4)));
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t f[8];
          bytes_to_f16(w[c].x, f[0], f[1]);
          bytes_to_f16(w[c].y, f[2], f[3]);
          bytes_to_f16(w[c].z, f[4], f[5]);
          bytes_to_f16(w[c].w, f[6], f[7]);
          tmem_st8(to_tmem + cst * 64 + (c0 + c) * 8, f);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bar.raw_empty[rst]));
      rst += kSets;
      if (rst >= (uint32_t)p.raw_stages) { rst -= (uint32_t)p.raw_stages; rph ^= 1; }
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster_relaxed(cv_full0 + cst * 8);
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsEpi));
    const int q = warp & 3, g = warp >> 2, wrow = q * 32 + lane;
    const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
    const uint32_t d_empty = mapa_shared(smem_u32(&bar.d_empty), 0);
    uint32_t dph = 0;
    bool ok = true;  // after a wait that ran out: on to the end without waiting or storing (see takes_tile)
    int buf = 0;
    for (int tile = pair; tile < p.tiles; tile += p.pairs, buf ^= 1) {
      const int tn = tile / p.tok_tiles, tm = tile - tn * p.tok_tiles;
      int acc[kBlocks][16];  // float32 bits of sums (one segment), or int32
      {
        const int64_t m = (int64_t)tm * p.nt + threadIdx.x;
        bar.scales[buf][threadIdx.x] = p.a.y_dtype != AQD_I32 && (int)threadIdx.x < p.nt && m < p.a.m ? __ldg(p.a.x_scale + m) : 0.0f;
        named_bar(1, kEpi * 32);
      }
      auto read_sums = [&](auto add) {  // waits for a segment, takes its sums and hands the accumulator back
        if (ok && !mbar_wait_inline(smem_u32(&bar.d_full), dph, abort_flag)) { ok = false; fail(abort_flag, p.a.status); }
        dph ^= 1;
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) return;
        tc_fence_after();
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
          const int col = (g + kEpiCols * b) * 16;
          if (col < p.nt) {
#pragma unroll
            for (int h = 0; h < 16; h += 8) {
              uint32_t r[8];
              tmem_ld8(lane_base + col + h, r);
              tmem_wait_ld();
              reg_fence8(r);
#pragma unroll
              for (int j = 0; j < 8; ++j) acc[b][h + j] = add.value ? acc[b][h + j] + __float2int_rn(__uint_as_float(r[j])) : (int)r[j];
            }
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster_relaxed(d_empty);
      };
      if (nseg == 1) {
        read_sums(std::false_type{});
      } else {
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int j = 0; j < 16; ++j) acc[b][j] = 0;
        for (int i = 0; i < nseg; ++i) read_sums(std::true_type{});
      }
      const int n = tn * 256 + (int)rank * 128 + wrow;
      if (!ok || n >= p.a.n) continue;
      const bool ints = nseg > 1;
      const float ws = p.a.y_dtype == AQD_I32 ? 0.0f : __ldg(p.a.w_scale + n);
      const float bias = p.a.bias ? __ldg(p.a.bias + n) : -0.0f;  // (x + -0 is x)
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        const int col = (g + kEpiCols * b) * 16;
        const int64_t m0 = (int64_t)tm * p.nt + col;
        if (col >= p.nt || m0 >= p.a.m) continue;
        const uint32_t xs = smem_u32(&bar.scales[buf][col]);
        if (p.a.y_dtype == AQD_F32) store_block<float>(p.a, m0, n, acc[b], ints, ws, bias, xs);
        else if (p.a.y_dtype == AQD_F16) store_block<__half>(p.a, m0, n, acc[b], ints, ws, bias, xs);
        else if (p.a.y_dtype == AQD_BF16) store_block<__nv_bfloat16>(p.a, m0, n, acc[b], ints, ws, bias, xs);
        else {
          int32_t* y = static_cast<int32_t*>(p.a.y) + m0 * p.a.ldy + n;
#pragma unroll
          for (int j = 0; j < 16; ++j) {
            if (m0 + j < p.a.m) *y = ints ? acc[b][j] : __float2int_rn(__int_as_float(acc[b][j]));
            y += p.a.ldy;
          }
        }
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  if (warp == kWarpMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// The tokens' codes as F16, rows of 16 `pieces` values, zero past k: a thread 16 codes at a time.
__global__ void __launch_bounds__(256) expand_kernel(const int8_t* __restrict__ x, int64_t ldx, int64_t m, int32_t k, int32_t pieces,
                                                     uint64_t div_pieces, uint4* __restrict__ out, int vec) {
  grid_dep_launch();
  grid_dep_wait();
  const int64_t total = m * pieces;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = total < (1LL << 31) ? fast_div((int)i, div_pieces) : i / pieces;
    const int c = (int)(i - row * pieces) * 16;
    const int8_t* from = x + row * ldx + c;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (vec && c + 16 <= k) v = __ldg(reinterpret_cast<const uint4*>(from));
    else if (c < k) {
      uint32_t q[4] = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < 16; ++j)
        if (c + j < k) q[j >> 2] |= (uint32_t)(uint8_t)__ldg(from + j) << (8 * (j & 3));
      v = make_uint4(q[0], q[1], q[2], q[3]);
    }
    uint32_t h[8];
    bytes_to_f16(v.x ^ 0x80808080u, h[0], h[1]);
    bytes_to_f16(v.y ^ 0x80808080u, h[2], h[3]);
    bytes_to_f16(v.z ^ 0x80808080u, h[4], h[5]);
    bytes_to_f16(v.w ^ 0x80808080u, h[6], h[7]);
    out[2 * i] = make_uint4(h[0], h[1], h[2], h[3]);
    out[2 * i + 1] = make_uint4(h[4], h[5], h[6], h[7]);
  }
}

// ---------------------------------------------------------------- host side

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
static EncodeTiledFn get_encode_fn() {
  static EncodeTiledFn fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* ptr = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault, &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<EncodeTiledFn>(ptr);
  });
  return fn;
}
// a matrix of rows of ld bytes; boxes of 128 bytes (values x their size) by box_rows
static bool encode(CUtensorMap* map, CUtensorMapDataType type, int size, const void* base, int64_t cols, int64_t rows, int64_t ld, int box_rows) {
  EncodeTiledFn enc = get_encode_fn();
  if (!enc) return false;
  cuuint64_t dim[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)ld};
  cuuint32_t box[2] = {(cuuint32_t)(128 / size), (cuuint32_t)box_rows}, es[2] = {1, 1};
  return enc(map, type, 2, const_cast<void*>(base), dim, stride, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static int sm_pairs() {
  int dev = 0, sms = 0;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms / 2;
}
static size_t x_bytes(int64_t m, int64_t k) { return ((size_t)m * (size_t)lin_pitch((int32_t)k) * 2 + 255) / 256 * 256; }

// The tiles' width: the one of the least estimated time. A pair's tiles follow one another; a stage of 128 K takes the longer of
// its conversion and its MMAs; the first fill, the last epilogue and the expansion pass stand outside. (Microseconds, fitted to
// n 512 .. 12288, k 512 .. 4096, m 80 .. 8192 at widths of 16 .. 256: within about 15%.)
static float plan(const LinArgs& a, int pairs, Params* p) {
  const int64_t tn = ((int64_t)a.n + 255) / 256;
  const int chunks = (a.k + kKC - 1) / kKC;
  float best = INFINITY;
  int64_t width = 16;
  for (int nt = 16; nt <= 256; nt += 16) {
    const int64_t tm = (a.m + nt - 1) / nt, waves = (tn * tm + pairs - 1) / pairs;
    const float t = (float)(waves * chunks) * fmaxf(0.38f, 0.00273f * nt) + 4.5f + 0.02f * nt;
    if (t < best) { best = t; width = nt; }
    if (tm == 1) break;
  }
  if (p) {
    p->a = a;
    p->chunks = chunks;
    p->tok_tiles = (int32_t)((a.m + width - 1) / width);
    p->nt = (int32_t)(((a.m + p->tok_tiles - 1) / p->tok_tiles + 15) / 16 * 16);
    p->tiles = (int32_t)(tn * p->tok_tiles);
    p->pairs = p->tiles < pairs ? p->tiles : pairs;
  }
  return best + 3e-6f * 0.15f * (float)a.m * (float)a.k;
}

}  // namespace lintc

float linear_tc_estimate(const LinArgs& a) {
  const int pairs = lintc::sm_pairs();
  // (a pair's stages are counted in 32 bits)
  if (pairs < 1 || a.m >= (1LL << 31) - 512 || (a.m + 15) / 16 * (((int64_t)a.n + 255) / 256) * ((a.k + 127) / 128) >= (1LL << 31) ||
      a.ws_bytes < lintc::x_bytes(a.m, a.k))
    return INFINITY;
  return lintc::plan(a, pairs, nullptr);
}

size_t linear_tc_workspace_bytes(int64_t m, int32_t k) { return m < 1 ? 0 : lintc::x_bytes(m, k); }

int launch_linear_tc(const LinArgs& a, cudaStream_t stream, std::string* err) {
  using namespace lintc;
  Params p{};
  plan(a, sm_pairs(), &p);
  const int rows_x = p.nt / 2, xs = 2 * rows_x * kKC;
  // narrow tiles leave room for more of the weights on their way, which their short stages need (64 tokens, n 12288, K 4096 17.8 us; 19.4
  // with kMinRaw); wide ones need it for the tokens
  p.raw_stages = p.nt <= 128 ? kMaxRaw : kMinRaw;
  p.x_stages = (kSmemLimit - (int)sizeof(Barriers) - p.raw_stages * kRawW) / xs;
  if (p.x_stages > kMaxX) p.x_stages = kMaxX;
  const size_t smem = (size_t)p.raw_stages * kRawW + (size_t)p.x_stages * xs + sizeof(Barriers);
  const int64_t pitch = lin_pitch(a.k);
  Maps maps;
  if (!encode(&maps.w, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.w + kLinHeader, pitch, a.n, pitch, 128) ||
      !encode(&maps.x, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, a.ws, pitch, a.m, 2 * pitch, rows_x)) {
    *err = "cuTensorMapEncodeTiled failed";
    return AQD_ERR_CUDA;
  }
  // raised to the same limit always: a captured graph's launches stay within it
  cudaError_t e = cudaFuncSetAttribute(linear_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit);
  if (e == cudaSuccess) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const int pieces = (int)(pitch / 16);
    const int64_t blocks = (a.m * pieces + 255) / 256;
    cfg.gridDim = dim3((unsigned)(blocks < 152 * 16 ? blocks : 152 * 16));
    cfg.blockDim = dim3(256);
    const int vec = a.ldx % 16 == 0 && (reinterpret_cast<uintptr_t>(a.x) & 15) == 0;
    e = cudaLaunchKernelEx(&cfg, expand_kernel, a.x, a.ldx, a.m, a.k, pieces, div_magic(pieces), reinterpret_cast<uint4*>(a.ws), vec);
    if (e == cudaSuccess) {
      cfg.gridDim = dim3(2u * (unsigned)p.pairs);
      cfg.blockDim = dim3(kThreads);
      cfg.dynamicSmemBytes = smem;
      e = cudaLaunchKernelEx(&cfg, linear_tc_kernel, maps, p);
    }
    if (e == cudaSuccess) e = cudaGetLastError();
  }
  if (e != cudaSuccess) { *err = std::string("8-bit product launch: ") + cudaGetErrorString(e); return AQD_ERR_CUDA; }
  return 0;
}

}  // namespace aqd
