// lm_linear_tc.cu -- product of int8 codes on the tensor cores, for more than a handful of tokens.
//
// sm_103a has no integer tcgen05.mma. int8 values are exact in F16, their products (up to 2^14) and sums up to 2^24 exact
// in the FP32 accumulator, so kind::f16 computes integer sums, in segments of K short enough for the weights at hand
// (the prepared weights carry the length, from the largest sum of |w| over any run of K); segments add up in int32.
//
// Codes stay one byte everywhere but in the operand buffers. CTA pairs take tiles of 256 output channels x up
// to 256 tokens, 128 K at a time: TMA brings the bytes of both operands into shared memory, 16 warps turn them into F16,
// and one thread of the pair issues the MMAs (cta_group::2). The weights are the A operand and go to
// TMEM, so that shared memory, which these MMAs, the copies and the conversion share, carries them once as bytes and
// not again as F16; the tokens are the B operand, in shared memory. Channels then lie along TMEM lanes, so a
// warp's store of one token's outputs is contiguous.
//
// Tiles beyond whole waves (all tiles, for few tokens) are split over K so that every pair gets an equal share; the shares
// of a tile add up in int32 in the workspace by atomics, whose order does not change integer sums, and the CTA that
// comes last writes the outputs and zeroes the workspace again.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <mutex>

#include "../../include/aqd.h"
#include "common.cuh"
#include "kernels.h"
#include "tc_ptx.cuh"

namespace aqd {
namespace lintc {

using namespace tc;

constexpr int kKC = 128;           // K per stage
constexpr int kCvt = 4;            // converted stages (TMEM: 64 columns each beside 256 accumulator columns)
constexpr int kMaxRaw = 8;         // stages of bytes
constexpr int kWorkers = 16;       // converting warps, which also read the accumulators
constexpr int kWarpTma = kWorkers, kWarpMma = kWorkers + 1;
constexpr int kThreads = (kWorkers + 2) * 32;
constexpr int kTmemA = 256;        // first column of the converted weights
constexpr int kRawW = 128 * kKC;   // bytes of a stage's weights
constexpr int kSmemLimit = 232448;

struct Params {
  LinArgs a;
  int32_t nt, tok_tiles;           // tokens per tile (multiple of 16), token tiles
  int32_t chunks;                  // K in pieces of kKC
  int32_t tiles, dp_tiles;         // all tiles; those that one pair computes whole, in waves
  int32_t pairs, sk_pairs;         // pairs of the grid; those that share the other tiles
  int64_t sk_total;                // chunks of the other tiles
  int32_t raw_stages;
  int32_t* partial;                // [tiles - dp_tiles][2][nt][128] int32, zero between calls
  uint32_t* counter;               // [tiles - dp_tiles][2], zero between calls
};
struct Maps {
  CUtensorMap w, x;
};

struct Barriers {
  uint64_t raw_full[kMaxRaw], raw_empty[kMaxRaw], cv_full[kCvt], cv_empty[kCvt], d_full, d_empty, done;
  uint32_t tmem, seg, last;
  int abort_flag;
};

// The pieces of work of one pair, in order: (tile, first chunk, chunks).
struct Units {
  const Params& p;
  int t, pos, hi;
  __device__ Units(const Params& q, int pair) : p(q), t(pair), pos(0), hi(0) {
    if (pair < q.sk_pairs) { pos = (int)(q.sk_total * pair / q.sk_pairs); hi = (int)(q.sk_total * (pair + 1) / q.sk_pairs); }
  }
  __device__ bool next(int& tile, int& k0, int& len) {
    if (t < p.dp_tiles) {
      tile = t; k0 = 0; len = p.chunks;
      t += p.pairs;
      return true;
    }
    if (pos >= hi) return false;
    const int j = pos / p.chunks;
    tile = p.dp_tiles + j;
    k0 = pos - j * p.chunks;
    len = min(hi - pos, p.chunks - k0);
    pos += len;
    return true;
  }
  // how many pairs share the tile's sums: chunk c belongs to pair floor(((c + 1) sk_pairs - 1) / sk_total)
  __device__ int sharers(int tile) const {
    const int64_t first = (int64_t)(tile - p.dp_tiles) * p.chunks, last = first + p.chunks - 1;
    return (int)(((last + 1) * p.sk_pairs - 1) / p.sk_total - ((first + 1) * p.sk_pairs - 1) / p.sk_total) + 1;
  }
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
__device__ __forceinline__ void arrive_cluster(uint32_t cluster_addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
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
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
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

// (asm volatile keeps its place among the stores: hoisted loads of all tokens' scales would spill)
__device__ __forceinline__ float ld_scale(const float* p) {
  float v;
  asm volatile("ld.global.nc.f32 %0, [%1];" : "=f"(v) : "l"(p));
  return v;
}
// The outputs of one 16-token block of a lane's channel from its sums (int32, or their float32 bits).
template <class T>
__device__ __forceinline__ void store_block(const LinArgs& a, int64_t m0, int n, const int (&acc)[16], bool ints, float ws, float bias) {
  T* y = static_cast<T*>(a.y) + m0 * a.ldy + n;
  const float* xs = a.x_scale + m0;
  const int left = (int)(a.m - m0 < 16 ? a.m - m0 : 16);
#pragma unroll
  for (int j0 = 0; j0 < 16; j0 += 4) {
    float s[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = j0 + j < left ? ld_scale(xs + j0 + j) : 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float v = ints ? __int2float_rn(acc[j0 + j]) : __int_as_float(acc[j0 + j]);
      float o = __fmul_rn(__fmul_rn(v, s[j]), ws);
      if (a.bias) o = __fadd_rn(o, bias);
      if (j0 + j < left) put(y, o);
      y += a.ldy;
    }
  }
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
linear_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Params p) {
  extern __shared__ uint8_t smem_raw[];
  __shared__ Barriers bar;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();
  const int pair = blockIdx.x >> 1;
  const int rows_x = p.nt >> 1;                      // tokens of this CTA
  const uint32_t raw_bytes = (uint32_t)(kRawW + rows_x * kKC);
  const uint32_t cvt0 = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t cvt_stride = (uint32_t)rows_x * 2 * kKC;  // (rows_x is a multiple of 8: both are whole kilobytes)
  const uint32_t raw0 = cvt0 + kCvt * cvt_stride, raw_stride = raw_bytes;
  volatile int* abort_flag = &bar.abort_flag;

  if (threadIdx.x == 0) {
    for (int i = 0; i < p.raw_stages; ++i) {
      mbar_init(smem_u32(&bar.raw_full[i]), 1);
      mbar_init(smem_u32(&bar.raw_empty[i]), kWorkers);
    }
    for (int i = 0; i < kCvt; ++i) {
      mbar_init(smem_u32(&bar.cv_full[i]), 2 * kWorkers);
      mbar_init(smem_u32(&bar.cv_empty[i]), 1);
    }
    mbar_init(smem_u32(&bar.d_full), 1);
    mbar_init(smem_u32(&bar.d_empty), 2 * kWorkers);
    mbar_init(smem_u32(&bar.done), 1);
    bar.abort_flag = 0;
    bar.seg = *reinterpret_cast<const uint32_t*>(p.a.w);
    fence_barrier_init();
  }
  if (warp == kWarpMma) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&bar.tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  cluster_sync();
  tc_fence_after();
  const uint32_t tmem = *const_cast<volatile uint32_t*>(&bar.tmem);
  const int seg = (int)bar.seg;

  if (warp == kWarpTma) {
    if (elect_one()) {
      Units it(p, pair);
      int tile, k0, len;
      uint32_t st = 0, ph = 0, issued = 0;
      bool ok = true;
      while (ok && it.next(tile, k0, len)) {
        const int tn = tile / p.tok_tiles, tm = tile - tn * p.tok_tiles;
        const int yw = tn * 256 + (int)rank * 128, yx = tm * p.nt + (int)rank * rows_x;
        for (int c = k0; c < k0 + len; ++c) {
          if (!mbar_wait(smem_u32(&bar.raw_empty[st]), ph ^ 1, abort_flag)) { ok = false; break; }
          const uint32_t full = smem_u32(&bar.raw_full[st]), dst = raw0 + st * raw_stride;
          mbar_arrive_expect_tx(full, raw_bytes);
          tma_load_2d(dst, &maps.w, c * kKC, yw, full);
          tma_load_2d(dst + kRawW, &maps.x, c * kKC, yx, full);
          ++issued;
          if (++st == (uint32_t)p.raw_stages) { st = 0; ph ^= 1; }
        }
      }
      if (!ok) {
        fail(abort_flag, p.a.status);
        // the copies in flight end before the block does (each of these waits is bounded too)
        const uint32_t n = issued < (uint32_t)p.raw_stages ? issued : (uint32_t)p.raw_stages;
        int never = 0;
        for (uint32_t i = 0; i < n; ++i) {
          const uint32_t q = issued - 1 - i;
          mbar_wait(smem_u32(&bar.raw_full[q % p.raw_stages]), (q / p.raw_stages) & 1, &never);
        }
      }
    }
  } else if (warp == kWarpMma) {
    if (rank == 0 && elect_one()) {
      const uint32_t idesc = idesc_e4m3(p.nt, 256);
      Units it(p, pair);
      int tile, k0, len;
      uint32_t st = 0, ph = 0, dph = 0;
      bool ok = true;
      while (ok && it.next(tile, k0, len)) {
        const int nseg = (len + seg - 1) / seg, per = (len + nseg - 1) / nseg;
        for (int c = 0; ok && c < len; c += per) {
          if (!wait_cluster(smem_u32(&bar.d_empty), dph ^ 1, abort_flag)) { ok = false; break; }
          dph ^= 1;
          tc_fence_after();
          const int end = c + per < len ? c + per : len;
          for (int i = c; i < end; ++i) {
            if (!wait_cluster(smem_u32(&bar.cv_full[st]), ph, abort_flag)) { ok = false; break; }
            tc_fence_after();
            const uint32_t a0 = tmem + kTmemA + st * 64, b0 = cvt0 + st * cvt_stride;
#pragma unroll
            for (int s = 0; s < 8; ++s) {
              const uint64_t db = sdesc_sw128(b0 + (uint32_t)(s >> 2) * (uint32_t)rows_x * 128u + (uint32_t)(s & 3) * 32u);
              mma_f16_pair_ta(tmem, a0 + s * 8, db, idesc, (i > c || s > 0) ? 1u : 0u);
            }
            mma_commit_pair_both(smem_u32(&bar.cv_empty[st]));
            if (++st == kCvt) { st = 0; ph ^= 1; }
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
  } else {
    const int q = warp & 3, g = warp >> 2;
    const uint32_t lane_base = tmem + ((uint32_t)(q * 32) << 16);
    const uint32_t cv_full0 = mapa_shared(smem_u32(&bar.cv_full[0]), 0);
    const uint32_t d_empty = mapa_shared(smem_u32(&bar.d_empty), 0);
    // this thread's bytes of a stage: 32 of one weight row, and up to two 16-byte pieces of the tokens
    const int wrow = q * 32 + lane;
    const uint32_t woff = (uint32_t)wrow * 128 + (uint32_t)(((2 * g) ^ (wrow & 7)) << 4);  // (the second half: ^ 16)
    const int pieces = rows_x * 8;
    uint32_t xoff[2], yoff[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int i = (int)threadIdx.x + j * (kWorkers * 32);
      const int c = i / rows_x, r = i - c * rows_x;
      xoff[j] = (uint32_t)(kRawW + r * 128 + ((c ^ (r & 7)) << 4));
      yoff[j] = (uint32_t)(((c >> 2) * rows_x + r) * 128 + ((((c & 3) * 2) ^ (r & 7)) << 4));
    }
    int total = p.dp_tiles > pair ? (p.dp_tiles - pair + p.pairs - 1) / p.pairs * p.chunks : 0;
    if (pair < p.sk_pairs) total += (int)(p.sk_total * (pair + 1) / p.sk_pairs - p.sk_total * pair / p.sk_pairs);
    uint32_t rst = 0, rph = 0, cst = 0, cph = 0, dph = 0;
    bool ok = true;  // after a wait that ran out: on to the end without waiting or storing (see takes_tile)
    int conv = 0, done = 0;
    Units it(p, pair);
    int tile, k0, len;
    int acc[4][16];
    while (it.next(tile, k0, len)) {
      const int nseg = (len + seg - 1) / seg, per = (len + nseg - 1) / nseg;
      const int tn = tile / p.tok_tiles, tm = tile - tn * p.tok_tiles;
      for (int c = 0; c < len; c += per) {
        done += (c + per < len ? per : len - c);
        // conversion runs up to three stages ahead of the accumulator that is read next, so the MMAs go on meanwhile
        const int want = done + kCvt - 1 < total ? done + kCvt - 1 : total;
        for (; conv < want; ++conv) {
          if (ok && !mbar_wait_inline(smem_u32(&bar.raw_full[rst]), rph, abort_flag)) { ok = false; fail(abort_flag, p.a.status); }
          if (ok) {
            const uint32_t raw = raw0 + rst * raw_stride, cv = cvt0 + cst * cvt_stride;
            if (!mbar_wait_inline(smem_u32(&bar.cv_empty[cst]), cph ^ 1, abort_flag)) { ok = false; fail(abort_flag, p.a.status); }
            ok = __all_sync(0xffffffffu, ok);
            if (ok) {
              tc_fence_after();
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint4 w = lds128(raw + (woff ^ (h << 4)));
                uint32_t f[8];
                bytes_to_f16(w.x, f[0], f[1]);
                bytes_to_f16(w.y, f[2], f[3]);
                bytes_to_f16(w.z, f[4], f[5]);
                bytes_to_f16(w.w, f[6], f[7]);
                tmem_st8(lane_base + kTmemA + cst * 64 + g * 16 + h * 8, f);
              }
#pragma unroll
              for (int j = 0; j < 2; ++j)
                if ((int)threadIdx.x + j * (kWorkers * 32) < pieces) {
                  const uint4 x = lds128(raw + xoff[j]);
                  uint32_t h[8];
                  bytes_to_f16(x.x ^ 0x80808080u, h[0], h[1]);
                  bytes_to_f16(x.y ^ 0x80808080u, h[2], h[3]);
                  bytes_to_f16(x.z ^ 0x80808080u, h[4], h[5]);
                  bytes_to_f16(x.w ^ 0x80808080u, h[6], h[7]);
                  sts128(cv + yoff[j], h[0], h[1], h[2], h[3]);
                  sts128(cv + (yoff[j] ^ 16u), h[4], h[5], h[6], h[7]);
                }
              __syncwarp();
              if (lane == 0) mbar_arrive(smem_u32(&bar.raw_empty[rst]));
              fence_proxy_async();
              tmem_wait_st();
              tc_fence_before();
              __syncwarp();
              if (lane == 0) arrive_cluster(cv_full0 + cst * 8);
            }
          }
          ok = __all_sync(0xffffffffu, ok);
          if (++rst == (uint32_t)p.raw_stages) { rst = 0; rph ^= 1; }
          if (++cst == kCvt) { cst = 0; cph ^= 1; }
        }
        // the segment's sums
        if (ok && !mbar_wait_inline(smem_u32(&bar.d_full), dph, abort_flag)) { ok = false; fail(abort_flag, p.a.status); }
        dph ^= 1;
        ok = __all_sync(0xffffffffu, ok);
        if (ok) {
          tc_fence_after();
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            if ((g + 4 * b) * 16 < p.nt) {
              uint32_t r[16];
              tmem_ld16(lane_base + (g + 4 * b) * 16, r);
              tmem_wait_ld();
              reg_fence16(r);
#pragma unroll
              for (int j = 0; j < 16; ++j)  // a tile of one segment keeps its sums as float32
                acc[b][j] = nseg == 1 ? (int)r[j] : (c == 0 ? 0 : acc[b][j]) + __float2int_rn(__uint_as_float(r[j]));
            }
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive_cluster_relaxed(d_empty);
        }
      }
      const int n = tn * 256 + (int)rank * 128 + wrow;
      bool mine = true, ints = nseg > 1;
      if (len != p.chunks) {
        const int sk = tile - p.dp_tiles;
        int32_t* part = p.partial + ((int64_t)sk * 2 + rank) * p.nt * 128 + wrow;
        if (ok) {
#pragma unroll
          for (int b = 0; b < 4; ++b)
            if ((g + 4 * b) * 16 < p.nt) {
#pragma unroll
              for (int j = 0; j < 16; ++j)
                atomicAdd(part + ((g + 4 * b) * 16 + j) * 128, ints ? acc[b][j] : __float2int_rn(__int_as_float(acc[b][j])));
            }
          __threadfence();
        }
        named_bar(1, kWorkers * 32);
        if (threadIdx.x == 0) {
          const uint32_t before = atomicAdd(p.counter + sk * 2 + rank, 1u);
          bar.last = before + 1 == (uint32_t)it.sharers(tile);
          if (bar.last) p.counter[sk * 2 + rank] = 0;
          __threadfence();
        }
        named_bar(1, kWorkers * 32);
        mine = *const_cast<volatile uint32_t*>(&bar.last) != 0;
        if (mine && ok) {
#pragma unroll
          for (int b = 0; b < 4; ++b)
            if ((g + 4 * b) * 16 < p.nt) {
#pragma unroll
              for (int j = 0; j < 16; ++j) acc[b][j] = __ldcg(part + ((g + 4 * b) * 16 + j) * 128);
#pragma unroll
              for (int j = 0; j < 16; ++j) part[((g + 4 * b) * 16 + j) * 128] = 0;
            }
        }
        ints = true;
      }
      if (mine && ok && n < p.a.n) {
        const float ws = p.a.y_dtype == AQD_I32 ? 0.0f : __ldg(p.a.w_scale + n);
        const float bias = p.a.bias ? __ldg(p.a.bias + n) : 0.0f;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int64_t m0 = (int64_t)tm * p.nt + (g + 4 * b) * 16;
          if ((g + 4 * b) * 16 >= p.nt || m0 >= p.a.m) continue;
          if (p.a.y_dtype == AQD_I32) {
            int32_t* y = static_cast<int32_t*>(p.a.y) + m0 * p.a.ldy + n;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
              if (m0 + j < p.a.m) *y = ints ? acc[b][j] : __float2int_rn(__int_as_float(acc[b][j]));
              y += p.a.ldy;
            }
            continue;
          }
          if (p.a.y_dtype == AQD_F32) store_block<float>(p.a, m0, n, acc[b], ints, ws, bias);
          else if (p.a.y_dtype == AQD_F16) store_block<__half>(p.a, m0, n, acc[b], ints, ws, bias);
          else store_block<__nv_bfloat16>(p.a, m0, n, acc[b], ints, ws, bias);
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
static bool encode(CUtensorMap* map, const void* base, int64_t cols, int64_t rows, int64_t ld, int box_rows) {
  EncodeTiledFn enc = get_encode_fn();
  if (!enc) return false;
  cuuint64_t dim[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, stride[1] = {(cuuint64_t)ld};
  cuuint32_t box[2] = {(cuuint32_t)kKC, (cuuint32_t)box_rows}, es[2] = {1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dim, stride, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

static int sm_pairs() {
  int dev = 0, sms = 0;
  cudaGetDevice(&dev);
  cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
  return sms / 2;
}
static int64_t tiles_of(int64_t m, int64_t n) { return (m + 255) / 256 * ((n + 255) / 256); }
static size_t round256(size_t v) { return (v + 255) / 256 * 256; }

// Tiles, and how they spread over the pairs of CTAs.
static Params plan(const LinArgs& a, int pairs) {
  Params p{};
  p.a = a;
  p.tok_tiles = (int32_t)((a.m + 255) / 256);
  p.nt = (int32_t)(((a.m + p.tok_tiles - 1) / p.tok_tiles + 15) / 16 * 16);
  p.chunks = (a.k + kKC - 1) / kKC;
  p.tiles = (int32_t)tiles_of(a.m, a.n);
  p.pairs = pairs;
  p.dp_tiles = p.tiles / pairs * pairs;
  const int64_t sk = p.tiles - p.dp_tiles;
  p.sk_total = sk * p.chunks;
  p.sk_pairs = p.sk_total < pairs ? (int32_t)p.sk_total : pairs;
  const size_t head = round256((size_t)sk * 8);
  if (sk > 0 && a.ws_bytes >= head + (size_t)sk * p.nt * 256 * 4) {
    p.counter = reinterpret_cast<uint32_t*>(a.ws);
    p.partial = reinterpret_cast<int32_t*>(a.ws + head);
  } else {  // whole tiles only
    p.dp_tiles = p.tiles;
    p.sk_total = 0;
    p.sk_pairs = 0;
  }
  return p;
}

}  // namespace lintc

bool linear_tc_takes(const LinArgs& a) {
  return a.ldx % 16 == 0 && a.ldx >= a.k && a.ldx < (1LL << 39) && (reinterpret_cast<uintptr_t>(a.x) & 15) == 0 &&
         lintc::tiles_of(a.m, a.n) * ((a.k + 127) / 128) < (1LL << 31) && a.m < (1LL << 31) - 512;
}

// Enough for any call with up to m tokens.
size_t linear_tc_workspace_bytes(int64_t m, int32_t n) {
  if (m < 1) return 0;
  const int pairs = lintc::sm_pairs();
  const int64_t tiles = lintc::tiles_of(m, n), sk = tiles < pairs - 1 ? tiles : pairs - 1;
  const int64_t nt = m < 256 ? (m + 15) / 16 * 16 : 256;
  return sk > 0 ? lintc::round256((size_t)sk * 8) + (size_t)sk * nt * 256 * 4 : 0;
}

int launch_linear_tc(const LinArgs& a, cudaStream_t stream, std::string* err) {
  using namespace lintc;
  const int sms2 = sm_pairs();
  if (sms2 < 1) { *err = "no device"; return AQD_ERR_CUDA; }
  Params p = plan(a, sms2);
  const int rows_x = p.nt / 2, cvt = rows_x * 2 * kKC, raw = kRawW + rows_x * kKC;
  p.raw_stages = (kSmemLimit - 2048 - kCvt * cvt) / raw;
  if (p.raw_stages > kMaxRaw) p.raw_stages = kMaxRaw;
  const size_t smem = 1024 + (size_t)kCvt * cvt + (size_t)p.raw_stages * raw;
  Maps maps;
  if (!encode(&maps.w, a.w + kLinHeader, lin_pitch(a.k), a.n, lin_pitch(a.k), 128) ||
      !encode(&maps.x, a.x, a.k, a.m, a.ldx, rows_x)) {
    *err = "cuTensorMapEncodeTiled failed";
    return AQD_ERR_CUDA;
  }
  // raised to the same limit always: a captured graph's launches stay within it
  cudaError_t e = cudaFuncSetAttribute(linear_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemLimit - 1024);
  if (e == cudaSuccess) {
    const int pairs = p.dp_tiles >= p.pairs ? p.pairs : (p.sk_pairs > 0 ? p.sk_pairs : p.dp_tiles);
    linear_tc_kernel<<<2 * pairs, kThreads, smem, stream>>>(maps, p);
    e = cudaGetLastError();
  }
  if (e != cudaSuccess) { *err = std::string("8-bit product launch: ") + cudaGetErrorString(e); return AQD_ERR_CUDA; }
  return 0;
}

}  // namespace aqd
