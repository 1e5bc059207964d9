// lm_prompt_tc.cu -- attention over packed prompts on the fifth-generation tensor cores, for heads of 64 and 128.
//
// A block takes 256 query rows of one head as two tiles of 128, and keys 128 at a time. Scores S = Q K^T and the outputs O of both tiles
// live in TMEM; a thread per row reads its scores from there, subtracts the running maximum, takes exponentials, and writes the weights over the
// scores as 16-bit numbers, from where they are the A operand of O += P V (V as it lies: its rows are K of that product). While one
// tile's rows are at their exponentials, the tensor cores have the other tile's two products, so a step of both takes the longer of four
// products of 128 x 128 x D (4 x 512 cycles for D = 128) and two passes over 128 scores a thread.
//
// The outputs are brought to a new maximum only where it grew by more than a factor of 2^8 since the last time: weights stay below that, sums are
// float32, and the division at the end is exact in it. So after the first few tiles of keys no row touches its outputs before the end.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <mutex>
#include <type_traits>

#include "../../include/aqd.h"
#include "common.cuh"
#include "kernels.h"
#include "lm_prompt.cuh"
#include "tc_ptx.cuh"

namespace aqd {
namespace prompttc {

using namespace tc;
using prompt::Job;
using prompt::ex2;
using prompt::kLn2;
using prompt::kLog2e;
using prompt::pack;

constexpr int kTile = 128;                  // rows of a query tile, keys of a step
constexpr int kSoftWarps = 8, kWarpTma = 8, kWarpMma = 9, kWarpFix = 10, kThreads = 384;
// registers: a row's 128 scores stay in its thread's
constexpr int kRegsLaunch = 168, kRegsSoft = 200, kRegsIssue = 104;
static_assert(kSoftWarps * kRegsSoft + 4 * kRegsIssue <= kThreads / 32 * kRegsLaunch, "the launch's registers");
constexpr int kSmemLimit = 232448;
constexpr float kGrowth = 8.0f;             // powers of two that a maximum may grow by before sums are brought to it

__host__ __device__ constexpr int tile_bytes(int dim) { return kTile * dim * 2; }
__host__ __device__ constexpr int ring(int dim) { return dim == 128 ? 5 : 8; }

struct Barriers {
  uint64_t q_full, full[8], empty[8], s_full[2], p_full[2], o_done[2], last_v, fixed;
  uint64_t red[kThreads / 32];
  Job job;
  uint32_t tmem;
  int abort_flag;
};
struct Maps {
  CUtensorMap q, k, v;
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%2, %3, %4}], [%5];"
      ::"r"(dst), "l"((uint64_t)map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// D (+)= A B with A in TMEM (a lane per row, two 16-bit numbers a column)
__device__ __forceinline__ void mma_f16_ta(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc) : "memory");
}
// 128-byte-swizzled descriptor of an operand whose rows are K: blocks of 64 columns x 8 rows of K, 1024 bytes from 8 rows to the next (stride offset),
// `block` bytes from 64 columns to the next (leading offset)
__device__ __forceinline__ uint64_t sdesc_sw128_mn(uint32_t saddr, uint32_t block) {
  uint64_t d = (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(block >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* f) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]),
        "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
#pragma unroll
  for (int i = 0; i < 32; ++i) f[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
               "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// keeps uses of f behind this point (after the wait for a TMEM load)
__device__ __forceinline__ void settle(float* f) {
#pragma unroll
  for (int i = 0; i < 32; i += 8)
    asm volatile("" : "+f"(f[i]), "+f"(f[i + 1]), "+f"(f[i + 2]), "+f"(f[i + 3]), "+f"(f[i + 4]), "+f"(f[i + 5]), "+f"(f[i + 6]), "+f"(f[i + 7]));
}
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
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// The job's tiles of keys that query tile t sees.
__device__ __forceinline__ int steps_of(const Job& jb, int t, int causal) {
  const int row0 = jb.tile * 2 * kTile + t * kTile;
  const int rows = jb.queries - row0 < kTile ? jb.queries - row0 : kTile;
  if (rows <= 0) return 0;
  int64_t see = causal ? (int64_t)row0 + rows + (jb.keys - jb.queries) : jb.keys;
  see = see < 0 ? 0 : see > jb.keys ? jb.keys : see;
  return (int)((see + kTile - 1) / kTile);
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads, 1) prompt_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ PromptArgs p) {
  constexpr int kBytes = tile_bytes(D), kRing = ring(D), kBoxes = D / 64, kBox = kTile * 128;
  constexpr uint32_t kO = 256;  // TMEM: scores of the tiles from columns 0 and 128 on (weights over them), outputs from 256 and 256 + D on
  extern __shared__ __align__(1024) uint8_t smem[];  // queries of both tiles, the ring of keys and values, Barriers
  Barriers& bar = *reinterpret_cast<Barriers*>(smem + (2 + kRing) * kBytes);
  volatile int* abort_flag = &bar.abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t sq = smem_u32(smem), ring0 = sq + 2 * kBytes;

  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&bar.q_full), 1);
    for (int i = 0; i < kRing; ++i) {
      mbar_init(smem_u32(&bar.full[i]), 1);
      mbar_init(smem_u32(&bar.empty[i]), 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&bar.s_full[t]), 1);
      mbar_init(smem_u32(&bar.p_full[t]), 4);
      mbar_init(smem_u32(&bar.o_done[t]), 1);
    }
    mbar_init(smem_u32(&bar.last_v), 1);
    mbar_init(smem_u32(&bar.fixed), 1);
    bar.abort_flag = 0;
    fence_barrier_init();
  }
  grid_dep_wait();
  if (!prompt::find_job(p, 2 * kTile, blockIdx.y, &bar.job, bar.red)) return;
  const Job jb = bar.job;
  if (warp == kWarpMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bar.tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *const_cast<volatile uint32_t*>(&bar.tmem);
  const int head = blockIdx.x, kvh = head / (p.heads / p.kv_heads);
  const int n0 = steps_of(jb, 0, p.causal), n1 = steps_of(jb, 1, p.causal), n = n0 > n1 ? n0 : n1;
  const int rows = jb.queries - jb.tile * 2 * kTile;  // of both tiles, and behind them
  const bool cut = n * kTile > jb.keys;               // the last step's tile ends behind the sequence

  if (warp >= kSoftWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    if (warp == kWarpTma && elect_one() && n > 0) {
      const uint32_t qf = smem_u32(&bar.q_full);
      const int qrow = jb.start + jb.tile * 2 * kTile;
      mbar_arrive_expect_tx(qf, rows > kTile ? 2 * kBytes : kBytes);
#pragma unroll
      for (int b = 0; b < kBoxes; ++b) tma_load_3d(sq + b * kBox, &maps.q, b * 64, head, qrow, qf);
      if (rows > kTile) {
#pragma unroll
        for (int b = 0; b < kBoxes; ++b) tma_load_3d(sq + kBytes + b * kBox, &maps.q, b * 64, head, qrow + kTile, qf);
      }
      uint32_t st = 0, ph = 0;
      int issued = 0;
      auto load = [&](const CUtensorMap* map, int key) {
        if (!mbar_wait(smem_u32(&bar.empty[st]), ph ^ 1, abort_flag)) return false;
        const uint32_t full = smem_u32(&bar.full[st]);
        mbar_arrive_expect_tx(full, kBytes);
#pragma unroll
        for (int b = 0; b < kBoxes; ++b) tma_load_3d(ring0 + st * kBytes + b * kBox, map, b * 64, kvh, key, full);
        ++issued;
        if (++st == (uint32_t)kRing) { st = 0; ph ^= 1; }
        return true;
      };
      bool ok = true;
      for (int j = 0; ok && j < n; ++j) {
        const int key = jb.kv_start + j * kTile;
        ok = load(&maps.k, key) && load(&maps.v, key);
      }
      if (!ok) {
        fail(abort_flag, p.status);
        int never = 0;  // the copies in flight end before the block does (each of these waits is bounded too)
        mbar_wait(qf, 0, &never);
        for (int i = issued > kRing ? issued - kRing : 0; i < issued; ++i) mbar_wait(smem_u32(&bar.full[i % kRing]), (uint32_t)(i / kRing) & 1, &never);
      }
    }
    if (warp == kWarpMma && elect_one() && n > 0) {
      constexpr uint32_t type = std::is_same<T, __half>::value ? 0u : (1u << 7) | (1u << 10);
      const uint32_t id_s = idesc_e4m3(kTile) | type, id_o = idesc_e4m3(D) | type | 1u << 16;  // (bit 16: B's rows are K)
      auto scores = [&](int t, uint32_t k) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
          mma_f16(tmem + t * kTile, sdesc_sw128(sq + t * kBytes + (s >> 2) * kBox + (s & 3) * 32), sdesc_sw128(k + (s >> 2) * kBox + (s & 3) * 32), id_s, s > 0);
        mma_commit(smem_u32(&bar.s_full[t]));
      };
      bool ok = mbar_poll(smem_u32(&bar.q_full), 0, abort_flag) && mbar_poll(smem_u32(&bar.full[0]), 0, abort_flag);
      if (ok) {
        tc_fence_after();
        if (n0 > 0) scores(0, ring0);
        if (n1 > 0) scores(1, ring0);
        mma_commit(smem_u32(&bar.empty[0]));
      }
      for (int j = 0; ok && j < n; ++j) {
        const int iv = 2 * j + 1, ik = 2 * j + 2;  // places in the ring's order
        const uint32_t v = ring0 + iv % kRing * kBytes, k = ring0 + ik % kRing * kBytes;
        if (!mbar_poll(smem_u32(&bar.full[iv % kRing]), (uint32_t)(iv / kRing) & 1, abort_flag)) { ok = false; break; }
        if (j == n - 1 && cut) {
          mbar_arrive(smem_u32(&bar.last_v));
          if (!mbar_poll(smem_u32(&bar.fixed), 0, abort_flag)) { ok = false; break; }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int nt = t ? n1 : n0;
          if (j >= nt) continue;
          if (!mbar_poll(smem_u32(&bar.p_full[t]), (uint32_t)j & 1, abort_flag)) { ok = false; break; }
          tc_fence_after();
#pragma unroll
          for (int s = 0; s < kTile / 16; ++s)
            mma_f16_ta(tmem + kO + t * D, tmem + t * kTile + s * 8, sdesc_sw128_mn(v + s * 2048, kBox), id_o, j > 0 || s > 0);
          if (j + 1 == nt) mma_commit(smem_u32(&bar.o_done[t]));
          if (j + 1 < nt) {
            if (!mbar_poll(smem_u32(&bar.full[ik % kRing]), (uint32_t)(ik / kRing) & 1, abort_flag)) { ok = false; break; }
            tc_fence_after();
            scores(t, k);
          }
        }
        if (!ok) break;
        mma_commit(smem_u32(&bar.empty[iv % kRing]));
        if (j + 1 < n) mma_commit(smem_u32(&bar.empty[ik % kRing]));
      }
      if (!ok) fail(abort_flag, p.status);
    }
    if (warp == kWarpFix && cut && n > 0) {
      // the last tile's value rows behind the sequence's end are another's: 0 instead, so that weights of 0 meet no NaN
      const int iv = 2 * (n - 1) + 1, first = jb.keys - (n - 1) * kTile;
      if (mbar_wait(smem_u32(&bar.last_v), 0, abort_flag)) {
        uint8_t* v = smem + (2 + iv % kRing) * kBytes;
        for (int i = first * 8 + lane; i < kTile * 8; i += 32)
          for (int b = 0; b < kBoxes; ++b) reinterpret_cast<uint4*>(v + b * kBox)[i] = make_uint4(0, 0, 0, 0);
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bar.fixed));
      } else {
        fail(abort_flag, p.status);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoft));
    const int t = warp >> 2, row = (warp & 3) * 32 + lane;  // (a warp reads the quarter of TMEM's lanes that its number gives)
    const int nt = t ? n1 : n0, at = jb.tile * 2 * kTile + t * kTile + row;  // this thread's row of the sequence
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, ts = tmem + t * kTile + lanes, to = tmem + kO + t * D + lanes;
    const float c2 = fmaxf(p.scale * kLog2e, 1.4e-45f), grow = kGrowth / c2;
    int64_t see = p.causal ? (int64_t)at + (jb.keys - jb.queries) + 1 : jb.keys;
    const int lim = (int)(see < 0 ? 0 : see > jb.keys ? jb.keys : see);
    float m = -INFINITY, l = 0.0f;
    bool ok = true;
    for (int j = 0; j < nt; ++j) {
      if (!mbar_wait_inline(smem_u32(&bar.s_full[t]), (uint32_t)j & 1, abort_flag)) { ok = false; break; }
      tc_fence_after();
      float s[kTile];
#pragma unroll
      for (int i = 0; i < kTile; i += 32) tmem_ld32(ts + i, s + i);
      tmem_wait_ld();
#pragma unroll
      for (int i = 0; i < kTile; i += 32) settle(s + i);
      const int here = lim - j * kTile;  // places of this tile that the row sees
      if (__any_sync(0xffffffffu, here < kTile)) {
#pragma unroll
        for (int i = 0; i < kTile; ++i)
          if (i >= here) s[i] = -INFINITY;
      }
      float a[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
      for (int i = 4; i < kTile; i += 4)
#pragma unroll
        for (int c = 0; c < 4; ++c) a[c] = fmaxf(a[c], s[i + c]);
      const float top = fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3]));
      const bool grew = top > m + grow;  // (from -infinity: any score)
      if (__any_sync(0xffffffffu, grew)) {
        const float f = grew ? ex2((m - top) * c2) : 1.0f;
        if (grew) m = top;
        l *= f;
        if (j > 0) {
          // (the last step's products are done: this step's scores were issued behind them and have arrived)
#pragma unroll
          for (int i = 0; i < D; i += 16) {
            uint32_t o[16];
            tmem_ld16(to + i, o);
            tmem_wait_ld();
            reg_fence16(o);
#pragma unroll
            for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * f);
            tmem_st16(to + i, o);
          }
        }
      }
      float ref = m == -INFINITY ? 0.0f : m;
      // the factor goes into one multiply-add with the maximum, but where scores are so large that its rounding shows
      if (__any_sync(0xffffffffu, fabsf(ref * c2) > 1e5f)) {
#pragma unroll
        for (int i = 0; i < kTile; ++i) s[i] -= ref;
        ref = 0.0f;
      }
      const uint64_t c22 = two_of(c2, c2), r22 = two_of(-ref * c2, -ref * c2);
      uint64_t sum[2] = {0, 0};
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          float x, y;
          one_each(fma2(two_of(s[32 * h + 2 * i], s[32 * h + 2 * i + 1]), c22, r22), x, y);
          x = ex2(x);
          y = ex2(y);
          sum[i & 1] = add2(sum[i & 1], two_of(x, y));
          w[i] = pack(x, y, (T*)nullptr);
        }
        tmem_st16(ts + 16 * h, w);
      }
      float u, v;
      one_each(add2(sum[0], sum[1]), u, v);
      l += u + v;
      tmem_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bar.p_full[t]));
    }
    if (ok && nt > 0 && !mbar_wait_inline(smem_u32(&bar.o_done[t]), 0, abort_flag)) ok = false;
    if (!ok) fail(abort_flag, p.status);
    tc_fence_after();
    const bool live = t * kTile + row < rows;
    const float inv = m == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l;
    T* y = static_cast<T*>(p.out) + (int64_t)(jb.start + at) * p.ldo + (int64_t)head * p.ldoh;
    if (t * kTile < rows) {
#pragma unroll
      for (int i = 0; i < D; i += 32) {
        float o[32];
        if (nt > 0) {
          tmem_ld32(to + i, o);
          tmem_wait_ld();
          settle(o);
        } else {
#pragma unroll
          for (int c = 0; c < 32; ++c) o[c] = 0.0f;
        }
        if (live && ok) {
#pragma unroll
          for (int c = 0; c < 32; c += 8)
            *reinterpret_cast<uint4*>(y + i + c) = make_uint4(pack(o[c] * inv, o[c + 1] * inv, (T*)nullptr), pack(o[c + 2] * inv, o[c + 3] * inv, (T*)nullptr),
                                                              pack(o[c + 4] * inv, o[c + 5] * inv, (T*)nullptr), pack(o[c + 6] * inv, o[c + 7] * inv, (T*)nullptr));
        }
      }
      if (live && ok && p.lse) p.lse[(int64_t)(jb.start + at) * p.heads + head] = fmaf(m, c2, log2f(l)) * kLn2;
    }
    tc_fence_before();
  }
  __syncthreads();
  if (warp == kWarpMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
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
// [tokens][heads][dim] of 16-bit numbers, boxes of 128 tokens x 64 numbers of one head
static bool encode(CUtensorMap* map, bool half, const void* base, int64_t dim, int64_t heads, int64_t tokens, int64_t ld, int64_t ldh) {
  EncodeTiledFn enc = get_encode_fn();
  if (!enc) return false;
  // (a stride over one head or token only is never used)
  if (heads == 1) ldh = dim;
  if (tokens == 1) ld = heads * dim;
  cuuint64_t size[3] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)tokens}, stride[2] = {(cuuint64_t)ldh * 2, (cuuint64_t)ld * 2};
  cuuint32_t box[3] = {64, 1, kTile}, es[3] = {1, 1, 1};
  return enc(map, half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), size, stride, box, es,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <class T, int D>
static cudaError_t run(const PromptArgs& a, const Maps& maps, cudaStream_t stream) {
  constexpr size_t smem = (2 + ring(D)) * tile_bytes(D) + sizeof(Barriers);
  static_assert(smem <= kSmemLimit, "");
  cudaError_t e = cudaFuncSetAttribute(prompt_tc_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)a.heads, (unsigned)(a.tokens / (2 * kTile) + a.seqs));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, prompt_tc_kernel<T, D>, maps, a);
}

}  // namespace prompttc

bool prompt_tc_takes(const PromptArgs& a) {
  // strides that a tensor map can hold; blocks along the grid's second axis
  const int64_t most = 1LL << 38;
  const int64_t ld[6] = {a.ldq, a.ldqh, a.ldk, a.ldkh, a.ldv, a.ldvh};
  for (int i = 0; i < 6; ++i)
    if (ld[i] < 1 || ld[i] > most) return false;
  return (a.dim == 64 || a.dim == 128) && a.kv_tokens > 0 && a.tokens / (2 * prompttc::kTile) + a.seqs <= 65535;
}

int launch_prompt_tc(const PromptArgs& a, cudaStream_t stream, std::string* err) {
  using namespace prompttc;
  Maps maps;
  const bool half = a.dtype == AQD_F16;
  if (!encode(&maps.q, half, a.q, a.dim, a.heads, a.tokens, a.ldq, a.ldqh) || !encode(&maps.k, half, a.k, a.dim, a.kv_heads, a.kv_tokens, a.ldk, a.ldkh) ||
      !encode(&maps.v, half, a.v, a.dim, a.kv_heads, a.kv_tokens, a.ldv, a.ldvh)) {
    *err = "cuTensorMapEncodeTiled failed";
    return AQD_ERR_CUDA;
  }
  const cudaError_t e = half ? (a.dim == 64 ? run<__half, 64>(a, maps, stream) : run<__half, 128>(a, maps, stream))
                             : (a.dim == 64 ? run<__nv_bfloat16, 64>(a, maps, stream) : run<__nv_bfloat16, 128>(a, maps, stream));
  if (e == cudaSuccess) return 0;
  *err = std::string("prompt attention: ") + cudaGetErrorString(e);
  return AQD_ERR_CUDA;
}

}  // namespace aqd
