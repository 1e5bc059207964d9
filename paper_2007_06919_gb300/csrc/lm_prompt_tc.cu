// lm_prompt_tc.cu -- attention over packed prompts on the fifth-generation tensor cores: heads of 64 and 128 (first), of 192 and 256.
//
// A job is 256 query rows of one head, as two tiles of 128, and keys 128 at a time. Scores S = Q K^T and the outputs O of both tiles
// live in TMEM; a thread per row reads its scores from there, subtracts the running maximum, takes exponentials, and writes the weights over the
// scores as 16-bit numbers, from where they are the A operand of O += P V (V as it lies: its rows are K of that product). While one
// tile's rows are at their exponentials, the tensor cores have the other tile's two products. For heads of 128 a step of
// both takes four products of 128 x 128 x 128 (4 x 512 cycles), which bound it: 16,384 tokens of 32 heads 1,260 us, 1,745 TFLOP/s, 90% of the measured
// rate. For heads of 64 the exponentials bound it (2 x 128 x 128 at 32 a cycle, 1024), and a row must not wait for its next scores: TMEM
// has 192 columns for a tile there, in three blocks X, Y, Z. Even steps have their scores in XY and their weights in X, odd ones in YZ and Z: Y is free
// once a row's scores are read, so the next scores come while the exponentials run. (Scores behind the products that read the last
// weights, as for heads of 128: 8192 tokens of 32 heads 263 us, this way 248, 1,108 TFLOP/s. Two threads to a row, 281; the tiles taking turns at the
// exponentials, 267: what is left there is a row's chain of maximum, exponentials and stores, not one unit's rate.)
//
// The outputs are brought to a new maximum only where it grew by more than a factor of 2^8 since the last time: weights stay below that, sums are
// float32, and the division at the end is exact in it. So after the first few tiles of keys no row touches its outputs before the end.
//
// Weights are rounded to 16 bits, which the product takes; the sum that divides has them before that. Where few keys carry a row this shows (bfloat16, by simulation:
// 2.4e-3 of a row off the exact output where sums of rounded weights would leave 1.7e-3, the output's own rounding among both; where many do, 2.3e-3 either way), but
// to take the rounded ones apart again is two more operations a pair in the rows' chain: heads of 64 +15%, of 128 +6%.
//
// Blocks stay and take over the jobs of blocks that have not begun (clusterlaunchcontrol), one warp asking and looking up the sequence ahead of the
// others: a job's first copies and scores run beside the last one's end. (13 prompts of up to
// 2500 tokens, 28 heads of 64: 63 us; with a block for each job, whose start and end cost 6 to 7 us, 84.)
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
constexpr int kSoftWarps = 8, kWarpTma = 8, kWarpMma = 9, kWarpFix = 10, kWarpJobs = 11, kThreads = 384;
constexpr int kSlots = 3;                   // jobs known at a time
constexpr int kAhead = 3;                   // tiles of keys before its end at which a job's block asks for the next one: late, so that blocks end evenly
constexpr int kReaders = kSoftWarps + 3;    // arrivals that free a slot: each softmax warp, and the warps of copies, products and ends
// registers: a row's 128 scores stay in its thread's
constexpr int kRegsLaunch = 168, kRegsSoft = 200, kRegsIssue = 104;
static_assert(kSoftWarps * kRegsSoft + 4 * kRegsIssue <= kThreads / 32 * kRegsLaunch, "the launch's registers");
constexpr int kSmemLimit = 232448;
constexpr float kGrowth = 8.0f;             // powers of two that a maximum may grow by before sums are brought to it

__host__ __device__ constexpr int tile_bytes(int dim) { return kTile * dim * 2; }
__host__ __device__ constexpr int ring(int dim) { return dim == 128 ? 5 : 8; }
__host__ __device__ constexpr int job_rows(int dim) { return dim > 128 ? kTile : 2 * kTile; }

struct Slot {
  Job job;
  int32_t head, valid, n0, n1;  // n: steps of the two tiles
};
// Jobs with outputs that are not finite, of which a value that their rows do not see may be the reason: those rows are taken again at the block's end. The rows' warps mark
// a job by its number, modulo kMarks; the warp that hands jobs out, which gives out one more when they have begun the one kSlots before it, keeps the one before
// that if it is marked, and takes over no more jobs once it has kSpoiled.
constexpr int kSpoiled = 8, kMarks = 8;
static_assert(kMarks > kSlots + 1 && (kMarks & (kMarks - 1)) == 0, "");
struct Marked {
  Job job;
  int32_t head;
};
struct Spoiled {
  int32_t mark[kMarks];
  Marked last[kMarks];                    // the jobs of these numbers
  Marked jobs[kSpoiled];
  int32_t count;
  // (a whole warp, which counts)
  __device__ __forceinline__ void keep(int number, int lane, int& kept) {
    const int at = number & (kMarks - 1);
    if (*const_cast<volatile int32_t*>(&mark[at])) {
      __syncwarp();
      if (lane == 0) {
        jobs[kept] = last[at];
        mark[at] = 0;
      }
      ++kept;
    }
  }
};
// Whoever waits on a barrier meets every one of its phases, and none of them runs two ahead of it. Where scores run ahead, a warp may hand over its next
// weights before another warp of the tile has its last ones ready: weights of even and odd steps have barriers of their own.
struct Barriers {
  uint64_t q_full[2], q_empty[2], full[8], empty[8], s_full[2], p_full[2][2], o_done[2], o_free[2], s_read[2], last_v, fixed, job_full[kSlots], job_empty[kSlots], want, answer;
  alignas(16) uint4 response;
  Slot slots[kSlots];
  Spoiled spoiled;
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
// Shared-memory descriptors, 128-byte swizzle: the upper word is the same for all here (1024 bytes from 8 rows to the next, version 1, the swizzle), the
// lower one has the address and the leading offset: of operands whose rows are M or N (K adjacent), unused; of the one whose rows are K, blocks of 64 columns x 8
// rows, the bytes from 64 columns to the next.
constexpr uint32_t kDescHigh = (1024u >> 4) | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t desc_low(uint32_t saddr, uint32_t leading) { return (saddr & 0x3FFFFu) >> 4 | (leading >> 4) << 16; }
// D (+)= A B, both in shared memory; and with A in TMEM (a lane per row, two 16-bit numbers a column)
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 x, y;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 x, {%1, %5};\n\tmov.b64 y, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc), "n"(kDescHigh) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 y;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "mov.b64 y, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], y, %3, p;\n\t}"
      ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(acc), "n"(kDescHigh) : "memory");
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

// Steps of query tile t of a job: tiles of keys that its rows see.
template <int kTiles>
__device__ __forceinline__ int steps_of(const Job& jb, int t, int causal) {
  const int row0 = (jb.tile * kTiles + t) * kTile, behind = jb.queries - row0, rows = behind < kTile ? behind : kTile;
  int64_t see = causal ? (int64_t)row0 + rows + (jb.keys - jb.queries) : jb.keys;
  see = see < 0 ? 0 : see > jb.keys ? jb.keys : see;
  return rows > 0 ? (int)((see + kTile - 1) / kTile) : 0;
}

// Bounded like mbar_wait, but for as long as a job may take (64 times over), while no other role gave up.
__device__ __forceinline__ bool wait_long(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  for (int i = 0; i < 64; ++i) {
    if (mbar_wait_inline(bar, parity, abort_flag)) return true;
    if (*abort_flag) return false;
  }
  return false;
}

// The same for warps that wait most of a job: asleep in between, since a warp that keeps asking takes issue slots from the rows' warps beside it
// (8192 tokens, 32 heads of 64: 3% with two such warps asking).
__device__ __forceinline__ bool wait_asleep(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  if (mbar_test(bar, parity)) return true;
  const uint64_t deadline = globaltimer() + 64 * kTimeoutNs;
  for (;;) {
    __nanosleep(256);
    if (mbar_test(bar, parity)) return true;
    if (*abort_flag || globaltimer() > deadline) return false;
  }
}

// At the end of a job's row: its mark where an output is not finite (sums of its row's products with 0 are NaN then).
__device__ __forceinline__ void mark_if_spoiled(const uint64_t (&sums)[2], bool live, uint32_t mark) {
  float a, b;
  one_each(add2(sums[0], sums[1]), a, b);
  // (without a branch: the loop around keeps its registers)
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.s32 q, %1, 0;\n\tsetp.neu.and.f32 p, %0, 0f00000000, q;\n\t@p st.shared.u32 [%2], 1;\n\t}" ::"f"(a + b), "r"((int)live), "r"(mark) : "memory");
}
// The block's end: the rows of the kept jobs, and of the last ones that are marked, whose last key lies before a value that is not finite. For the four warps beside the
// rows' (it takes up to 88 registers, of their 104), as a call, with a copy of the arguments: what the compiler does to the jobs' loop for the code here, for a call of theirs, or for one that
// might change the arguments, costs heads of 64 1 to 4% more. (With marks and this against neither: 8192 tokens, 32 heads of 64 247 us and 245, of 128 336 and 336; 200 prompts of up
// to 64 tokens 148 and 143, 155 and 149, of 192 159 and 148, of 256 191 and 184. A look at the values instead, by the warp that clears those behind a sequence: 255, 339; 155, 176, 177, 206.)
template <class T, int D, int kTiles>
static __device__ __noinline__ void take_rows_again(const PromptArgs& p, const Spoiled& spoiled, int warp) {
  for (int i = 0; i < spoiled.count + kMarks; ++i) {
    const int number = i - spoiled.count;  // (behind the kept jobs the last ones)
    if (number >= 0 && !spoiled.mark[number]) continue;
    const Marked& which = number < 0 ? spoiled.jobs[i] : spoiled.last[number];
    const Job jb = which.job;
    const int head = which.head;
    const T* v = static_cast<const T*>(p.v) + (int64_t)jb.kv_start * p.ldv + (int64_t)(head / (p.heads / p.kv_heads)) * p.ldvh;
    for (int t = 0; t < kTiles; ++t) {
      const int first = (jb.tile * kTiles + t) * kTile, end = first + kTile < jb.queries ? first + kTile : jb.queries, keys = steps_of<kTiles>(jb, t, 1) * kTile;
      if (first >= end) break;
      const int last = prompt::last_not_finite<T, D>(prompt::seen_by(jb, first), keys < jb.keys ? keys : jb.keys,
                                                     [&](int key, int c) { return reinterpret_cast<const uint4*>(v + key * p.ldv)[c]; });
      for (int at = first + warp; at < end && prompt::seen_by(jb, at) <= last; at += 4) prompt::attend_again<T, D>(p, jb, head, at);
    }
  }
}

template <class T, int D>
__global__ void __launch_bounds__(kThreads, 1) prompt_tc_kernel(const __grid_constant__ Maps maps, const __grid_constant__ PromptArgs p) {
  constexpr int kBytes = tile_bytes(D), kRing = ring(D), kBoxes = D / 64, kBox = kTile * 128;
  // TMEM: 128 columns for each tile's scores, weights over them, or 192 (see above); then their outputs
  constexpr bool kAhead2 = D == 64;
  constexpr uint32_t kCols = kAhead2 ? 192 : 128, kO = 2 * kCols;
  static_assert(kO + 2 * D <= 512, "");
  extern __shared__ __align__(1024) uint8_t smem[];  // queries of both tiles, the ring of keys and values, Barriers
  Barriers& bar = *reinterpret_cast<Barriers*>(smem + (2 + kRing) * kBytes);
  volatile int* abort_flag = &bar.abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t sq = smem_u32(smem), ring0 = sq + 2 * kBytes;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kRing; ++i) {
      mbar_init(smem_u32(&bar.full[i]), 1);
      mbar_init(smem_u32(&bar.empty[i]), 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(smem_u32(&bar.q_full[t]), 1);
      mbar_init(smem_u32(&bar.q_empty[t]), 1);
      mbar_init(smem_u32(&bar.s_full[t]), 1);
      mbar_init(smem_u32(&bar.p_full[t][0]), 4);
      mbar_init(smem_u32(&bar.p_full[t][1]), 4);
      mbar_init(smem_u32(&bar.o_done[t]), 1);
      mbar_init(smem_u32(&bar.o_free[t]), 4);
      mbar_init(smem_u32(&bar.s_read[t]), 4);
    }
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(smem_u32(&bar.job_full[i]), 1);
      mbar_init(smem_u32(&bar.job_empty[i]), kReaders);
    }
    mbar_init(smem_u32(&bar.last_v), 1);
    mbar_init(smem_u32(&bar.fixed), 1);
    mbar_init(smem_u32(&bar.want), 1);
    mbar_init(smem_u32(&bar.answer), 1);
    for (int i = 0; i < kMarks; ++i) bar.spoiled.mark[i] = 0;
    bar.abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == kWarpMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bar.tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  grid_dep_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *const_cast<volatile uint32_t*>(&bar.tmem);
  const int group = p.heads / p.kv_heads;

  if (warp >= kSoftWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsIssue));
    if (warp == kWarpJobs) {
      // this block's own job first, then others'
      int x = blockIdx.x, y = blockIdx.y, i = 0, kept = 0;
      int seq0 = 0, base = 0, start = 0, queries = 0, tiles = 0, upto = 0;  // 32 sequences, a lane each: tiles of them, and up to the lane's end
      auto load = [&] {
        const int q = seq0 + lane;
        start = queries = 0;
        if (q < p.seqs) {
          start = prompt::clamp_at(p.starts[q], p.tokens);
          const int end = prompt::clamp_at(p.starts[q + 1], p.tokens);
          queries = end > start ? end - start : 0;
        }
        tiles = (queries + 2 * kTile - 1) / (2 * kTile);
        upto = tiles;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int u = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += u;
        }
        upto += base;
      };
      load();
      bool ok = true;
      for (uint32_t asked = 0;; ++asked) {
        // the sequence of unit y, and its tile: the last tiles of a sequence, which see the most keys, first
        if (y < base) { seq0 = base = 0; load(); }
        int end;
        while (y >= (end = __shfl_sync(0xffffffffu, upto, 31)) && seq0 + 32 < p.seqs) {
          base = end;
          seq0 += 32;
          load();
        }
        if (y < end) {
          const int slot = i % kSlots;
          if (!wait_asleep(smem_u32(&bar.job_empty[slot]), (uint32_t)(i / kSlots & 1) ^ 1, abort_flag)) ok = false;
          if (ok && y >= upto - tiles && y < upto) {
            const int q = seq0 + lane;
            const int32_t* ks = p.kv_starts ? p.kv_starts : p.starts;
            const int k0 = prompt::clamp_at(ks[q], p.kv_tokens), k1 = prompt::clamp_at(ks[q + 1], p.kv_tokens);
            const Job jb{1, start, queries, k0, k1 > k0 ? k1 - k0 : 0, upto - 1 - y};
            bar.spoiled.last[i & (kMarks - 1)] = {jb, x};
            bar.slots[slot] = {jb, x, 1, steps_of<2>(jb, 0, p.causal), steps_of<2>(jb, 1, p.causal)};
            mbar_arrive(smem_u32(&bar.job_full[slot]));
          }
          bar.spoiled.keep(i - kSlots - 1, lane, kept);
          if (!ok || !wait_asleep(smem_u32(&bar.want), (uint32_t)i & 1, abort_flag)) { ok = false; break; }
          ++i;
        }
        if (kept >= kSpoiled) break;
        if (lane == 0) {
          fence_proxy_async();  // (the last answer has been read)
          mbar_arrive_expect_tx(smem_u32(&bar.answer), 16);
          asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
                       ::"r"(smem_u32(&bar.response)), "r"(smem_u32(&bar.answer)) : "memory");
        }
        if (!mbar_wait_inline(smem_u32(&bar.answer), asked & 1, abort_flag)) {
          int never = 0;
          if (!mbar_wait_inline(smem_u32(&bar.answer), asked & 1, &never)) ok = false;
        }
        uint32_t taken, nx, ny;
        asm volatile(
            "{\n\t.reg .b128 r;\n\t.reg .pred p;\n\t.reg .b32 z, u;\n\t"
            "ld.shared.b128 r, [%3];\n\t"
            "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t"
            "mov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\t"
            "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, %2, z, u}, r;\n\t}"
            : "=r"(taken), "=r"(nx), "=r"(ny) : "r"(smem_u32(&bar.response)) : "memory");
        __syncwarp();
        if (!taken || !ok) break;
        x = (int)nx;
        y = (int)ny;
      }
      const int slot = i % kSlots;
      if (ok && !wait_asleep(smem_u32(&bar.job_empty[slot]), (uint32_t)(i / kSlots & 1) ^ 1, abort_flag)) ok = false;
      if (!ok) fail(abort_flag, p.status);
      __syncwarp();
      if (lane == 0) {
        bar.slots[slot].valid = 0;
        bar.spoiled.count = kept;
        mbar_arrive(smem_u32(&bar.job_full[slot]));
      }
    }
    if (warp == kWarpTma && elect_one()) {
      uint32_t st = 0, ph = 0, q_phase = 3;  // (q_phase: a bit for each tile, the parity that its next wait has)
      int issued = 0, q_issued[2] = {0, 0};
      bool ok = true;
      auto load = [&](const CUtensorMap* map, int head, int key) {
        if (!mbar_wait(smem_u32(&bar.empty[st]), ph ^ 1, abort_flag)) return false;
        const uint32_t full = smem_u32(&bar.full[st]);
        mbar_arrive_expect_tx(full, kBytes);
#pragma unroll
        for (int b = 0; b < kBoxes; ++b) tma_load_3d(ring0 + st * kBytes + b * kBox, map, b * 64, head, key, full);
        ++issued;
        if (++st == (uint32_t)kRing) { st = 0; ph ^= 1; }
        return true;
      };
      for (int i = 0; ok; ++i) {
        const int slot = i % kSlots;
        if (!wait_asleep(smem_u32(&bar.job_full[slot]), (uint32_t)(i / kSlots) & 1, abort_flag)) { ok = false; break; }
        const Slot sl = bar.slots[slot];
        mbar_arrive(smem_u32(&bar.job_empty[slot]));
        if (!sl.valid) break;
        const int keys = sl.n0 > sl.n1 ? sl.n0 : sl.n1, kvh = sl.head / group;
        // queries of tile 0, the first keys, queries of tile 1: in the order in which their places come free
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if (ok && (t ? sl.n1 : sl.n0) > 0) {
            const uint32_t qf = smem_u32(&bar.q_full[t]);
            if (!mbar_wait(smem_u32(&bar.q_empty[t]), q_phase >> t & 1, abort_flag)) { ok = false; break; }
            q_phase ^= 1u << t;
            ++q_issued[t];
            mbar_arrive_expect_tx(qf, kBytes);
#pragma unroll
            for (int b = 0; b < kBoxes; ++b) tma_load_3d(sq + t * kBytes + b * kBox, &maps.q, b * 64, sl.head, sl.job.start + (sl.job.tile * 2 + t) * kTile, qf);
          }
          if (t == 0 && ok && keys > 0) ok = load(&maps.k, kvh, sl.job.kv_start);
        }
        for (int j = 0; ok && j < keys; ++j) {
          const int key = sl.job.kv_start + j * kTile;
          ok = (j == 0 || load(&maps.k, kvh, key)) && load(&maps.v, kvh, key);
        }
      }
      // the last arrivals at these barriers come before the block ends
      for (int t = 0; ok && t < 2; ++t)
        if (q_issued[t] > 0) ok = mbar_wait(smem_u32(&bar.q_empty[t]), q_phase >> t & 1, abort_flag);
      for (int i = issued > kRing ? issued - kRing : 0; ok && i < issued; ++i) ok = mbar_wait(smem_u32(&bar.empty[i % kRing]), (uint32_t)(i / kRing) & 1, abort_flag);
      if (!ok) {
        fail(abort_flag, p.status);
        int never = 0;  // the copies in flight end before the block does (each of these waits is bounded too)
        for (int t = 0; t < 2; ++t)
          if (q_issued[t] > 0) mbar_wait(smem_u32(&bar.q_full[t]), (uint32_t)(q_issued[t] - 1) & 1, &never);
        for (int i = issued > kRing ? issued - kRing : 0; i < issued; ++i) mbar_wait(smem_u32(&bar.full[i % kRing]), (uint32_t)(i / kRing) & 1, &never);
      }
    }
    if (warp == kWarpMma && elect_one()) {
      constexpr uint32_t type = std::is_same<T, __half>::value ? 0u : (1u << 7) | (1u << 10);
      const uint32_t id_s = idesc_e4m3(kTile) | type, id_o = idesc_e4m3(D) | type | 1u << 16;  // (bit 16: B's rows are K)
      // (This thread's own instructions, at about ten cycles each beside the rows' warps, could bound a step: descriptors move by their low words, places in the
      // ring by additions.)
      const uint32_t dq = desc_low(sq, 16), dk = desc_low(ring0, 16), dv = desc_low(ring0, kBox);
      int slot = 0;
      uint32_t used = 0, ks = 0, kp = 0, vs = 1, vp = 0;  // the job's slot and its use; the next tiles of keys and of values in the ring
      uint32_t q_phase = 0, o_phase = 3, p_phase = 0, fix_phase = 0;
      uint32_t odd = 0, weights = 0, read_phase = 3;  // a bit for each tile: whether its next scores, and products, are those of an odd step
      bool ok = true, begun[2] = {false, false};
      auto scores = [&](int t, uint32_t stage) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
          const uint32_t at = ((s >> 2) * kBox + (s & 3) * 32) >> 4;
          mma_ss(tmem + t * kCols + (kAhead2 ? (odd >> t & 1) * 64 : 0), dq + t * (kBytes >> 4) + at, dk + stage * (kBytes >> 4) + at, id_s, s > 0);
        }
        mma_commit(smem_u32(&bar.s_full[t]));
        if (kAhead2) { odd ^= 1u << t; read_phase ^= 1u << t; }
      };
      // (the rows have read the last step's scores, whose place these take in part)
      auto read = [&](int t) { return !kAhead2 || mbar_poll(smem_u32(&bar.s_read[t]), read_phase >> t & 1, abort_flag); };
      while (ok) {
        if (!wait_long(smem_u32(&bar.job_full[slot]), used, abort_flag)) { ok = false; break; }
        const Slot& sl = bar.slots[slot];
        if (!sl.valid) break;
        const int n0 = sl.n0, n1 = sl.n1, n = n0 > n1 ? n0 : n1, want = n > kAhead ? n - kAhead : 0;
        const bool cut = n * kTile > sl.job.keys;
        mbar_arrive(smem_u32(&bar.job_empty[slot]));
        if (++slot == kSlots) { slot = 0; used ^= 1; }
        if (n == 0) {
          mbar_arrive(smem_u32(&bar.want));
          continue;
        }
        // the first scores, where they were not begun beside the last job's end
        if (!mbar_poll(smem_u32(&bar.full[ks]), kp, abort_flag)) { ok = false; break; }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          if ((t ? n1 : n0) == 0) continue;
          if (!begun[t]) {
            if (!mbar_poll(smem_u32(&bar.q_full[t]), q_phase >> t & 1, abort_flag) || !read(t)) { ok = false; break; }
            tc_fence_after();
            scores(t, ks);
          }
          begun[t] = false;
          q_phase ^= 1u << t;
          if ((t ? n1 : n0) == 1) mma_commit(smem_u32(&bar.q_empty[t]));
        }
        if (!ok) break;
        mma_commit(smem_u32(&bar.empty[ks]));
        ks += 2;
        if (ks >= (uint32_t)kRing) { ks -= kRing; kp ^= 1; }
        for (int j = 0; j < n; ++j) {
          if (j == want) mbar_arrive(smem_u32(&bar.want));
          if (!mbar_poll(smem_u32(&bar.full[vs]), vp, abort_flag)) { ok = false; break; }
          if (cut && j == n - 1) {
            mbar_arrive(smem_u32(&bar.last_v));
            if (!mbar_poll(smem_u32(&bar.fixed), fix_phase, abort_flag)) { ok = false; break; }
            fix_phase ^= 1;
          }
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const int nt = t ? n1 : n0;
            auto products = [&] {
              if (j >= nt) return true;
              if (j == 0) {  // the last job's outputs have been read
                if (!mbar_poll(smem_u32(&bar.o_free[t]), o_phase >> t & 1, abort_flag)) return false;
                o_phase ^= 1u << t;
              }
              const uint32_t even_odd = kAhead2 ? weights >> t & 1 : 0;
              if (!mbar_poll(smem_u32(&bar.p_full[t][even_odd]), p_phase >> (2 * t + even_odd) & 1, abort_flag)) return false;
              p_phase ^= 1u << (2 * t + even_odd);
              tc_fence_after();
              const uint32_t w = tmem + t * kCols + even_odd * 128;
#pragma unroll
              for (int s = 0; s < kTile / 16; ++s) mma_ts(tmem + kO + t * D, w + s * 8, dv + vs * (kBytes >> 4) + (s * 2048 >> 4), id_o, j > 0 || s > 0);
              if (kAhead2) weights ^= 1u << t;
              if (j + 1 == nt || (kAhead2 && j + 2 == nt)) mma_commit(smem_u32(&bar.o_done[t]));
              return true;
            };
            if (!kAhead2 && !products()) { ok = false; break; }
            if (j + 1 < nt) {  // scores of the next step
              if (!mbar_poll(smem_u32(&bar.full[ks]), kp, abort_flag) || !read(t)) { ok = false; break; }
              tc_fence_after();
              scores(t, ks);
              if (j + 2 == nt) mma_commit(smem_u32(&bar.q_empty[t]));
            } else if (j == n - 1 && !begun[t]) {  // or of the next job's first one, if that is known and its copies are there
              const Slot& nx = bar.slots[slot];
              if (mbar_test(smem_u32(&bar.job_full[slot]), used) && nx.valid && (t ? nx.n1 : nx.n0) > 0 && mbar_test(smem_u32(&bar.q_full[t]), q_phase >> t & 1) &&
                  mbar_test(smem_u32(&bar.full[ks]), kp) && (!kAhead2 || mbar_test(smem_u32(&bar.s_read[t]), read_phase >> t & 1))) {
                tc_fence_after();
                scores(t, ks);
                begun[t] = true;
              }
            }
            if (kAhead2 && !products()) { ok = false; break; }
          }
          if (!ok) break;
          mma_commit(smem_u32(&bar.empty[vs]));
          vs += 2;
          if (vs >= (uint32_t)kRing) { vs -= kRing; vp ^= 1; }
          if (j + 1 < n) {
            mma_commit(smem_u32(&bar.empty[ks]));
            ks += 2;
            if (ks >= (uint32_t)kRing) { ks -= kRing; kp ^= 1; }
          }
        }
      }
      if (!ok) fail(abort_flag, p.status);
    }
    if (warp == kWarpFix) {
      uint32_t ring_at = 0, ends = 0;
      for (int i = 0;; ++i) {
        const int slot = i % kSlots;
        if (!wait_asleep(smem_u32(&bar.job_full[slot]), (uint32_t)(i / kSlots) & 1, abort_flag)) break;
        const Slot sl = bar.slots[slot];
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bar.job_empty[slot]));
        if (!sl.valid) break;
        const int keys = sl.n0 > sl.n1 ? sl.n0 : sl.n1;
        ring_at += 2 * keys;
        if (keys * kTile <= sl.job.keys) continue;
        // the last tile's value rows behind the sequence's end are another's: 0 instead, so that weights of 0 meet no NaN
        if (!wait_asleep(smem_u32(&bar.last_v), ends & 1, abort_flag)) break;
        ++ends;
        uint8_t* v = smem + (2 + (ring_at - 1) % kRing) * kBytes;
        for (int r = (sl.job.keys - (keys - 1) * kTile) * 8 + lane; r < kTile * 8; r += 32)
          for (int b = 0; b < kBoxes; ++b) reinterpret_cast<uint4*>(v + b * kBox)[r] = make_uint4(0, 0, 0, 0);
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bar.fixed));
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoft));
    const int t = warp >> 2, row = (warp & 3) * 32 + lane;  // (a warp reads the quarter of TMEM's lanes that its number gives)
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, to = tmem + kO + t * D + lanes;
    const uint32_t marks = smem_u32(bar.spoiled.mark);
    const float c2 = prompt::factor(p.scale), grow = fminf(kGrowth / c2, 3.402823466e38f);
    uint32_t steps = 0, ends = 0;  // this tile's steps so far, and phases of o_done
    const uint32_t tile = tmem + t * kCols + lanes;
    bool ok = true;
    for (int i = 0; ok; ++i) {
      const int slot = i % kSlots;
      if (!wait_long(smem_u32(&bar.job_full[slot]), (uint32_t)(i / kSlots) & 1, abort_flag)) { ok = false; break; }
      const Job jb = bar.slots[slot].job;
      const int head = bar.slots[slot].head, valid = bar.slots[slot].valid, nt = t ? bar.slots[slot].n1 : bar.slots[slot].n0;
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bar.job_empty[slot]));
      if (!valid) break;
      const int at = jb.tile * 2 * kTile + t * kTile + row;  // this thread's row of the sequence
      int64_t see = p.causal ? (int64_t)at + (jb.keys - jb.queries) + 1 : jb.keys;
      const int lim = (int)(see < 0 ? 0 : see > jb.keys ? jb.keys : see);
      float m = -INFINITY, l = 0.0f;
      bool before = false;  // whether the end of the products before the last has been met
      for (int j = 0; j < nt; ++j) {
        if (!mbar_wait_inline(smem_u32(&bar.s_full[t]), steps & 1, abort_flag)) { ok = false; break; }
        const uint32_t ts = tile + (kAhead2 ? (steps & 1) * 64 : 0), tp = tile + (kAhead2 ? (steps & 1) * 128 : 0);
        const uint32_t handed = smem_u32(&bar.p_full[t][kAhead2 ? steps & 1 : 0]);
        ++steps;
        tc_fence_after();
        float s[kTile];
#pragma unroll
        for (int i2 = 0; i2 < kTile; i2 += 32) tmem_ld32(ts + i2, s + i2);
        tmem_wait_ld();
#pragma unroll
        for (int i2 = 0; i2 < kTile; i2 += 32) settle(s + i2);
        if (kAhead2) {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&bar.s_read[t]));
        }
        const int here = lim - j * kTile;  // places of this tile that the row sees
        if (__any_sync(0xffffffffu, here < kTile)) {
#pragma unroll
          for (int i2 = 0; i2 < kTile; ++i2)
            if (i2 >= here) s[i2] = -INFINITY;
        }
        float a[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int i2 = 4; i2 < kTile; i2 += 4)
#pragma unroll
          for (int c = 0; c < 4; ++c) a[c] = fmaxf(a[c], s[i2 + c]);
        const float top = fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3]));
        const bool grew = top > m + grow;  // (from -infinity: any score; `grow` is finite for that)
        if (__any_sync(0xffffffffu, grew)) {
          const float f = grew ? ex2((m - top) * c2) : 1.0f;
          if (grew) m = top;
          l *= f;
          if (j > 0) {
            // The last step's products are done: this step's scores were issued behind them and have arrived; or, where scores run ahead, the next
            // step's are (of which there is none behind the last, where the products tell it themselves).
            if (kAhead2 && j + 1 < nt) {
              if (!mbar_wait_inline(smem_u32(&bar.s_full[t]), steps & 1, abort_flag)) { ok = false; break; }
              tc_fence_after();
            } else if (kAhead2) {
              if (!mbar_wait_inline(smem_u32(&bar.o_done[t]), ends & 1, abort_flag)) { ok = false; break; }
              ++ends;
              before = true;
              tc_fence_after();
            }
#pragma unroll
            for (int i2 = 0; i2 < D; i2 += 16) {
              uint32_t o[16];
              tmem_ld16(to + i2, o);
              tmem_wait_ld();
              reg_fence16(o);
#pragma unroll
              for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * f);
              tmem_st16(to + i2, o);
            }
          }
        }
        float ref = m == -INFINITY ? 0.0f : m;
        // the factor goes into one multiply-add with the maximum, but where scores are so large that its rounding shows
        if (__any_sync(0xffffffffu, fabsf(ref * c2) > 1e5f)) {
#pragma unroll
          for (int i2 = 0; i2 < kTile; ++i2) s[i2] -= ref;
          ref = 0.0f;
        }
        const uint64_t c22 = two_of(c2, c2), r22 = two_of(-ref * c2, -ref * c2);
        uint64_t sum[2] = {0, 0};
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          uint32_t w[16];
#pragma unroll
          for (int i2 = 0; i2 < 16; ++i2) {
            float x, y;
            one_each(fma2(two_of(s[32 * h + 2 * i2], s[32 * h + 2 * i2 + 1]), c22, r22), x, y);
            x = ex2(x);
            y = ex2(y);
            sum[i2 & 1] = add2(sum[i2 & 1], two_of(x, y));
            w[i2] = pack(x, y, (T*)nullptr);
          }
          tmem_st16(tp + 16 * h, w);
        }
        float u, v;
        one_each(add2(sum[0], sum[1]), u, v);
        l += u + v;
        // (every phase of a barrier is met)
        if (kAhead2 && j > 0 && j + 1 == nt && !before) {
          if (!mbar_wait_inline(smem_u32(&bar.o_done[t]), ends & 1, abort_flag)) { ok = false; break; }
          ++ends;
        }
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(handed);
      }
      if (ok && nt > 0 && !mbar_wait_inline(smem_u32(&bar.o_done[t]), ends & 1, abort_flag)) ok = false;
      if (!ok) break;
      ends += nt > 0;
      tc_fence_after();
      const int behind = jb.queries - jb.tile * 2 * kTile - t * kTile;
      const bool live = row < behind;
      const float inv = m == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l;
      T* y = static_cast<T*>(p.out) + (int64_t)(jb.start + at) * p.ldo + (int64_t)head * p.ldoh;
      if (behind > 0) {
        uint64_t zero[2] = {0, 0};
#pragma unroll
        for (int i2 = 0; i2 < D; i2 += 32) {
          float o[32];
          if (nt > 0) {
            tmem_ld32(to + i2, o);
            tmem_wait_ld();
            settle(o);
          } else {
#pragma unroll
            for (int c = 0; c < 32; ++c) o[c] = 0.0f;
          }
          if (i2 + 32 == D && nt > 0) {  // read: the next job's products may come
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bar.o_free[t]));
          }
#pragma unroll
          for (int c = 0; c < 32; c += 2) zero[c >> 1 & 1] = fma2(two_of(o[c], o[c + 1]), 0, zero[c >> 1 & 1]);
          if (live) {
#pragma unroll
            for (int c = 0; c < 32; c += 8)
              *reinterpret_cast<uint4*>(y + i2 + c) = make_uint4(pack(o[c] * inv, o[c + 1] * inv, (T*)nullptr), pack(o[c + 2] * inv, o[c + 3] * inv, (T*)nullptr),
                                                                 pack(o[c + 4] * inv, o[c + 5] * inv, (T*)nullptr), pack(o[c + 6] * inv, o[c + 7] * inv, (T*)nullptr));
          }
        }
        if (live && p.lse) p.lse[(int64_t)(jb.start + at) * p.heads + head] = fmaf(m, c2, log2f(l)) * kLn2;
        mark_if_spoiled(zero, live, marks + (i & (kMarks - 1)) * 4);
      }
    }
    if (!ok) fail(abort_flag, p.status);
    tc_fence_before();
  }
  __syncthreads();
  if (warp >= kSoftWarps && p.causal && !bar.abort_flag && (bar.spoiled.count > 0 || __any_sync(0xffffffffu, bar.spoiled.mark[lane & (kMarks - 1)]))) {
    const PromptArgs copy = p;
    take_rows_again<T, D, 2>(copy, bar.spoiled, warp - kSoftWarps);
  }
  if (warp == kWarpMma) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

// ---------------------------------------------------------------- heads of 192 and 256

// Two such tiles' outputs would leave TMEM no room for scores: a block takes one tile of 128 rows, whose outputs have up to 256 columns, and its scores go
// to the other two times 128 in turn. The tensor cores have the next step's scores, and the last step's products, while the four warps of the rows are at
// their exponentials. Keys and values come in pieces that a product takes whole: 128 x 128 numbers of a head of 256, 128 x 192 of 192. Bound by the products
// (8192 tokens of 32 heads of 256: 639 us, 1,720 TFLOP/s) and, for 192, the rows' chain beside shorter ones (511 us, 1,613). Blocks stay, as above: with
// a block for each job 651 and 534; 13 prompts of up to 2500 tokens, 28 heads of 256: 152 us and 182, 100 prompts of 64 tokens 99 and 163.
struct WideBarriers {
  uint64_t q_full, q_empty, full[8], empty[8], s_full[2], p_full[2], o_done[2], o_free, last_v, fixed, job_full[kSlots], job_empty[kSlots], want, answer;
  alignas(16) uint4 response;
  Slot slots[kSlots];
  Spoiled spoiled;
  uint32_t tmem;
  int abort_flag;
};
__host__ __device__ constexpr int pieces(int dim) { return dim == 256 ? 2 : 1; }
__host__ __device__ constexpr int wide_ring(int dim) { return dim == 256 ? 5 : 3; }
__host__ __device__ constexpr size_t wide_smem(int dim) { return (size_t)tile_bytes(dim) + wide_ring(dim) * (tile_bytes(dim) / pieces(dim)) + sizeof(WideBarriers); }
constexpr int kWideThreads = 256, kWideTma = 4, kWideMma = 5, kWideFix = 6, kWideJobs = 7, kWideReaders = 4 + 3;

// One warp's part: this block's job, and others' of blocks that have not begun, to the slots. (The kernel above has the same written out: its part as a
// function takes 16,384 tokens of 32 heads of 128 from 1,262 to 1,285 us.)
__device__ __forceinline__ void hand_out_jobs(const PromptArgs& p, WideBarriers& bar, volatile int* abort_flag, int lane) {
  // this block's own job first, then others'
  int x = blockIdx.x, y = blockIdx.y, i = 0, kept = 0;
  int seq0 = 0, base = 0, start = 0, queries = 0, tiles = 0, upto = 0;  // 32 sequences, a lane each: tiles of them, and up to the lane's end
  auto load = [&] {
    const int q = seq0 + lane;
    start = queries = 0;
    if (q < p.seqs) {
      start = prompt::clamp_at(p.starts[q], p.tokens);
      const int end = prompt::clamp_at(p.starts[q + 1], p.tokens);
      queries = end > start ? end - start : 0;
    }
    tiles = (queries + kTile - 1) / kTile;
    upto = tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += u;
    }
    upto += base;
  };
  load();
  bool ok = true;
  for (uint32_t asked = 0;; ++asked) {
    // the sequence of unit y, and its tile: the last tiles of a sequence, which see the most keys, first
    if (y < base) { seq0 = base = 0; load(); }
    int end;
    while (y >= (end = __shfl_sync(0xffffffffu, upto, 31)) && seq0 + 32 < p.seqs) {
      base = end;
      seq0 += 32;
      load();
    }
    if (y < end) {
      const int slot = i % kSlots;
      if (!wait_asleep(smem_u32(&bar.job_empty[slot]), (uint32_t)(i / kSlots & 1) ^ 1, abort_flag)) ok = false;
      if (ok && y >= upto - tiles && y < upto) {
        const int q = seq0 + lane;
        const int32_t* ks = p.kv_starts ? p.kv_starts : p.starts;
        const int k0 = prompt::clamp_at(ks[q], p.kv_tokens), k1 = prompt::clamp_at(ks[q + 1], p.kv_tokens);
        const Job jb{1, start, queries, k0, k1 > k0 ? k1 - k0 : 0, upto - 1 - y};
        bar.spoiled.last[i & (kMarks - 1)] = {jb, x};
        bar.slots[slot] = {jb, x, 1, steps_of<1>(jb, 0, p.causal), 0};
        mbar_arrive(smem_u32(&bar.job_full[slot]));
      }
      bar.spoiled.keep(i - kSlots - 1, lane, kept);
      if (!ok || !wait_asleep(smem_u32(&bar.want), (uint32_t)i & 1, abort_flag)) { ok = false; break; }
      ++i;
    }
    if (kept >= kSpoiled) break;
    if (lane == 0) {
      fence_proxy_async();  // (the last answer has been read)
      mbar_arrive_expect_tx(smem_u32(&bar.answer), 16);
      asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];"
                   ::"r"(smem_u32(&bar.response)), "r"(smem_u32(&bar.answer)) : "memory");
    }
    if (!mbar_wait_inline(smem_u32(&bar.answer), asked & 1, abort_flag)) {
      int never = 0;
      if (!mbar_wait_inline(smem_u32(&bar.answer), asked & 1, &never)) ok = false;
    }
    uint32_t taken, nx, ny;
    asm volatile(
        "{\n\t.reg .b128 r;\n\t.reg .pred p;\n\t.reg .b32 z, u;\n\t"
        "ld.shared.b128 r, [%3];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t"
        "mov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, %2, z, u}, r;\n\t}"
        : "=r"(taken), "=r"(nx), "=r"(ny) : "r"(smem_u32(&bar.response)) : "memory");
    __syncwarp();
    if (!taken || !ok) break;
    x = (int)nx;
    y = (int)ny;
  }
  const int slot = i % kSlots;
  if (ok && !wait_asleep(smem_u32(&bar.job_empty[slot]), (uint32_t)(i / kSlots & 1) ^ 1, abort_flag)) ok = false;
  if (!ok) fail(abort_flag, p.status);
  __syncwarp();
  if (lane == 0) {
    bar.slots[slot].valid = 0;
    bar.spoiled.count = kept;
    mbar_arrive(smem_u32(&bar.job_full[slot]));
  }
}

template <class T, int D>
__global__ void __launch_bounds__(kWideThreads, 1) prompt_wide_kernel(const __grid_constant__ Maps maps, const __grid_constant__ PromptArgs p) {
  constexpr int kPieces = pieces(D), kRing = wide_ring(D), kBox = kTile * 128, kBoxes = D / 64 / kPieces, kPiece = kBoxes * kBox;
  constexpr uint32_t kO = 2 * kTile;
  static_assert(kO + D <= 512 && kPieces <= kRing && kRing <= 8, "");
  extern __shared__ __align__(1024) uint8_t smem[];  // queries, the ring of keys and values, WideBarriers
  WideBarriers& bar = *reinterpret_cast<WideBarriers*>(smem + tile_bytes(D) + kRing * kPiece);
  volatile int* abort_flag = &bar.abort_flag;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t sq = smem_u32(smem), ring0 = sq + tile_bytes(D);
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&bar.q_full), 1);
    mbar_init(smem_u32(&bar.q_empty), 1);
    for (int i = 0; i < kRing; ++i) {
      mbar_init(smem_u32(&bar.full[i]), 1);
      mbar_init(smem_u32(&bar.empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&bar.s_full[i]), 1);
      mbar_init(smem_u32(&bar.p_full[i]), 4);
      mbar_init(smem_u32(&bar.o_done[i]), 1);
    }
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(smem_u32(&bar.job_full[i]), 1);
      mbar_init(smem_u32(&bar.job_empty[i]), kWideReaders);
    }
    mbar_init(smem_u32(&bar.o_free), 4);
    mbar_init(smem_u32(&bar.last_v), 1);
    mbar_init(smem_u32(&bar.fixed), 1);
    mbar_init(smem_u32(&bar.want), 1);
    mbar_init(smem_u32(&bar.answer), 1);
    for (int i = 0; i < kMarks; ++i) bar.spoiled.mark[i] = 0;
    bar.abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == kWideMma) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bar.tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  grid_dep_wait();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *const_cast<volatile uint32_t*>(&bar.tmem);
  const int group = p.heads / p.kv_heads;

  if (warp == kWideJobs) hand_out_jobs(p, bar, abort_flag, lane);
  if (warp == kWideTma && elect_one()) {
    uint32_t st = 0, ph = 0, with_keys = 0;  // (with_keys: jobs that have steps so far)
    int issued = 0;
    bool ok = true;
    auto load = [&](const CUtensorMap* map, int kvh, int key) {
#pragma unroll
      for (int c = 0; c < kPieces; ++c) {
        if (!mbar_wait(smem_u32(&bar.empty[st]), ph ^ 1, abort_flag)) { ok = false; return; }
        const uint32_t full = smem_u32(&bar.full[st]);
        mbar_arrive_expect_tx(full, kPiece);
#pragma unroll
        for (int b = 0; b < kBoxes; ++b) tma_load_3d(ring0 + st * kPiece + b * kBox, map, (c * kBoxes + b) * 64, kvh, key, full);
        ++issued;
        if (++st == (uint32_t)kRing) { st = 0; ph ^= 1; }
      }
    };
    for (int i = 0; ok; ++i) {
      const int slot = i % kSlots;
      if (!wait_asleep(smem_u32(&bar.job_full[slot]), (uint32_t)(i / kSlots) & 1, abort_flag)) { ok = false; break; }
      const Slot sl = bar.slots[slot];
      mbar_arrive(smem_u32(&bar.job_empty[slot]));
      if (!sl.valid) break;
      const int n = sl.n0, kvh = sl.head / group;
      if (n == 0) continue;
      if (!mbar_wait(smem_u32(&bar.q_empty), (with_keys & 1) ^ 1, abort_flag)) { ok = false; break; }
      ++with_keys;
      const uint32_t qf = smem_u32(&bar.q_full);
      mbar_arrive_expect_tx(qf, tile_bytes(D));
#pragma unroll
      for (int b = 0; b < D / 64; ++b) tma_load_3d(sq + b * kBox, &maps.q, b * 64, sl.head, sl.job.start + sl.job.tile * kTile, qf);
      // in the order of the products: two steps' scores lead
      for (int j = -2; ok && j < n; ++j) {
        const int key = sl.job.kv_start + j * kTile;
        if (j >= 0) load(&maps.v, kvh, key);
        if (ok && j + 2 < n) load(&maps.k, kvh, key + 2 * kTile);
      }
    }
    // the last arrivals at these barriers come before the block ends
    if (ok && with_keys > 0) ok = mbar_wait(smem_u32(&bar.q_empty), (with_keys - 1) & 1, abort_flag);
    for (int i = issued > kRing ? issued - kRing : 0; ok && i < issued; ++i) ok = mbar_wait(smem_u32(&bar.empty[i % kRing]), (uint32_t)(i / kRing) & 1, abort_flag);
    if (!ok) {
      fail(abort_flag, p.status);
      int never = 0;  // the copies in flight end before the block does (each of these waits is bounded too)
      if (with_keys > 0) mbar_wait(smem_u32(&bar.q_full), (with_keys - 1) & 1, &never);
      for (int i = issued > kRing ? issued - kRing : 0; i < issued; ++i) mbar_wait(smem_u32(&bar.full[i % kRing]), (uint32_t)(i / kRing) & 1, &never);
    }
  }
  if (warp == kWideMma && elect_one()) {
    constexpr uint32_t type = std::is_same<T, __half>::value ? 0u : (1u << 7) | (1u << 10);
    const uint32_t id_s = idesc_e4m3(kTile) | type, id_o = idesc_e4m3(kBoxes * 64) | type | 1u << 16;  // (bit 16: B's rows are K)
    const uint32_t dq = desc_low(sq, 16), dk = desc_low(ring0, 16), dv = desc_low(ring0, kBox);
    uint32_t st = 0, ph = 0, base = 0, with_keys = 0, fix_phase = 0;  // (base: steps of the jobs so far)
    bool ok = true;
    auto there = [&] {
      ok = ok && mbar_poll(smem_u32(&bar.full[st]), ph, abort_flag);
      tc_fence_after();
      return ok;
    };
    auto used = [&] {
      mma_commit(smem_u32(&bar.empty[st]));
      if (++st == (uint32_t)kRing) { st = 0; ph ^= 1; }
    };
    for (int i = 0; ok; ++i) {
      const int slot = i % kSlots;
      if (!wait_long(smem_u32(&bar.job_full[slot]), (uint32_t)(i / kSlots) & 1, abort_flag)) { ok = false; break; }
      const int valid = bar.slots[slot].valid, n = bar.slots[slot].n0, want = n > kAhead ? n - kAhead : 0;
      const bool cut = n * kTile > bar.slots[slot].job.keys;  // the last step's tile ends behind the sequence
      mbar_arrive(smem_u32(&bar.job_empty[slot]));
      if (!valid) break;
      if (n == 0) {
        mbar_arrive(smem_u32(&bar.want));
        continue;
      }
      auto scores = [&](int j) {
        const uint32_t odd = (base + j) & 1;
#pragma unroll
        for (int c = 0; c < kPieces; ++c) {
          if (!there()) return;
#pragma unroll
          for (int s = 0; s < kBoxes * 4; ++s) {
            const uint32_t at = ((s >> 2) * kBox + (s & 3) * 32) >> 4;
            mma_ss(tmem + odd * kTile, dq + c * (kPiece >> 4) + at, dk + st * (kPiece >> 4) + at, id_s, c > 0 || s > 0);
          }
          used();
        }
        mma_commit(smem_u32(&bar.s_full[odd]));
        if (j + 1 == n) mma_commit(smem_u32(&bar.q_empty));
      };
      if (!mbar_poll(smem_u32(&bar.q_full), with_keys & 1, abort_flag)) { ok = false; break; }
      scores(0);
      if (ok && n > 1) scores(1);
      for (int j = 0; ok && j < n; ++j) {
        const uint32_t step = base + j, odd = step & 1;
        if (j == want) mbar_arrive(smem_u32(&bar.want));
        if (cut && j == n - 1) {
          // (all of the last values: the pieces behind this one are in the next places)
#pragma unroll
          for (int c = 0; c < kPieces; ++c) {
            const bool over = st + c >= (uint32_t)kRing;
            ok = ok && mbar_poll(smem_u32(&bar.full[over ? st + c - kRing : st + c]), over ? ph ^ 1 : ph, abort_flag);
          }
          if (ok) mbar_arrive(smem_u32(&bar.last_v));
          ok = ok && mbar_poll(smem_u32(&bar.fixed), fix_phase, abort_flag);
          fix_phase ^= 1;
        }
        // (the last job's outputs have been read)
        if (j == 0) ok = ok && mbar_poll(smem_u32(&bar.o_free), (with_keys & 1) ^ 1, abort_flag);
        ok = ok && mbar_poll(smem_u32(&bar.p_full[odd]), (step >> 1) & 1, abort_flag);
#pragma unroll
        for (int c = 0; c < kPieces; ++c) {
          if (!there()) break;
#pragma unroll
          for (int s = 0; s < kTile / 16; ++s)
            mma_ts(tmem + kO + c * (kBoxes * 64), tmem + odd * kTile + s * 8, dv + st * (kPiece >> 4) + (s * 2048 >> 4), id_o, j > 0 || s > 0);
          used();
        }
        if (!ok) break;
        mma_commit(smem_u32(&bar.o_done[odd]));
        if (j + 2 < n) scores(j + 2);
      }
      base += n;
      ++with_keys;
    }
    if (!ok) fail(abort_flag, p.status);
  }
  if (warp == kWideFix) {
    uint32_t ring_at = 0, ends = 0;
    for (int i = 0;; ++i) {
      const int slot = i % kSlots;
      if (!wait_asleep(smem_u32(&bar.job_full[slot]), (uint32_t)(i / kSlots) & 1, abort_flag)) break;
      const Slot sl = bar.slots[slot];
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bar.job_empty[slot]));
      if (!sl.valid) break;
      const int n = sl.n0;
      ring_at += 2 * n * kPieces;
      if (n * kTile <= sl.job.keys) continue;
      // the last tile's value rows behind the sequence's end are another's: 0 instead, so that weights of 0 meet no NaN
      if (!wait_asleep(smem_u32(&bar.last_v), ends & 1, abort_flag)) break;
      ++ends;
      for (int c = 1; c <= kPieces; ++c) {
        uint8_t* v = smem + tile_bytes(D) + (ring_at - c) % kRing * kPiece;
        for (int r = (sl.job.keys - (n - 1) * kTile) * 8 + lane; r < kTile * 8; r += 32)
          for (int b = 0; b < kBoxes; ++b) reinterpret_cast<uint4*>(v + b * kBox)[r] = make_uint4(0, 0, 0, 0);
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bar.fixed));
    }
  }
  if (warp < 4) {
    const int row = warp * 32 + lane;  // this thread's row of the tile
    const uint32_t lanes = (uint32_t)(warp * 32) << 16, to = tmem + kO + lanes;
    const uint32_t marks = smem_u32(bar.spoiled.mark);
    const float c2 = prompt::factor(p.scale), grow = fminf(kGrowth / c2, 3.402823466e38f);
    uint32_t base = 0;
    bool ok = true;
    for (int i = 0; ok; ++i) {
      const int slot = i % kSlots;
      if (!wait_long(smem_u32(&bar.job_full[slot]), (uint32_t)(i / kSlots) & 1, abort_flag)) { ok = false; break; }
      const Job jb = bar.slots[slot].job;
      const int head = bar.slots[slot].head, valid = bar.slots[slot].valid, n = bar.slots[slot].n0;
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bar.job_empty[slot]));
      if (!valid) break;
      const int at = jb.tile * kTile + row;  // and of the sequence
      int64_t see = p.causal ? (int64_t)at + (jb.keys - jb.queries) + 1 : jb.keys;
      const int lim = (int)(see < 0 ? 0 : see > jb.keys ? jb.keys : see);
      float m = -INFINITY, l = 0.0f;
      auto products = [&](uint32_t step) { return mbar_wait_inline(smem_u32(&bar.o_done[step & 1]), (step >> 1) & 1, abort_flag); };
      for (int j = 0; j < n; ++j) {
        const uint32_t step = base + j, ts = tmem + (step & 1) * kTile + lanes;
        if (!mbar_wait_inline(smem_u32(&bar.s_full[step & 1]), (step >> 1) & 1, abort_flag)) { ok = false; break; }
        // (every phase of a barrier is met: these products came before the scores)
        if (j >= 2 && !products(step - 2)) { ok = false; break; }
        tc_fence_after();
        float s[kTile];
#pragma unroll
        for (int k = 0; k < kTile; k += 32) tmem_ld32(ts + k, s + k);
        tmem_wait_ld();
#pragma unroll
        for (int k = 0; k < kTile; k += 32) settle(s + k);
        const int here = lim - j * kTile;  // places of this tile that the row sees
        if (__any_sync(0xffffffffu, here < kTile)) {
#pragma unroll
          for (int k = 0; k < kTile; ++k)
            if (k >= here) s[k] = -INFINITY;
        }
        float a[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int k = 4; k < kTile; k += 4)
#pragma unroll
          for (int c = 0; c < 4; ++c) a[c] = fmaxf(a[c], s[k + c]);
        const float top = fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3]));
        const bool grew = top > m + grow;  // (from -infinity: any score; `grow` is finite for that)
        if (__any_sync(0xffffffffu, grew)) {
          const float f = grew ? ex2((m - top) * c2) : 1.0f;
          if (grew) m = top;
          l *= f;
          if (j > 0) {
            // (the last step's products come behind these scores)
            if (!products(step - 1)) { ok = false; break; }
            tc_fence_after();
#pragma unroll
            for (int k = 0; k < D; k += 16) {
              uint32_t o[16];
              tmem_ld16(to + k, o);
              tmem_wait_ld();
              reg_fence16(o);
#pragma unroll
              for (int c = 0; c < 16; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * f);
              tmem_st16(to + k, o);
            }
          }
        }
        float ref = m == -INFINITY ? 0.0f : m;
        // the factor goes into one multiply-add with the maximum, but where scores are so large that its rounding shows
        if (__any_sync(0xffffffffu, fabsf(ref * c2) > 1e5f)) {
#pragma unroll
          for (int k = 0; k < kTile; ++k) s[k] -= ref;
          ref = 0.0f;
        }
        const uint64_t c22 = two_of(c2, c2), r22 = two_of(-ref * c2, -ref * c2);
        uint64_t sum[2] = {0, 0};
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          uint32_t w[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            float x, y;
            one_each(fma2(two_of(s[32 * h + 2 * k], s[32 * h + 2 * k + 1]), c22, r22), x, y);
            x = ex2(x);
            y = ex2(y);
            sum[k & 1] = add2(sum[k & 1], two_of(x, y));
            w[k] = pack(x, y, (T*)nullptr);
          }
          tmem_st16(ts + 16 * h, w);
        }
        float u, v;
        one_each(add2(sum[0], sum[1]), u, v);
        l += u + v;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bar.p_full[step & 1]));
      }
      for (int j = n > 1 ? n - 2 : 0; ok && j < n; ++j) ok = products(base + j);
      if (!ok) break;
      base += n;
      tc_fence_after();
      const bool live = at < jb.queries;
      const float inv = m == -INFINITY && l == 0.0f ? 0.0f : 1.0f / l;
      T* y = static_cast<T*>(p.out) + (int64_t)(jb.start + at) * p.ldo + (int64_t)head * p.ldoh;
      uint64_t zero[2] = {0, 0};
#pragma unroll
      for (int k = 0; k < D; k += 32) {
        float o[32];
        if (n > 0) {
          tmem_ld32(to + k, o);
          tmem_wait_ld();
          settle(o);
        } else {
#pragma unroll
          for (int c = 0; c < 32; ++c) o[c] = 0.0f;
        }
        if (k + 32 == D && n > 0) {  // read: the next job's products may come
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&bar.o_free));
        }
#pragma unroll
        for (int c = 0; c < 32; c += 2) zero[c >> 1 & 1] = fma2(two_of(o[c], o[c + 1]), 0, zero[c >> 1 & 1]);
        if (live) {
#pragma unroll
          for (int c = 0; c < 32; c += 8)
            *reinterpret_cast<uint4*>(y + k + c) = make_uint4(pack(o[c] * inv, o[c + 1] * inv, (T*)nullptr), pack(o[c + 2] * inv, o[c + 3] * inv, (T*)nullptr),
                                                              pack(o[c + 4] * inv, o[c + 5] * inv, (T*)nullptr), pack(o[c + 6] * inv, o[c + 7] * inv, (T*)nullptr));
        }
      }
      if (live && p.lse) p.lse[(int64_t)(jb.start + at) * p.heads + head] = fmaf(m, c2, log2f(l)) * kLn2;
      mark_if_spoiled(zero, live, marks + (i & (kMarks - 1)) * 4);
    }
    if (!ok) fail(abort_flag, p.status);
    tc_fence_before();
  }
  __syncthreads();
  if (warp >= 4 && p.causal && !bar.abort_flag && (bar.spoiled.count > 0 || __any_sync(0xffffffffu, bar.spoiled.mark[lane & (kMarks - 1)]))) {
    const PromptArgs copy = p;
    take_rows_again<T, D, 1>(copy, bar.spoiled, warp - 4);
  }
  if (warp == kWideMma) {
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
  constexpr bool kWide = D > 128;
  constexpr size_t smem = kWide ? wide_smem(D) : (2 + ring(D)) * tile_bytes(D) + sizeof(Barriers);
  static_assert(smem <= kSmemLimit, "");
  void (*kernel)(Maps, PromptArgs);
  if constexpr (kWide) kernel = prompt_wide_kernel<T, D>;
  else kernel = prompt_tc_kernel<T, D>;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)a.heads, (unsigned)(a.tokens / job_rows(D) + a.seqs));
  cfg.blockDim = dim3(kWide ? kWideThreads : kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, maps, a);
}
template <class T>
static cudaError_t run_type(const PromptArgs& a, const Maps& maps, cudaStream_t stream) {
  switch (a.dim) {
    case 64: return run<T, 64>(a, maps, stream);
    case 128: return run<T, 128>(a, maps, stream);
    case 192: return run<T, 192>(a, maps, stream);
    default: return run<T, 256>(a, maps, stream);
  }
}

}  // namespace prompttc

bool prompt_tc_takes(const PromptArgs& a) {
  // strides that a tensor map can hold; blocks along the grid's second axis
  const int64_t most = 1LL << 38;
  const int64_t ld[6] = {a.ldq, a.ldqh, a.ldk, a.ldkh, a.ldv, a.ldvh};
  for (int i = 0; i < 6; ++i)
    if (ld[i] < 1 || ld[i] > most) return false;
  return a.kv_tokens > 0 && a.tokens / prompttc::job_rows(a.dim) + a.seqs <= 65535;
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
  const cudaError_t e = half ? run_type<__half>(a, maps, stream) : run_type<__nv_bfloat16>(a, maps, stream);
  if (e == cudaSuccess) return 0;
  *err = std::string("prompt attention: ") + cudaGetErrorString(e);
  return AQD_ERR_CUDA;
}

}  // namespace aqd
