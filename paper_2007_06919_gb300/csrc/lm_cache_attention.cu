// lm_cache_attention.cu -- attention of each sequence's last tokens over the 4-bit cache.
//
// A cached key is k = z + s n (n the 4-bit codes), so q . k = s (q . n) + z sum(q); an output is sum_t p_t v_t = sum_t (p_t s_t) n_t +
// sum_t p_t z_t. Codes meet the matrix instructions as they are: a nibble under the float16 exponent of 64 is 64 + n, one shift and one
// logic operation for two of them, and in a score the 64 leaves as -64 sum(q) in the first accumulator. Steps and lowest
// values act once per place, not once per value. Value codes lose 72 first (n - 8, the lowest value raised by 8 steps in turn): their
// weighted sums over a long cache are small against what 64 + n adds up to, and the matrix instructions' sums cut instead of rounding
// (200,001 places, float16: 1.5e-3 off the exact output that way, 2.6e-4 this way, of which rounding it takes 2.1e-4).
//
// Bound by the cache's bytes: 136 for a place and head of 128 (key and value), which 6.8 TB/s bring to an SM in 6 cycles, 23 issue slots of its
// four schedulers. So the products are transposed, with the places (keys) or channels (values) as the 16 rows of mma.m16n8k16 and 8
// query rows as its columns: a group's heads fill them, where the usual form would pad them to 16, and codes go from shared memory into operand
// registers with no exchange between lanes. (tcgen05 would want the expanded codes in shared memory or TMEM first, and its 128 rows mostly empty.)
//
// A block takes one key-value head, 8 or 16 rows (queries x heads of the group) and a run of places; its 8 warps take steps of 32 places in turn,
// each with its own ring of bulk copies (a step is one or two runs of bytes in the cache), and join at the end. The run's length follows from all
// sequences' lengths, so the blocks are even however these differ; parts of one sequence are joined by combine_kernel.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/aqd.h"
#include "common.cuh"
#include "kernels.h"
#include "lm_seq.cuh"
#include "tc_ptx.cuh"

namespace aqd {
namespace cacheattn {

using namespace tc;

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kStep = 32;                 // places of a step
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__host__ __device__ constexpr int stage_bytes(int dim) { return 2 * 16 * (dim + 8); }
__host__ __device__ constexpr int stages(int dim) { return dim == 64 ? 6 : dim == 192 ? 4 : 3; }
__host__ __device__ constexpr int row_tiles(int dim) { return dim <= 128 ? 2 : 1; }  // most tiles of 8 rows a block

struct Split {
  int32_t units;        // blocks of a key-value head that fill the GPU
  int32_t tiles;        // bound of the row tiles of all sequences
  int32_t group;        // query heads of a key-value head
  uint64_t group_magic;
  int32_t q_vec;        // rows of q on 16 bytes
  int32_t* meta;        // [1 + 8 * tiles]
  float* part;          // [unit][kv head][row]: dim sums, then maximum, sum, factor
};

__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put(__half* y, float v) { *y = __float2half_rn(v); }
__device__ __forceinline__ void put(__nv_bfloat16* y, float v) { *y = __float2bfloat16_rn(v); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}
// nibble j of each 16-bit half, as the float16 numbers 64 + n
template <int j>
__device__ __forceinline__ uint32_t nibbles(uint32_t w) {
  const uint32_t x = j == 0 ? w << 4 : j == 1 ? w : j == 2 ? w >> 4 : w >> 8;
  return (x & 0x00f000f0u) | 0x54005400u;
}
// the same less 8, exactly: n - 8
template <int j>
__device__ __forceinline__ uint32_t centred(uint32_t w) {
  uint32_t y;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(y) : "r"(nibbles<j>(w)), "r"(0x54805480u));
  return y;
}
template <int kWords>
__device__ __forceinline__ void lds(uint32_t addr, uint32_t (&w)[kWords]) {
  if constexpr (kWords % 4 == 0) {
#pragma unroll
    for (int i = 0; i < kWords; i += 4)
      asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]) : "r"(addr + 4 * i));
  } else if constexpr (kWords % 2 == 0) {
#pragma unroll
    for (int i = 0; i < kWords; i += 2) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[i]), "=r"(w[i + 1]) : "r"(addr + 4 * i));
  } else {
#pragma unroll
    for (int i = 0; i < kWords; ++i) asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[i]) : "r"(addr + 4 * i));
  }
}
__device__ __forceinline__ float low_of(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float step_of(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

struct Job {
  int32_t seq, tile, chunk, chunks, first_unit, ordinal, start, queries, len, steps;  // steps: of a chunk
};

// A sequence's queries, first token and length, within what the caller's tensors hold.
__device__ __forceinline__ void sequence(const CacheAttnArgs& p, int s, int& start, int& queries, int& len) {
  start = s;
  queries = 1;
  if (p.starts) {
    const int64_t a = p.starts[s], b = p.starts[s + 1];
    start = (int)(a < 0 ? 0 : a > p.tokens ? p.tokens : a);
    const int64_t e = b > p.tokens ? p.tokens : b;
    queries = e > start ? (int)(e - start) : 0;
  }
  const int64_t most = (int64_t)p.columns << p.cache.page_shift;
  const int n = p.lengths[s];
  len = n < 0 ? 0 : n > most ? (int)most : n;
}

// The unit of this block: its sequence, row tile and run of places. False where there are fewer units.
__device__ bool find_job(const CacheAttnArgs& p, const Split& sp, int rows, int unit, Job* job, uint64_t* red) {
  // steps of all tiles, and from them the steps of a run: whole rounds of the warps
  uint64_t work = 0, before;
  for (int b = 0; b < p.seqs; b += kThreads) {
    uint64_t v = 0;
    if (b + (int)threadIdx.x < p.seqs) {
      int start, n, len;
      sequence(p, b + threadIdx.x, start, n, len);
      v = (uint64_t)((n * (int64_t)sp.group + rows - 1) / rows) * (uint64_t)((len + kStep - 1) / kStep);
    }
    work += seq::block_scan(v, red, before);
  }
  const int64_t per = (int64_t)((work + sp.units - 1) / sp.units);
  const int steps = (int)((per < 1 ? 1 : per) + kWarps - 1) / kWarps * kWarps;
  if (threadIdx.x == 0) job->chunks = 0;
  uint64_t base = 0;
  for (int b = 0; b < p.seqs; b += kThreads) {
    uint64_t v = 0;
    int start = 0, n = 0, len = 0, tiles = 0, chunks = 1;
    if (b + (int)threadIdx.x < p.seqs) {
      sequence(p, b + threadIdx.x, start, n, len);
      tiles = (int)((n * (int64_t)sp.group + rows - 1) / rows);
      chunks = (int)(((len + kStep - 1) / kStep + (int64_t)steps - 1) / steps);
      if (chunks < 1) chunks = 1;
      v = (uint64_t)tiles << 32 | (uint32_t)(tiles * chunks);
    }
    const uint64_t total = seq::block_scan(v, red, before);
    const int first = (int)(uint32_t)(base + before), ordinal = (int)((base + before) >> 32);
    if (unit >= first && unit < first + tiles * chunks && ordinal + (unit - first) / chunks < sp.tiles) {
      const int tile = (unit - first) / chunks;
      *job = {b + (int)threadIdx.x, tile, unit - first - tile * chunks, chunks, first + tile * chunks, ordinal + tile, start, n, len, steps};
    }
    base += total;
  }
  // (starts that fall make more units than there are blocks: nothing is joined then)
  if (unit == 0 && blockIdx.y == 0 && threadIdx.x == 0) sp.meta[0] = (uint32_t)base <= gridDim.x && (base >> 32) <= (uint64_t)sp.tiles ? (int)(base >> 32) : 0;
  __syncthreads();
  return job->chunks > 0;
}

template <class T, int D, int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 && D <= 128 ? 2 : 1)
cache_attention_kernel(const __grid_constant__ CacheAttnArgs p, const __grid_constant__ Split sp) {
  constexpr int kStages = stages(D), kStage = stage_bytes(D), kBlock = kStage / 2, kRows = 8 * NT;
  constexpr int KW = D / 32, VW = D / 64;  // words of a key row, and of a value row, that a lane reads
  extern __shared__ __align__(128) uint8_t smem[];  // [warp][stage]; at the end the warps' sums
  __shared__ uint64_t bars[kWarps * kStages], red[kWarps];
  __shared__ Job job;
  __shared__ int abort_word;
  __shared__ float wm[kWarps][kRows], wl[kWarps][kRows], wc[kRows];  // maxima, sums; rows' factors of scores
  volatile int* abort_flag = &abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  if (threadIdx.x < kWarps * kStages) mbar_init(smem_u32(&bars[threadIdx.x]), 1);
  if (threadIdx.x == 0) {
    abort_word = 0;
    fence_barrier_init();
  }
  grid_dep_wait();
  if (!find_job(p, sp, kRows, blockIdx.x, &job, red)) return;
  const int head = blockIdx.y;
  const Job jb = job;
  if (jb.chunk == 0 && head == 0 && threadIdx.x == 0) {
    int* m = sp.meta + 4 + 4 * jb.ordinal;
    m[0] = jb.first_unit; m[1] = jb.chunks; m[2] = jb.start; m[3] = jb.tile;
    sp.meta[4 + 4 * sp.tiles + jb.ordinal] = jb.queries;
  }

  // this lane's query rows (column g of each tile) as float16 with a power of two in front; the sums and factors of columns 2q, 2q + 1
  uint32_t qf[NT][KW][4];
  float qs[NT][2], c2[NT][2];
  int lim[NT][2], lim_all = 0, lim_any = 0;  // places that a column sees; the least of the tile's rows, the most
  const int last_row = jb.queries * sp.group - jb.tile * kRows;  // rows of this tile and behind it
  {
    const int j0 = fast_div(jb.tile * kRows, sp.group_magic);
    const int top = last_row < kRows ? last_row : kRows, j1 = fast_div(jb.tile * kRows + top - 1, sp.group_magic);
    lim_all = jb.len - jb.queries + j0 + 1;
    lim_any = jb.len - jb.queries + j1 + 1;
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int r = t * 8 + g;
    float f[KW][8], top = 0.0f, sum = 0.0f;
    const bool live = r < last_row;
    const int j = fast_div(jb.tile * kRows + r, sp.group_magic), h = jb.tile * kRows + r - j * sp.group;
    const T* x = static_cast<const T*>(p.q) + (live ? (int64_t)(jb.start + j) * p.ldq + (int64_t)(head * sp.group + h) * p.ldqh : 0) + q * (D / 4);
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      if (live && sp.q_vec) {
        const uint4 v = *reinterpret_cast<const uint4*>(x + 8 * w);
        const T* e = reinterpret_cast<const T*>(&v);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[w][i] = to_f32(e[i]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[w][i] = live ? to_f32(x[8 * w + i]) : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(f[w][i]));
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // the row's largest to [2^14, 2^15)
    int e = 268 - (int)(__float_as_uint(top) >> 23);
    e = top == 0.0f ? 127 : e > 253 ? 253 : e;
    const float up = __uint_as_float((uint32_t)e << 23), down = p.scale * kLog2e * __uint_as_float((uint32_t)(254 - e) << 23);
#pragma unroll
    for (int w = 0; w < KW; ++w) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __half2 h2 = __floats2half2_rn(f[w][i] * up, f[w][i + 4] * up);
        qf[t][w][i] = *reinterpret_cast<const uint32_t*>(&h2);
        sum += __low2float(h2) + __high2float(h2);
      }
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      qs[t][c] = __shfl_sync(0xffffffffu, sum, (2 * q + c) * 4);
      c2[t][c] = fmaxf(__shfl_sync(0xffffffffu, down, (2 * q + c) * 4), 1.4e-45f);
      const int rr = jb.tile * kRows + t * 8 + 2 * q + c;
      lim[t][c] = t * 8 + 2 * q + c < last_row ? jb.len - jb.queries + fast_div(rr, sp.group_magic) + 1 : 0;
    }
  }

  // this warp's steps of the run: step0 + warp, step0 + warp + kWarps, ... while before the last place that a row sees
  const int step0 = jb.chunk * jb.steps;
  int end = (lim_any + kStep - 1) / kStep;  // (lim_any <= 0: none)
  end = end < step0 + jb.steps ? end : step0 + jb.steps;
  const int mine = end > step0 + warp ? (end - step0 - warp + kWarps - 1) / kWarps : 0;
  const int blocks_of_page = 1 << (p.cache.page_shift - 4);
  const int32_t* table = p.table + (int64_t)jb.seq * p.ld_table;
  const uint32_t ring = smem_u32(smem) + warp * (kStages * kStage), bar0 = smem_u32(&bars[warp * kStages]);
  int page0 = -1, page1 = -1;  // of step `lane` of the batch of 32 steps that is being issued
  uint32_t there = 0;          // two bits a stage: its blocks were copied
  __syncwarp();

  auto issue = [&](int i) {
    const int st = i % kStages;
    if ((i & 31) == 0) {
      const int place = (step0 + warp + kWarps * (i + lane)) * kStep;
      page0 = i + lane < mine ? table[place >> p.cache.page_shift] : -1;
      page1 = i + lane < mine && place + 16 < lim_any ? table[(place + 16) >> p.cache.page_shift] : -1;
      if (page0 < 0 || page0 >= p.cache.pages) page0 = -1;
      if (page1 < 0 || page1 >= p.cache.pages) page1 = -1;
    }
    const int a = __shfl_sync(0xffffffffu, page0, i & 31), b = __shfl_sync(0xffffffffu, page1, i & 31);
    there = (there & ~(3u << (2 * st))) | (uint32_t)((a >= 0 ? 1 : 0) | (b >= 0 ? 2 : 0)) << (2 * st);
    if (lane == 0) {
      const int blk = (step0 + warp + kWarps * i) * 2;
      const uint32_t dst = ring + st * kStage, bar = bar0 + 8 * st;
      mbar_arrive_expect_tx(bar, (uint32_t)((a >= 0) + (b >= 0)) * kBlock);
      if (a >= 0) {
        const uint8_t* src = p.cache.data + (((int64_t)a * p.cache.kv_heads + head) * blocks_of_page + (blk & (blocks_of_page - 1))) * kBlock;
        bulk_load(dst, src, a == b && blocks_of_page > 1 ? kStage : kBlock, bar);
      }
      if (b >= 0 && !(a == b && blocks_of_page > 1)) {
        const uint8_t* src = p.cache.data + (((int64_t)b * p.cache.kv_heads + head) * blocks_of_page + ((blk + 1) & (blocks_of_page - 1))) * kBlock;
        bulk_load(dst + kBlock, src, kBlock, bar);
      }
    }
  };

  float o[NT][D / 16][4], m[NT][2], l[NT][2], zs[NT][2];
  // the value steps' power of two: weights p s reach float16 times `up_v`, so that the largest step lies in [2^14, 2^15); an exponent
  // field, which only falls (0: no step so far)
  int up_v = 0;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) o[t][i][c] = 0.0f;
#pragma unroll
    for (int c = 0; c < 2; ++c) { m[t][c] = -INFINITY; l[t][c] = 0.0f; zs[t][c] = 0.0f; }
  }
  __syncthreads();  // barriers are set up
  for (int i = 0; i < kStages - 1 && i < mine; ++i) issue(i);
  int done = 0;
  bool ok = true;
  for (; done < mine; ++done) {
    const int i = done, st = i % kStages;
    if (i + kStages - 1 < mine) issue(i + kStages - 1);  // (the stage that the last step freed: every lane has read it)
    if (!mbar_wait(bar0 + 8 * st, (uint32_t)(i / kStages) & 1, abort_flag)) { ok = false; break; }
    const uint32_t base = ring + st * kStage;
    const int place = (step0 + warp + kWarps * i) * kStep;
    const uint32_t here = there >> (2 * st) & 3u;
    const bool edge = place + kStep > lim_all || here != 3u;
    float x[2][NT][4];
    uint32_t vz[2][2];
    float steps_top = 0.0f;
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint32_t blk = base + b * kBlock;
      uint32_t k0[KW], k1[KW], kz[2];
      lds<KW>(blk + g * (D / 2) + q * (D / 8), k0);
      lds<KW>(blk + (g + 8) * (D / 2) + q * (D / 8), k1);
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(kz[0]) : "r"(blk + 16 * D + 4 * g));
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(kz[1]) : "r"(blk + 16 * D + 4 * g + 32));
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(vz[b][0]) : "r"(blk + 16 * D + 64 + 4 * g));
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(vz[b][1]) : "r"(blk + 16 * D + 64 + 4 * g + 32));
      float acc[NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        acc[t][0] = acc[t][2] = -64.0f * qs[t][0];
        acc[t][1] = acc[t][3] = -64.0f * qs[t][1];
      }
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        {
          const uint32_t a0 = nibbles<0>(k0[w]), a1 = nibbles<0>(k1[w]), a2 = nibbles<1>(k0[w]), a3 = nibbles<1>(k1[w]);
#pragma unroll
          for (int t = 0; t < NT; ++t) mma(acc[t], a0, a1, a2, a3, qf[t][w][0], qf[t][w][1]);
        }
        {
          const uint32_t a0 = nibbles<2>(k0[w]), a1 = nibbles<2>(k1[w]), a2 = nibbles<3>(k0[w]), a3 = nibbles<3>(k1[w]);
#pragma unroll
          for (int t = 0; t < NT; ++t) mma(acc[t], a0, a1, a2, a3, qf[t][w][2], qf[t][w][3]);
        }
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c) x[b][t][c] = fmaf(acc[t][c], step_of(kz[c >> 1]), low_of(kz[c >> 1]) * qs[t][c & 1]);
      if (edge) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = place + 16 * b + 8 * h + g;
          const bool gone = !(here >> b & 1);
          if (gone || at >= lim_any) vz[b][h] = 0u;  // a stale place's step and lowest value count nowhere
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < 2; ++c)
              if (gone || at >= lim[t][c]) x[b][t][2 * h + c] = -INFINITY;
        }
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float s = step_of(vz[b][h]);
        if (s < INFINITY) steps_top = fmaxf(steps_top, s);
      }
    }
    // new maxima, of each column's scores and of the value steps; what was summed so far is brought to them
    const int top_e = (int)(__reduce_max_sync(0xffffffffu, __float_as_uint(steps_top)) >> 23);
    const int up_new = top_e == 0 ? up_v : top_e < 15 ? 253 : 268 - top_e;
    float mx[NT][2];
    bool grew = up_new < up_v || up_v == 0;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float v = fmaxf(fmaxf(x[0][t][c], x[0][t][c + 2]), fmaxf(x[1][t][c], x[1][t][c + 2]));
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
        v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
        mx[t][c] = fmaxf(m[t][c], v);
        grew = grew || mx[t][c] > m[t][c];
      }
    if (__any_sync(0xffffffffu, grew)) {
      float fs = 1.0f;
      if (up_new < up_v || up_v == 0) {
        fs = up_new - up_v > -127 ? __uint_as_float((uint32_t)(127 + (up_v == 0 ? 0 : up_new - up_v)) << 23) : 0.0f;
        up_v = up_new;
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float f[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          f[c] = mx[t][c] == -INFINITY ? 1.0f : ex2((m[t][c] - mx[t][c]) * c2[t][c]);
          m[t][c] = mx[t][c];
          l[t][c] *= f[c];
          zs[t][c] *= f[c];
          f[c] *= fs;
        }
#pragma unroll
        for (int i2 = 0; i2 < D / 16; ++i2)
#pragma unroll
          for (int c = 0; c < 4; ++c) o[t][i2][c] *= f[c & 1];
      }
    }
    float mu[NT][2];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int c = 0; c < 2; ++c) mu[t][c] = m[t][c] == -INFINITY ? 0.0f : m[t][c];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint32_t blk = base + b * kBlock + 8 * D;
      uint32_t p0[NT], p1[NT];
      const float f = __uint_as_float((uint32_t)up_v << 23), s0 = step_of(vz[b][0]) * f, s1 = step_of(vz[b][1]) * f;
      const float z0 = fmaf(8.0f, step_of(vz[b][0]), low_of(vz[b][0])), z1 = fmaf(8.0f, step_of(vz[b][1]), low_of(vz[b][1]));
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float w[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float pr = ex2((x[b][t][c] - mu[t][c & 1]) * c2[t][c & 1]);
          l[t][c & 1] += pr;
          w[c] = pr * (c < 2 ? s0 : s1);
          float z = pr * (c < 2 ? z0 : z1);
          if (edge && x[b][t][c] == -INFINITY) w[c] = z = 0.0f;  // (a place that only later queries see may hold a NaN)
          zs[t][c & 1] += z;
        }
        const __half2 h0 = __floats2half2_rn(w[0], w[1]), h1 = __floats2half2_rn(w[2], w[3]);
        p0[t] = transposed(*reinterpret_cast<const uint32_t*>(&h0));
        p1[t] = transposed(*reinterpret_cast<const uint32_t*>(&h1));
      }
      uint32_t v[4][VW];
      lds<VW>(blk + (2 * q) * (D / 2) + g * (D / 16), v[0]);
      lds<VW>(blk + (2 * q + 1) * (D / 2) + g * (D / 16), v[1]);
      lds<VW>(blk + (2 * q + 8) * (D / 2) + g * (D / 16), v[2]);
      lds<VW>(blk + (2 * q + 9) * (D / 2) + g * (D / 16), v[3]);
#pragma unroll
      for (int u = 0; u < VW; ++u) {
        const uint32_t e0 = __byte_perm(v[0][u], v[1][u], 0x5410), e1 = __byte_perm(v[0][u], v[1][u], 0x7632);
        const uint32_t e2 = __byte_perm(v[2][u], v[3][u], 0x5410), e3 = __byte_perm(v[2][u], v[3][u], 0x7632);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          mma(o[t][4 * u + 0], centred<0>(e0), centred<0>(e1), centred<0>(e2), centred<0>(e3), p0[t], p1[t]);
          mma(o[t][4 * u + 1], centred<1>(e0), centred<1>(e1), centred<1>(e2), centred<1>(e3), p0[t], p1[t]);
          mma(o[t][4 * u + 2], centred<2>(e0), centred<2>(e1), centred<2>(e2), centred<2>(e3), p0[t], p1[t]);
          mma(o[t][4 * u + 3], centred<3>(e0), centred<3>(e1), centred<3>(e2), centred<3>(e3), p0[t], p1[t]);
        }
      }
    }
    __syncwarp();
  }
  if (!ok) {  // the copies in flight end before the block does (each wait is bounded)
    fail(abort_flag, p.status);
    int never = 0;
    for (int i = done; i < mine && i < done + kStages; ++i) mbar_wait(bar0 + 8 * (i % kStages), (uint32_t)(i / kStages) & 1, &never);
  }
  grid_dep_launch();
  __syncthreads();  // every warp is through with the rings

  // sums of this warp, at its own maxima: [row][channel]
  float* mineo = reinterpret_cast<float*>(smem) + warp * kRows * D;
  const float back = up_v == 0 ? 0.0f : __uint_as_float((uint32_t)(254 - up_v) << 23);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      float z = zs[t][c], s = l[t][c];
#pragma unroll
      for (int k = 4; k < 32; k <<= 1) {
        z += __shfl_xor_sync(0xffffffffu, z, k);
        s += __shfl_xor_sync(0xffffffffu, s, k);
      }
      const int row = t * 8 + 2 * q + c;
      if (g == 0) { wm[warp][row] = m[t][c]; wl[warp][row] = s; }
      if (g == 0 && warp == 0) wc[row] = c2[t][c];
      float* y = mineo + row * D + g * (8 * VW);
#pragma unroll
      for (int u = 0; u < VW; ++u)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          y[8 * u + j] = fmaf(o[t][4 * u + j][c], back, z);
          y[8 * u + 4 + j] = fmaf(o[t][4 * u + j][c + 2], back, z);
        }
    }
  __syncthreads();
  const int rows = last_row < kRows ? last_row : kRows;
  for (int i = threadIdx.x; i < rows * D; i += kThreads) {
    const int row = i / D, ch = i - row * D;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, wm[w][row]);
    const float ref = top == -INFINITY ? 0.0f : top, cs = wc[row];
    float sum = 0.0f, all = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = ex2((wm[w][row] - ref) * cs);
      all = fmaf(wl[w][row], f, all);
      sum = fmaf(reinterpret_cast<const float*>(smem)[(w * kRows + row) * D + ch], f, sum);
    }
    if (jb.chunks == 1) {
      const int rr = jb.tile * kRows + row, j = fast_div(rr, sp.group_magic), h = head * sp.group + rr - j * sp.group;
      const int64_t token = jb.start + j;
      put(static_cast<T*>(p.out) + token * p.ldo + (int64_t)h * p.ldoh + ch, top == -INFINITY && all == 0.0f ? 0.0f : sum / all);
      if (p.lse && ch == 0) p.lse[token * p.heads + h] = fmaf(top, cs, log2f(all)) * kLn2;
    } else {
      float* part = sp.part + (((int64_t)blockIdx.x * gridDim.y + head) * kRows + row) * (D + 4);
      part[ch] = sum;
      if (ch == 0) { part[D] = top; part[D + 1] = all; part[D + 2] = cs; }
    }
  }
}

// One block for a row tile's row of a key-value head: the parts of its sequence, in a fixed order.
template <class T, int D>
__global__ void __launch_bounds__(kThreads) combine_kernel(const __grid_constant__ CacheAttnArgs p, const __grid_constant__ Split sp, const int rows) {
  __shared__ float so[kWarps][D], sm[kWarps], sl[kWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  grid_dep_wait();
  if ((int)blockIdx.x >= sp.meta[0]) return;
  const int* meta = sp.meta + 4 + 4 * blockIdx.x;
  const int first = meta[0], chunks = meta[1], start = meta[2], tile = meta[3], queries = sp.meta[4 + 4 * sp.tiles + blockIdx.x];
  const int row = blockIdx.z, rr = tile * rows + row;
  if (chunks == 1 || rr >= queries * sp.group) return;
  float o[D / 32], m = -INFINITY, l = 0.0f;
#pragma unroll
  for (int i = 0; i < D / 32; ++i) o[i] = 0.0f;
  const int64_t pitch = (int64_t)gridDim.y * rows * (D + 4);
  const float* part = sp.part + (((int64_t)first * gridDim.y + blockIdx.y) * rows + row) * (D + 4);
  const float cs = part[D + 2];
  for (int c = warp; c < chunks; c += kWarps) {
    const float* x = part + c * pitch;
    const float mc = x[D], lc = x[D + 1];
    float v[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i) v[i] = x[lane + 32 * i];
    const float top = fmaxf(m, mc), ref = top == -INFINITY ? 0.0f : top;
    const float fa = ex2((m - ref) * cs), fb = ex2((mc - ref) * cs);
    m = top;
    l = l * fa + lc * fb;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) o[i] = o[i] * fa + v[i] * fb;
  }
  if (lane == 0) { sm[warp] = m; sl[warp] = l; }
#pragma unroll
  for (int i = 0; i < D / 32; ++i) so[warp][lane + 32 * i] = o[i];
  __syncthreads();
  for (int ch = threadIdx.x; ch < D; ch += kThreads) {
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sm[w]);
    const float ref = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, all = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float f = ex2((sm[w] - ref) * cs);
      all = fmaf(sl[w], f, all);
      sum = fmaf(so[w][ch], f, sum);
    }
    const int j = fast_div(rr, sp.group_magic), h = blockIdx.y * sp.group + rr - j * sp.group;
    const int64_t token = start + j;
    put(static_cast<T*>(p.out) + token * p.ldo + (int64_t)h * p.ldoh + ch, top == -INFINITY && all == 0.0f ? 0.0f : sum / all);
    if (p.lse && ch == 0) p.lse[token * p.heads + h] = fmaf(top, cs, log2f(all)) * kLn2;
  }
}

struct Sizes {
  int rows;             // of a block
  int64_t tiles, units; // bounds: row tiles; units of a key-value head
  int per_head;         // units that fill the GPU
  size_t part_off, bytes;
};
static Sizes sizes(int64_t tokens, int32_t seqs, int32_t heads, int32_t kv_heads, int32_t dim) {
  Sizes s{};
  const int64_t group = heads / kv_heads;
  // 16 rows a block where most sequences have them: the codes' unpacking serves twice as many
  const bool two = row_tiles(dim) > 1 && tokens * group > 8 * (int64_t)seqs;
  s.rows = two ? 16 : 8;
  s.tiles = tokens == seqs ? seqs * ((group + s.rows - 1) / s.rows) : tokens * group / s.rows + seqs;
  // (tokens == seqs with starts: each of n > 0 queries has at most ceil(n group / rows) <= n ceil(group / rows) tiles)
  s.per_head = (int)((two || dim > 128 ? 152 : 304) / kv_heads);
  if (s.per_head < 1) s.per_head = 1;
  s.units = s.per_head + s.tiles;
  s.part_off = ((size_t)(4 + 5 * s.tiles) * 4 + 255) / 256 * 256;
  s.bytes = s.part_off + (size_t)s.units * kv_heads * s.rows * (dim + 4) * 4;
  return s;
}

template <class T, int D, int NT>
static cudaError_t run(const CacheAttnArgs& a, const Sizes& s, cudaStream_t stream) {
  Split sp{};
  sp.units = s.per_head;
  sp.tiles = (int32_t)s.tiles;
  sp.group = a.heads / a.cache.kv_heads;
  sp.group_magic = div_magic(sp.group);
  sp.q_vec = (reinterpret_cast<uintptr_t>(a.q) & 15) == 0 && (a.ldq | a.ldqh) % 8 == 0;
  sp.meta = reinterpret_cast<int32_t*>(a.ws);
  sp.part = reinterpret_cast<float*>(a.ws + s.part_off);
  constexpr int ring = kWarps * stages(D) * stage_bytes(D), join = kWarps * 8 * NT * D * 4;
  constexpr int smem = ring > join ? ring : join;
  static_assert(smem <= 227 * 1024 - 4096, "");
  cudaError_t e = cudaFuncSetAttribute(cache_attention_kernel<T, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)s.units, (unsigned)a.cache.kv_heads);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelEx(&cfg, cache_attention_kernel<T, D, NT>, a, sp);
  if (e != cudaSuccess) return e;
  // a table of no more than one run's places has no parts to join
  if (((int64_t)a.columns << a.cache.page_shift) <= kWarps * kStep) return cudaSuccess;
  cfg.gridDim = dim3((unsigned)s.tiles, (unsigned)a.cache.kv_heads, (unsigned)s.rows);
  cfg.dynamicSmemBytes = 0;
  return cudaLaunchKernelEx(&cfg, combine_kernel<T, D>, a, sp, s.rows);
}

template <class T>
static cudaError_t run_type(const CacheAttnArgs& a, const Sizes& s, cudaStream_t stream) {
  switch (a.cache.dim) {
    case 64: return s.rows == 16 ? run<T, 64, 2>(a, s, stream) : run<T, 64, 1>(a, s, stream);
    case 128: return s.rows == 16 ? run<T, 128, 2>(a, s, stream) : run<T, 128, 1>(a, s, stream);
    case 192: return run<T, 192, 1>(a, s, stream);
    default: return run<T, 256, 1>(a, s, stream);
  }
}

}  // namespace cacheattn

size_t cache_attention_workspace_bytes(int64_t tokens, int32_t seqs, int32_t heads, int32_t kv_heads, int32_t dim) {
  return cacheattn::sizes(tokens, seqs, heads, kv_heads, dim).bytes;
}

int launch_cache_attention(const CacheAttnArgs& a, cudaStream_t stream, std::string* err) {
  const cacheattn::Sizes s = cacheattn::sizes(a.tokens, a.seqs, a.heads, a.cache.kv_heads, a.cache.dim);
  if (s.units > 0x7fffffff || s.tiles > (1 << 26)) {
    *err = "too many tokens in one call";
    return 2;
  }
  const cudaError_t e = a.dtype == AQD_F16 ? cacheattn::run_type<__half>(a, s, stream) : cacheattn::run_type<__nv_bfloat16>(a, s, stream);
  if (e == cudaSuccess) return 0;
  *err = std::string("cache attention: ") + cudaGetErrorString(e);
  return 3;
}

}  // namespace aqd
