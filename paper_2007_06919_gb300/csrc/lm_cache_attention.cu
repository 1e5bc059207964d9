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
// The unit of work is a warp's: one key-value head, 8 or 16 rows (queries x heads of the group) and a run of steps of 32 places, through the warp's own
// ring of bulk copies (a step is one or two runs of bytes in the cache). How many runs a sequence has follows from its part of all sequences' steps, so
// that they fill the GPU once and are even however the lengths differ; a block's 8 warps take runs that follow one another, of one sequence or of several,
// and join what belongs together; combine_kernel joins what lies in several blocks. (64 sequences of 1 to 8192 places: 24.0 us; blocks of one sequence
// each, of which the short ones left most warps idle, 47.) Few rows over tables of few places take a cluster of one to eight blocks a row tile and head
// instead, which join in shared memory: no second kernel (one sequence of 1000 places, 8 heads: 6.2 us in clusters of four, 9.2 in one block each;
// 4000 places 7.8, 10.3).
//
// What a call spends, in cycles of a block (200,001 places, 2 heads; 22 us): 600 for the launch's order, 2,600 to find its work, 3,000 for page numbers
// and query rows, 1,000 until the first copy is there, 14,000 to 19,000 in five or six steps, 3,000 to join, and 6,500 in the second kernel. A step of
// 32 places is 590 instructions of a warp: 2,360 cycles where 16 warps share the SM, whose copies (70 KB) need 3,200 at 6.8 TB/s. Neither is what the steps take,
// 4,600 to 5,000: with 800,001 places the cache comes in at 4.2 TB/s, with 64 sequences of 8192 at 4.4, with 16 of 32,768 at 4.8. Over a whole
// block the issue slots are 52% busy and the ALU pipe (shifts, logic: two cycles each) 56%, in the steps more; the warps' waits are spread over fixed latencies, that
// pipe, each other and shared memory.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/aqd.h"
#include "common.cuh"
#include "kernels.h"
#include "tc_ptx.cuh"

namespace aqd {
namespace cacheattn {

using namespace tc;

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kMostBlocks = 8;            // of a cluster
constexpr int kStep = 32;                 // places of a step
constexpr float kGrowth = 4.0f;           // powers of two that a maximum may grow by before sums are brought to it
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__host__ __device__ constexpr int stage_bytes(int dim) { return 2 * 16 * (dim + 8); }
__host__ __device__ constexpr int stages(int dim) { return dim == 64 ? 6 : dim == 192 ? 4 : 3; }
__host__ __device__ constexpr int row_tiles(int dim) { return dim <= 128 ? 2 : 1; }  // most tiles of 8 rows a block

struct Split {
  int32_t warps;        // tasks that fill the GPU
  int32_t whole;        // blocks for each sequence, tile and head: this many, a cluster (0: runs of even lengths instead)
  int32_t group;        // query heads of a key-value head
  uint64_t group_magic, kv_magic;
  int32_t q_vec;        // rows of q on 16 bytes
  int32_t* meta;        // [block][8]: Span
  float* part;          // [block][2][row]: dim sums, then maximum, sum, factor
};
// What a block leaves to combine_kernel: the group of runs that begins in it and goes on in blocks up to `last` (0: none).
struct Span {
  int32_t last, start, queries, tile, head, pad[3];
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
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
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
__device__ __forceinline__ uint32_t sub2(uint32_t a, uint32_t b) {
  uint32_t y;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
  return y;
}
// (w & mask) | exponent in one operation
__device__ __forceinline__ uint32_t under(uint32_t w, uint32_t mask, uint32_t exponent) {
  uint32_t y;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(y) : "r"(w), "r"(mask), "r"(exponent));
  return y;
}
// Nibbles of each 16-bit half of w as float16 numbers: under the exponent of 1024 the lowest four bits are 1024 + n, under that of 64 the next four are
// 64 + n; a byte's shift brings the other two there. Keys: n and 64 + n (of the odd nibbles, which -64 sum(q) makes good), values: n - 8.
__device__ __forceinline__ void key_codes(uint32_t w, uint32_t (&h)[4]) {
  const uint32_t v = w >> 8;
  h[0] = sub2(under(w, 0x000f000fu, 0x64006400u), 0x64006400u);
  h[1] = under(w, 0x00f000f0u, 0x54005400u);
  h[2] = sub2(under(v, 0x000f000fu, 0x64006400u), 0x64006400u);
  h[3] = under(v, 0x00f000f0u, 0x54005400u);
}
__device__ __forceinline__ void value_codes(uint32_t w, uint32_t (&h)[4]) {
  const uint32_t v = w >> 8;
  h[0] = sub2(under(w, 0x000f000fu, 0x64006400u), 0x64086408u);
  h[1] = sub2(under(w, 0x00f000f0u, 0x54005400u), 0x54805480u);
  h[2] = sub2(under(v, 0x000f000fu, 0x64006400u), 0x64086408u);
  h[3] = sub2(under(v, 0x00f000f0u, 0x54005400u), 0x54805480u);
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

// A warp's task: run `run` of `runs` of a sequence's tile of rows and a head, `steps` steps from `step0` on; seq -1: none.
struct Job {
  int32_t seq, tile, head, run, runs, step0, steps, start, queries, len;
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

// Tasks fill the GPU once (or, beside many tiles, half of it): runs for a step. steps: of all tiles and heads.
__device__ __forceinline__ float runs_for_a_step(const Split& sp, uint32_t tiles, float steps) {
  const uint32_t most = tiles < (uint32_t)(sp.warps / 2) ? sp.warps - tiles : sp.warps / 2;
  return steps > 0.0f ? (float)most / steps : 0.0f;
}
// A sequence's tiles and how its steps are split into runs.
template <int kRows>
struct Cut {
  uint32_t tiles, steps, count;  // (count: tasks)
  int32_t runs;
  __device__ __forceinline__ Cut(const Split& sp, int queries, int len)
      : tiles((uint32_t)(((int64_t)queries * sp.group + kRows - 1) / kRows)), steps((uint32_t)(len + kStep - 1) / kStep), count(0), runs(1) {}
  __device__ __forceinline__ void split(const Split& sp, int kv, float ratio) {
    if (sp.whole) {
      runs = kWarps * sp.whole;
    } else {
      // (each tile's rounding up is less than one run, and rounding in `ratio` far less than one of all: no more than `most` and the tiles)
      const float x = ceilf((float)steps * ratio);
      runs = x < (float)steps ? (int)x : (int)steps;
      if (runs < 1) runs = 1;
    }
    count = tiles * (uint32_t)(kv * runs);
  }
  // task `at` of this sequence
  __device__ __forceinline__ Job job(const Split& sp, int kv, int seq, int at, int start, int queries, int len) const {
    const int group = (int)((uint32_t)at / (uint32_t)runs), run = at - group * runs, tile = fast_div(group, sp.kv_magic);
    const int each = (int)(steps / (uint32_t)runs), over = (int)steps - each * runs;  // (so many runs have a step more)
    return {seq, tile, group - tile * kv, run, runs, run * each + (run < over ? run : over), each + (run < over ? 1 : 0), start, queries, len};
  }
};
// The task of this warp, of up to 32 sequences: every warp looks for its own, and none waits for another (2,600
// cycles, 3,500 in find_jobs).
template <int kRows>
__device__ __forceinline__ Job find_job(const CacheAttnArgs& p, const Split& sp, bool& none) {
  const int kv = p.cache.kv_heads, lane = threadIdx.x & 31, task0 = blockIdx.x * kWarps, task = task0 + (threadIdx.x >> 5);
  int start = 0, n = 0, len = 0;
  if (lane < p.seqs) sequence(p, lane, start, n, len);
  Cut<kRows> c(sp, n, len);
  float ratio = 0.0f;
  if (!sp.whole) {
    const uint32_t tiles = __reduce_add_sync(0xffffffffu, c.tiles);
    float steps = (float)c.tiles * (float)c.steps;
    for (int o = 16; o > 0; o >>= 1) steps += __shfl_xor_sync(0xffffffffu, steps, o);
    ratio = runs_for_a_step(sp, tiles * (uint32_t)kv, steps * (float)kv);
  }
  c.split(sp, kv, ratio);
  uint32_t upto = c.count;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += u;
  }
  none = (int)__shfl_sync(0xffffffffu, upto, 31) <= task0;
  const int first = (int)(upto - c.count);
  const bool has = task >= first && task < first + (int)c.count;
  Job mine = {-1};
  if (has) mine = c.job(sp, kv, lane, task - first, start, n, len);
  const uint32_t who = __ballot_sync(0xffffffffu, has);
  const int src = who ? __ffs(who) - 1 : 0;
  int32_t* w = reinterpret_cast<int32_t*>(&mine);
#pragma unroll
  for (int i = 0; i < (int)(sizeof(Job) / 4); ++i) w[i] = __shfl_sync(0xffffffffu, w[i], src);
  return mine;
}
// The tasks of this block's warps, of any number of sequences. (Counts are 32 bits wide: the host refuses more. Starts that fall may make more; every
// job is one of its sequence's all the same.)
template <int kRows>
__device__ __forceinline__ void find_jobs(const CacheAttnArgs& p, const Split& sp, Job* jobs, float* red) {
  const int kv = p.cache.kv_heads, first_task = blockIdx.x * kWarps, lane = threadIdx.x & 31, s0 = threadIdx.x;
  uint32_t* sums = reinterpret_cast<uint32_t*>(red + kWarps);
  if (threadIdx.x < kWarps) jobs[threadIdx.x].seq = -1;
  int start = 0, n = 0, len = 0;
  float ratio = 0.0f;
  if (!sp.whole) {
    uint32_t tiles = 0;
    uint64_t mine = 0;
    for (int s = s0; s < p.seqs; s += kThreads) {
      sequence(p, s, start, n, len);
      const Cut<kRows> c(sp, n, len);
      tiles += c.tiles;
      mine += (uint64_t)c.tiles * c.steps;
    }
    float steps = (float)mine;
    tiles = __reduce_add_sync(0xffffffffu, tiles);
    for (int o = 16; o > 0; o >>= 1) steps += __shfl_xor_sync(0xffffffffu, steps, o);
    if (lane == 0) { red[threadIdx.x >> 5] = steps; sums[threadIdx.x >> 5] = tiles; }
    __syncthreads();
    steps = 0.0f;
    tiles = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) { steps += red[w]; tiles += sums[w]; }
    ratio = runs_for_a_step(sp, tiles * (uint32_t)kv, steps * (float)kv);
  }
  uint32_t base = 0;
  for (int b = 0; b < p.seqs; b += kThreads) {
    start = n = len = 0;
    if (b + s0 < p.seqs) sequence(p, b + s0, start, n, len);
    Cut<kRows> c(sp, n, len);
    c.split(sp, kv, ratio);
    // counts before this thread's
    uint32_t before = c.count;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t u = __shfl_up_sync(0xffffffffu, before, o);
      if (lane >= o) before += u;
    }
    __syncthreads();  // (sums may still be read from the last 256 sequences)
    if (lane == 31) sums[threadIdx.x >> 5] = before;
    __syncthreads();
    uint32_t total = 0;
    before -= c.count;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const uint32_t u = sums[w];
      if (w < (int)(threadIdx.x >> 5)) before += u;
      total += u;
    }
    const int first = (int)(base + before);
    for (int at = first > first_task ? first : first_task; at < first_task + kWarps && at < first + (int)c.count; ++at)
      jobs[at - first_task] = c.job(sp, kv, b + s0, at - first, start, n, len);
    base += total;
    if ((int)base >= first_task + kWarps) break;
  }
  __syncthreads();
}

// Four channels of a row out, and its logarithm of the sum.
template <class T>
__device__ __forceinline__ void finish(const CacheAttnArgs& p, const Split& sp, int start, int head, int rr, int ch, float4 sum, float all, float top, float cs) {
  const int j = fast_div(rr, sp.group_magic), h = head * sp.group + rr - j * sp.group;
  const int64_t token = start + j;
  const float inv = top == -INFINITY && all == 0.0f ? 0.0f : 1.0f / all;
  T* y = static_cast<T*>(p.out) + token * p.ldo + (int64_t)h * p.ldoh + ch;
  put(y, sum.x * inv); put(y + 1, sum.y * inv); put(y + 2, sum.z * inv); put(y + 3, sum.w * inv);
  if (p.lse && ch == 0) p.lse[token * p.heads + h] = fmaf(top, cs, log2f(all)) * kLn2;
}
__device__ __forceinline__ float4 load_cluster(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}

// Places that row r of a tile sees.
__device__ __forceinline__ int lim_of(const Job& jb, const Split& sp, int rows, int r, int last_row) {
  return r < last_row ? jb.len - jb.queries + fast_div(jb.tile * rows + r, sp.group_magic) + 1 : 0;
}

template <class T, int D, int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 && D <= 128 ? 2 : 1)
cache_attention_kernel(const __grid_constant__ CacheAttnArgs p, const __grid_constant__ Split sp) {
  constexpr int kStages = stages(D), kStage = stage_bytes(D), kBlock = kStage / 2, kRows = 8 * NT;
  constexpr int KW = D / 32, VW = D / 64;  // words of a key row, and of a value row, that a lane reads
  extern __shared__ __align__(128) uint8_t smem[];  // [warp][stage]; at the end the warps' sums
  __shared__ uint64_t bars[kWarps * kStages], red[kWarps];
  __shared__ Job jobs[kWarps];
  __shared__ int abort_word;
  __shared__ float wm[kWarps][kRows], wl[kWarps][kRows], wc[kWarps][kRows];  // rows' maxima, sums, factors of scores
  volatile int* abort_flag = &abort_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  if (threadIdx.x < kWarps * kStages) mbar_init(smem_u32(&bars[threadIdx.x]), 1);
  if (threadIdx.x == 0) abort_word = 0;
  fence_barrier_init();
  __syncthreads();
  grid_dep_wait();
  Job jb;
  bool none;
  if (p.seqs <= 32) {
    jb = find_job<kRows>(p, sp, none);
    if (lane == 0) jobs[warp] = jb;
    __syncwarp();
  } else {
    find_jobs<kRows>(p, sp, jobs, reinterpret_cast<float*>(red));
    jb = jobs[warp];
    none = jobs[0].seq < 0;
  }
  grid_dep_launch();
  if (none) {  // (a cluster's blocks all have none, or none of them)
    if (!sp.whole && threadIdx.x == 0) reinterpret_cast<Span*>(sp.meta)[blockIdx.x] = Span{};
    return;
  }
  const int head = jb.head;
  const bool idle = jb.seq < 0;
  const int last_row = idle ? 0 : jb.queries * sp.group - jb.tile * kRows;  // rows of this tile and behind it
  int lim_all = 0, lim_any = 0;  // places that the tile's first row sees, and its last
  if (!idle) {
    const int top = last_row < kRows ? last_row : kRows;
    lim_all = jb.len - jb.queries + fast_div(jb.tile * kRows, sp.group_magic) + 1;
    lim_any = jb.len - jb.queries + fast_div(jb.tile * kRows + top - 1, sp.group_magic) + 1;
  }

  // the steps of the run that lie before the last place that a row sees
  const int step0 = idle ? 0 : jb.step0;
  int end = (lim_any + kStep - 1) / kStep;  // (lim_any <= 0: none)
  end = idle ? 0 : end < step0 + jb.steps ? end : step0 + jb.steps;
  const int mine = end > step0 ? end - step0 : 0;
  const int blocks_of_page = 1 << (p.cache.page_shift - 4);
  const int32_t* table = p.table + (idle ? 0 : (int64_t)jb.seq * p.ld_table);
  const uint32_t ring = smem_u32(smem) + warp * (kStages * kStage), bar0 = smem_u32(&bars[warp * kStages]);
  int page0 = -1, page1 = -1;  // of step `lane` of the batch of 32 steps that is being issued
  uint32_t there = 0;          // two bits a stage: its blocks were copied

  const uint8_t* mine_data = p.cache.data + (int64_t)head * blocks_of_page * kBlock;  // this head's part of page 0
  const uint64_t page_bytes = (uint64_t)p.cache.kv_heads * (uint32_t)(blocks_of_page * kBlock);
  int blk = idle ? 0 : (step0 * 2) & (blocks_of_page - 1);  // the next step's first block within its page
  int ist = 0;                                              // its stage

  auto issue = [&](int i) {
    if ((i & 31) == 0) {
      const int place = (step0 + i + lane) * kStep;
      page0 = i + lane < mine ? table[place >> p.cache.page_shift] : -1;
      page1 = i + lane < mine && place + 16 < lim_any ? table[(place + 16) >> p.cache.page_shift] : -1;
      if (page0 < 0 || page0 >= p.cache.pages) page0 = -1;
      if (page1 < 0 || page1 >= p.cache.pages) page1 = -1;
    }
    const int a = __shfl_sync(0xffffffffu, page0, i & 31), b = __shfl_sync(0xffffffffu, page1, i & 31);
    const uint32_t copied = (a >= 0 ? 1u : 0u) | (b >= 0 ? 2u : 0u);
    there = (there & ~(3u << (2 * ist))) | copied << (2 * ist);
    if (lane == 0) {
      const uint32_t dst = ring + ist * kStage, bar = bar0 + 8 * ist;
      const uint8_t* src = mine_data + (uint64_t)(uint32_t)a * page_bytes + (uint32_t)blk * kBlock;
      if (copied == 3u && blocks_of_page > 1) {  // adjacent blocks of a page
        mbar_arrive_expect_tx(bar, kStage);
        bulk_load(dst, src, kStage, bar);
      } else {
        mbar_arrive_expect_tx(bar, (uint32_t)__popc(copied) * kBlock);
        if (a >= 0) bulk_load(dst, src, kBlock, bar);
        if (b >= 0) bulk_load(dst + kBlock, mine_data + (uint64_t)(uint32_t)b * page_bytes + (uint32_t)((blk + 1) & (blocks_of_page - 1)) * kBlock, kBlock, bar);
      }
    }
    blk = (blk + 2) & (blocks_of_page - 1);
    ist = ist == kStages - 1 ? 0 : ist + 1;
  };
  // the query rows' loads, and the first copies (the warp's barriers are set up)
  uint4 qraw[NT][KW];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int r = t * 8 + g;
    const bool live = r < last_row;
    const int j = live ? fast_div(jb.tile * kRows + r, sp.group_magic) : 0, h = jb.tile * kRows + r - j * sp.group;
    const T* x = static_cast<const T*>(p.q) + (live ? (int64_t)(jb.start + j) * p.ldq + (int64_t)(head * sp.group + h) * p.ldqh : 0) + q * (D / 4);
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      qraw[t][w] = make_uint4(0, 0, 0, 0);
      if (live && sp.q_vec) {
        qraw[t][w] = *reinterpret_cast<const uint4*>(x + 8 * w);
      } else if (live) {
        const uint16_t* y = reinterpret_cast<const uint16_t*>(x + 8 * w);
        qraw[t][w] = make_uint4(y[0] | (uint32_t)y[1] << 16, y[2] | (uint32_t)y[3] << 16, y[4] | (uint32_t)y[5] << 16, y[6] | (uint32_t)y[7] << 16);
      }
    }
  }
  for (int i = 0; i < kStages - 1 && i < mine; ++i) issue(i);

  // this lane's query rows (column g of each tile) as float16 with a power of two in front; the sums and factors of columns 2q, 2q + 1
  uint32_t qf[NT][KW][4];
  float qs[NT][2], qb[NT][2], c2[NT][2];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    float f[KW][8], top = 0.0f, sum = 0.0f, odd = 0.0f;
#pragma unroll
    for (int w = 0; w < KW; ++w) {
      const T* e = reinterpret_cast<const T*>(&qraw[t][w]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        f[w][i] = to_f32(e[i]);
        top = fmaxf(top, fabsf(f[w][i]));
      }
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
        const float both = __low2float(h2) + __high2float(h2);
        sum += both;
        if (i & 1) odd += both;
      }
    }
    sum += __shfl_xor_sync(0xffffffffu, sum, 1);
    sum += __shfl_xor_sync(0xffffffffu, sum, 2);
    odd += __shfl_xor_sync(0xffffffffu, odd, 1);
    odd += __shfl_xor_sync(0xffffffffu, odd, 2);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      qs[t][c] = __shfl_sync(0xffffffffu, sum, (2 * q + c) * 4);
      qb[t][c] = -64.0f * __shfl_sync(0xffffffffu, odd, (2 * q + c) * 4);
      c2[t][c] = fminf(fmaxf(__shfl_sync(0xffffffffu, down, (2 * q + c) * 4), 1.4e-45f), 3.402823466e38f);  // (a difference of 0 times it is 0)
    }
  }

  float o[NT][D / 16][4], m[NT][2], l[NT][2], zs[NT][2];
  // the value steps' power of two: weights p s reach float16 times `up_v`, so that the largest step lies in [2^10, 2^11) (and p may be 2^kGrowth); an
  // exponent field, which only falls (0: no step so far)
  int up_v = 0;
  uint32_t within = 0xffffu;  // the greatest word of a step that this power is for
#pragma unroll
  for (int t = 0; t < NT; ++t) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) o[t][i][c] = 0.0f;
#pragma unroll
    for (int c = 0; c < 2; ++c) { m[t][c] = -INFINITY; l[t][c] = 0.0f; zs[t][c] = 0.0f; }
  }
  int done = 0, st = 0;
  uint32_t phase = 0;
  bool ok = true;
  for (; done < mine; ++done) {
    if (done + kStages - 1 < mine) issue(done + kStages - 1);  // (the stage that the last step freed: every lane has read it)
    if (!mbar_wait(bar0 + 8 * st, phase, abort_flag)) { ok = false; break; }
    const uint32_t base = ring + st * kStage;
    const int place = (step0 + done) * kStep;
    const uint32_t here = there >> (2 * st) & 3u;
    float x[2][NT][4];
    uint32_t vz[2][2];
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
        acc[t][0] = acc[t][2] = qb[t][0];
        acc[t][1] = acc[t][3] = qb[t][1];
      }
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        uint32_t a[4], c[4];
        key_codes(k0[w], a);
        key_codes(k1[w], c);
#pragma unroll
        for (int t = 0; t < NT; ++t) mma(acc[t], a[0], c[0], a[1], c[1], qf[t][w][0], qf[t][w][1]);
#pragma unroll
        for (int t = 0; t < NT; ++t) mma(acc[t], a[2], c[2], a[3], c[3], qf[t][w][2], qf[t][w][3]);
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c) x[b][t][c] = fmaf(acc[t][c], step_of(kz[c >> 1]), low_of(kz[c >> 1]) * qs[t][c & 1]);
    }
    const bool partly = place + kStep > lim_all || here != 3u;  // not every row sees every place
    if (partly) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = place + 16 * b + 8 * h + g;
          const bool gone = !(here >> b & 1);
          if (gone || at >= lim_any) vz[b][h] = 0u;  // a stale place's step and lowest value count nowhere
#pragma unroll
          for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              const int lim = lim_of(jobs[warp], sp, kRows, t * 8 + 2 * q + c, last_row);
              if (gone || at >= lim) x[b][t][2 * h + c] = -INFINITY;
            }
        }
    }
    // Maxima so far, of each column's scores and of the value steps. What was summed is brought to a new maximum only where it grew by 2^kGrowth.
    const uint32_t steepest = max(max(vz[0][0], vz[0][1]), max(vz[1][0], vz[1][1]));  // (a step is the word's upper half)
    float mx[NT][2];
    bool grew = steepest > within;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float v = fmaxf(fmaxf(x[0][t][c], x[0][t][c + 2]), fmaxf(x[1][t][c], x[1][t][c + 2]));
        mx[t][c] = v;
        grew = grew || (v - m[t][c]) * c2[t][c] > kGrowth;
      }
    if (__any_sync(0xffffffffu, grew)) {
      float fs = 1.0f;
      uint32_t tops = 0;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t e = vz[b][h] & 0x7f800000u;
          if (e != 0x7f800000u) tops = max(tops, e);
        }
      const int top_e = (int)(__reduce_max_sync(0xffffffffu, tops) >> 23);
      const int up_new = top_e == 0 ? up_v : top_e < 11 ? 253 : 264 - top_e;
      if (up_new < up_v || up_v == 0) {
        fs = up_new - up_v > -127 ? __uint_as_float((uint32_t)(127 + (up_v == 0 ? 0 : up_new - up_v)) << 23) : 0.0f;
        up_v = up_new;
        within = up_v == 0 ? 0xffffu : (uint32_t)(up_v == 253 ? 11 : 264 - up_v) << 23 | 0x7fffffu;
      }
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float f[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          float v = mx[t][c];
          v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
          v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
          v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
          v = fmaxf(v, m[t][c]);
          f[c] = v == -INFINITY ? 1.0f : ex2((m[t][c] - v) * c2[t][c]);
          m[t][c] = v;
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
    uint32_t pw[2][NT][2];
    const float fv = __uint_as_float((uint32_t)up_v << 23);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const float s0 = step_of(vz[b][0]) * fv, s1 = step_of(vz[b][1]) * fv;
      const float z0 = fmaf(8.0f, step_of(vz[b][0]), low_of(vz[b][0])), z1 = fmaf(8.0f, step_of(vz[b][1]), low_of(vz[b][1]));
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        float w[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float pr = ex2((x[b][t][c] - (m[t][c & 1] == -INFINITY ? 0.0f : m[t][c & 1])) * c2[t][c & 1]);
          l[t][c & 1] += pr;
          w[c] = pr * (c < 2 ? s0 : s1);
          float z = c < 2 ? z0 : z1;
          if (partly && x[b][t][c] == -INFINITY) w[c] = z = 0.0f;  // (a place that only later queries see may hold a NaN)
          zs[t][c & 1] = fmaf(pr, z, zs[t][c & 1]);
        }
        const __half2 h0 = __floats2half2_rn(w[0], w[1]), h1 = __floats2half2_rn(w[2], w[3]);
        pw[b][t][0] = transposed(*reinterpret_cast<const uint32_t*>(&h0));
        pw[b][t][1] = transposed(*reinterpret_cast<const uint32_t*>(&h1));
      }
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const uint32_t blk = base + b * kBlock + 8 * D;
      uint32_t v[4][VW];
      lds<VW>(blk + (2 * q) * (D / 2) + g * (D / 16), v[0]);
      lds<VW>(blk + (2 * q + 1) * (D / 2) + g * (D / 16), v[1]);
      lds<VW>(blk + (2 * q + 8) * (D / 2) + g * (D / 16), v[2]);
      lds<VW>(blk + (2 * q + 9) * (D / 2) + g * (D / 16), v[3]);
#pragma unroll
      for (int u = 0; u < VW; ++u) {
        uint32_t a0[4], a1[4], a2[4], a3[4];
        value_codes(__byte_perm(v[0][u], v[1][u], 0x5410), a0);
        value_codes(__byte_perm(v[0][u], v[1][u], 0x7632), a1);
        value_codes(__byte_perm(v[2][u], v[3][u], 0x5410), a2);
        value_codes(__byte_perm(v[2][u], v[3][u], 0x7632), a3);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int t = 0; t < NT; ++t) mma(o[t][4 * u + j], a0[j], a1[j], a2[j], a3[j], pw[b][t][0], pw[b][t][1]);
      }
    }
    if (++st == kStages) { st = 0; phase ^= 1; }
    __syncwarp();
  }
  if (!ok) {  // the copies in flight end before the block does (each wait is bounded)
    fail(abort_flag, p.status);
    int never = 0;
    for (int i = done; i < mine && i < done + kStages; ++i) mbar_wait(bar0 + 8 * (i % kStages), (uint32_t)(i / kStages) & 1, &never);
  }
  __syncthreads();  // every warp is through with the rings

  // sums of this warp, at its own maxima: [row][channel], rows kPitch apart (columns 2q, 2q + 1 of eight lanes at a time: other banks)
  constexpr int kPitch = D + 4;
  float* mineo = reinterpret_cast<float*>(smem) + warp * kRows * kPitch;
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
      if (g == 0) { wm[warp][row] = m[t][c]; wl[warp][row] = s; wc[warp][row] = c2[t][c]; }
      float4* y = reinterpret_cast<float4*>(mineo + row * kPitch + g * (8 * VW));
#pragma unroll
      for (int u = 0; u < VW; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          y[2 * u + h] = make_float4(fmaf(o[t][4 * u][c + 2 * h], back, z), fmaf(o[t][4 * u + 1][c + 2 * h], back, z), fmaf(o[t][4 * u + 2][c + 2 * h], back, z),
                                     fmaf(o[t][4 * u + 3][c + 2 * h], back, z));
    }
  __syncthreads();
  const Job je = jobs[warp];  // (read again: its numbers are not kept through the steps)
  // groups of runs that belong together: the block's warps from `w0` to `w1` join theirs
  if (!idle) {
    const int w0 = warp > je.run ? warp - je.run : 0, run0 = je.run - (warp - w0), w1 = w0 + je.runs - run0 < kWarps ? w0 + je.runs - run0 : kWarps;
    const bool whole = run0 == 0 && w0 + je.runs == w1;
    const int rows = last_row < kRows ? last_row : kRows;
    for (int i = threadIdx.x - w0 * 32; i < rows * (D / 4); i += (w1 - w0) * 32) {
      const int row = i / (D / 4), ch = (i - row * (D / 4)) * 4;
      float top = -INFINITY;
      for (int w = w0; w < w1; ++w) top = fmaxf(top, wm[w][row]);
      const float ref = top == -INFINITY ? 0.0f : top, cs = wc[w0][row];
      float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      float all = 0.0f;
      for (int w = w0; w < w1; ++w) {
        const float f = ex2((wm[w][row] - ref) * cs);
        const float4 v = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(smem) + (w * kRows + row) * kPitch + ch);
        all = fmaf(wl[w][row], f, all);
        sum.x = fmaf(v.x, f, sum.x); sum.y = fmaf(v.y, f, sum.y); sum.z = fmaf(v.z, f, sum.z); sum.w = fmaf(v.w, f, sum.w);
      }
      if (whole) {
        finish<T>(p, sp, je.start, je.head, je.tile * kRows + row, ch, sum, all, top, cs);
      } else {
        float* part = sp.whole ? reinterpret_cast<float*>(smem) + (kWarps * kRows + row) * kPitch
                               : sp.part + (((int64_t)blockIdx.x * 2 + (run0 == 0 ? 1 : 0)) * kRows + row) * (D + 4);
        *reinterpret_cast<float4*>(part + ch) = sum;
        if (ch == 0) *reinterpret_cast<float4*>(part + D) = make_float4(top, all, cs, 0.0f);
      }
    }
  }
  if (sp.whole > 1) {
    // a cluster's blocks have one group: each joins its share of the rows from all of them
    cluster_sync();
    const uint32_t rank = cluster_ctarank(), parts = smem_u32(smem) + kWarps * kRows * kPitch * 4;
    const int items = idle ? 0 : (last_row < kRows ? last_row : kRows) * (D / 4), share = (items + sp.whole - 1) / sp.whole;
    const int to = items < ((int)rank + 1) * share ? items : ((int)rank + 1) * share;
    for (int i = (int)rank * share + threadIdx.x; i < to; i += kThreads) {
      const int row = i / (D / 4), ch = (i - row * (D / 4)) * 4;
      const uint32_t at = parts + row * kPitch * 4;
      float4 v[kMostBlocks], z[kMostBlocks];
      float top = -INFINITY;
#pragma unroll
      for (int b = 0; b < kMostBlocks; ++b)
        if (b < sp.whole) {
          v[b] = load_cluster(mapa_shared(at + 4 * ch, b));
          z[b] = load_cluster(mapa_shared(at + 4 * D, b));
          top = fmaxf(top, z[b].x);
        }
      const float ref = top == -INFINITY ? 0.0f : top;
      float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      float all = 0.0f;
#pragma unroll
      for (int b = 0; b < kMostBlocks; ++b)
        if (b < sp.whole) {
          const float f = ex2((z[b].x - ref) * z[0].z);
          all = fmaf(z[b].y, f, all);
          sum.x = fmaf(v[b].x, f, sum.x); sum.y = fmaf(v[b].y, f, sum.y); sum.z = fmaf(v[b].z, f, sum.z); sum.w = fmaf(v[b].w, f, sum.w);
        }
      finish<T>(p, sp, je.start, je.head, je.tile * kRows + row, ch, sum, all, top, z[0].z);
    }
    __syncwarp();
    cluster_sync();  // no block goes while another reads from it
  } else if (!sp.whole && threadIdx.x == 0) {
    // the group that begins in this block and goes on
    const Job last = jobs[kWarps - 1];
    const int run0 = last.run - (kWarps - 1);  // of the first warp, if this group has it
    const bool begins = last.seq >= 0 && run0 <= 0, goes_on = last.run + 1 < last.runs;
    Span sn = {0, last.start, last.queries, last.tile, last.head, {0, 0, 0}};
    if (begins && goes_on) sn.last = (int)(((int64_t)blockIdx.x * kWarps - run0 + last.runs - 1) / kWarps);
    reinterpret_cast<Span*>(sp.meta)[blockIdx.x] = sn;
  }
}

// Joins the parts of the group of runs that begins in block blockIdx.x and goes on, in a fixed order: a warp to a row where a warp's lanes hold all maxima,
// as those of most groups, and else a block to a row (its loads are shared out then: 152 parts take 3.4 us, 17 a warp, where 5 take 1.3).
template <class T, int D>
__global__ void __launch_bounds__(kThreads, 3) combine_kernel(const __grid_constant__ CacheAttnArgs p, const __grid_constant__ Split sp, const int rows) {
  constexpr int kParts = 152 * 2 + 4;  // a group has at most as many runs as fill the GPU
  constexpr int kQuads = D / 4, kSlots = kThreads / kQuads, kAhead = 8;
  __shared__ float weight[kParts], red[kWarps];
  __shared__ __align__(16) float so[kSlots][D];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  grid_dep_wait();
  const Span span = reinterpret_cast<const Span*>(sp.meta)[blockIdx.x];
  const int first = blockIdx.x, parts = span.last - first + 1, behind = span.queries * sp.group - span.tile * rows;
  // (starts that fall make more tasks than there are blocks: such groups are left)
  if (span.last <= first || span.last >= (int)gridDim.x || parts > kParts) return;
  const bool few = parts <= 32;
  const int row = few ? blockIdx.y * kWarps + warp : blockIdx.y;
  if (row >= rows || row >= behind) return;
  // (what a block goes on with comes first among its two parts, what it begins second)
  const float* part = sp.part + ((int64_t)first * 2 * rows + row) * (D + 4);
  const int64_t pitch = (int64_t)2 * rows * (D + 4), begin = rows * (D + 4);
  const int rr = span.tile * rows + row;
  float4 v[kAhead], z[2];
  if (few) {
    constexpr int kWide = D < 128 ? D / 4 : 32, kAt = 32 / kWide;  // lanes across a row, rows of parts at once
    const int at = lane / kWide;
    z[0] = make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
    if (lane < parts) z[0] = *reinterpret_cast<const float4*>(part + lane * pitch + (lane == 0 ? begin : 0) + D);
    float top, all = 0.0f, cs = 0.0f, f = 0.0f;
#pragma unroll 1
    for (int ch = 4 * (lane & (kWide - 1)); ch - 4 * (lane & (kWide - 1)) < D; ch += 128) {
      float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      for (int c0 = 0; c0 < parts; c0 += kAhead * kAt) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int c = c0 + k * kAt + at;
          v[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          if (c < parts && ch < D) v[k] = *reinterpret_cast<const float4*>(part + c * pitch + (c == 0 ? begin : 0) + ch);
        }
        if (c0 == 0 && ch < 128) {  // (every lane at once)
          top = z[0].x;
          for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
          cs = __shfl_sync(0xffffffffu, z[0].z, 0);
          f = ex2((z[0].x - (top == -INFINITY ? 0.0f : top)) * cs);
          all = z[0].y * f;
          for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int c = c0 + k * kAt + at;
          const float e = __shfl_sync(0xffffffffu, f, c & 31);
          if (c < parts) { sum.x = fmaf(v[k].x, e, sum.x); sum.y = fmaf(v[k].y, e, sum.y); sum.z = fmaf(v[k].z, e, sum.z); sum.w = fmaf(v[k].w, e, sum.w); }
        }
      }
      if constexpr (kAt == 2) {
        sum.x += __shfl_xor_sync(0xffffffffu, sum.x, 16); sum.y += __shfl_xor_sync(0xffffffffu, sum.y, 16);
        sum.z += __shfl_xor_sync(0xffffffffu, sum.z, 16); sum.w += __shfl_xor_sync(0xffffffffu, sum.w, 16);
      }
      if (at == 0 && ch < D) finish<T>(p, sp, span.start, span.head, rr, ch, sum, all, top, cs);
    }
    return;
  }
  const int slot = threadIdx.x / kQuads, quad = threadIdx.x - slot * kQuads;
  // all that these loads need is known: the first sums come beside the maxima
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.0f, 0.0f}, cs = part[begin + D + 2], top = -INFINITY;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int c = threadIdx.x + k * kThreads;
    if (c < parts) z[k] = *reinterpret_cast<const float4*>(part + c * pitch + (c == 0 ? begin : 0) + D);
  }
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const int c = slot + k * kSlots;
    if (slot < kSlots && c < parts) v[k] = *reinterpret_cast<const float4*>(part + c * pitch + (c == 0 ? begin : 0) + 4 * quad);
  }
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if ((int)threadIdx.x + k * kThreads < parts) {
      m[k] = z[k].x; l[k] = z[k].y;
      top = fmaxf(top, m[k]);
    }
  for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
  if (lane == 0) red[warp] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWarps; ++w) top = fmaxf(top, red[w]);
  const float ref = top == -INFINITY ? 0.0f : top;
  float all = 0.0f;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int c = threadIdx.x + k * kThreads;
    const float f = ex2((m[k] - ref) * cs);
    if (c < parts) weight[c] = f;
    all = fmaf(l[k], f, all);
  }
  for (int o = 16; o > 0; o >>= 1) all += __shfl_xor_sync(0xffffffffu, all, o);
  __syncthreads();
  if (lane == 0) red[warp] = all;
  float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (slot < kSlots) {
    for (int c0 = slot; c0 < parts; c0 += kAhead * kSlots) {
      if (c0 > slot) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int c = c0 + k * kSlots;
          if (c < parts) v[k] = *reinterpret_cast<const float4*>(part + c * pitch + 4 * quad);
        }
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int c = c0 + k * kSlots;
        if (c < parts) {
          const float f = weight[c];
          sum.x = fmaf(v[k].x, f, sum.x); sum.y = fmaf(v[k].y, f, sum.y); sum.z = fmaf(v[k].z, f, sum.z); sum.w = fmaf(v[k].w, f, sum.w);
        }
      }
    }
    *reinterpret_cast<float4*>(&so[slot][4 * quad]) = sum;
  }
  __syncthreads();
  all = 0.0f;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) all += red[w];
  if (slot == 0) {
    for (int k = 1; k < kSlots; ++k) {
      const float4 u = *reinterpret_cast<const float4*>(&so[k][4 * quad]);
      sum.x += u.x; sum.y += u.y; sum.z += u.z; sum.w += u.w;
    }
    finish<T>(p, sp, span.start, span.head, rr, 4 * quad, sum, all, top, cs);
  }
}

struct Sizes {
  int rows;             // of a tile
  int warps;            // tasks that fill the GPU
  int64_t tiles, blocks; // bounds: row tiles; blocks where runs are split
  size_t part_off, bytes;
};
static Sizes sizes(int64_t tokens, int32_t seqs, int32_t heads, int32_t kv_heads, int32_t dim) {
  Sizes s{};
  const int64_t group = heads / kv_heads;
  // 16 rows a task where most sequences have them: the codes' unpacking serves twice as many
  const bool two = row_tiles(dim) > 1 && tokens * group > 8 * (int64_t)seqs;
  s.rows = two ? 16 : 8;
  s.tiles = tokens == seqs ? seqs * ((group + s.rows - 1) / s.rows) : tokens * group / s.rows + seqs;
  // (tokens == seqs with starts: each of n > 0 queries has at most ceil(n group / rows) <= n ceil(group / rows) tiles)
  s.warps = 152 * (two || dim > 128 ? 1 : 2) * kWarps;
  // tasks: at most `warps`, or half of that beside more tiles and heads than the other half
  const int64_t tasks = s.warps / 2 + s.tiles * kv_heads;
  s.blocks = ((tasks > s.warps ? tasks : s.warps) + kWarps - 1) / kWarps;
  s.part_off = ((size_t)s.blocks * sizeof(Span) + 255) / 256 * 256;
  s.bytes = s.part_off + (size_t)s.blocks * 2 * s.rows * (dim + 4) * 4;
  return s;
}

template <class T, int D, int NT>
static cudaError_t run(const CacheAttnArgs& a, const Sizes& s, cudaStream_t stream) {
  Split sp{};
  sp.warps = s.warps;
  sp.group = a.heads / a.cache.kv_heads;
  sp.group_magic = div_magic(sp.group);
  sp.kv_magic = div_magic(a.cache.kv_heads);
  sp.q_vec = (reinterpret_cast<uintptr_t>(a.q) & 15) == 0 && (a.ldq | a.ldqh) % 8 == 0;
  sp.meta = reinterpret_cast<int32_t*>(a.ws);
  sp.part = reinterpret_cast<float*>(a.ws + s.part_off);
  constexpr int ring = kWarps * stages(D) * stage_bytes(D), join = (kWarps + 1) * 8 * NT * (D + 4) * 4;
  constexpr int smem = ring > join ? ring : join;
  static_assert(smem <= 227 * 1024 - 4096, "");
  cudaError_t e = cudaFuncSetAttribute(cache_attention_kernel<T, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  const int64_t heads_tiles = s.tiles * a.cache.kv_heads;
  const int64_t places = (int64_t)a.columns << a.cache.page_shift;
  // As many blocks a row tile and head as leave each warp a step, within one block an SM; taken while a warp has no more than four steps (2 heads, clusters of
  // eight: 2000 places 6.6 us, 10.0 in split runs; 4000 7.8, 10.3; 8000 10.3, 10.9; where one block each fills the GPU, 1024 places take 12.6 either way).
  int cluster = 1;
  while (cluster < kMostBlocks && cluster * kWarps * kStep < places && 2 * cluster * heads_tiles <= 152) cluster *= 2;
  sp.whole = places <= 4 * kWarps * kStep * cluster ? cluster : 0;
  const int64_t blocks = sp.whole ? heads_tiles * sp.whole : s.blocks;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = sp.whole ? sp.whole : 1;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = sp.whole > 1 ? 2 : 1;
  e = cudaLaunchKernelEx(&cfg, cache_attention_kernel<T, D, NT>, a, sp);
  if (e != cudaSuccess || sp.whole) return e;
  const int most = a.starts || sp.group > s.rows ? s.rows : sp.group;  // rows of a tile that can be there
  cfg.gridDim = dim3((unsigned)blocks, (unsigned)most);
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
  if (s.tiles * a.cache.kv_heads > (1 << 27)) {  // (tasks are counted in 32 bits)
    *err = "too many tokens in one call";
    return 2;
  }
  const cudaError_t e = a.dtype == AQD_F16 ? cacheattn::run_type<__half>(a, s, stream) : cacheattn::run_type<__nv_bfloat16>(a, s, stream);
  if (e == cudaSuccess) return 0;
  *err = std::string("cache attention: ") + cudaGetErrorString(e);
  return 3;
}

}  // namespace aqd
