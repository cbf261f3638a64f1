// Attention of many new tokens over the 4-bit cache: prompts and pieces of them.
//
// With many rows (new tokens x query heads of a key/value head) the products bound, not the cache: a CTA takes 256 rows of
// one sequence and key/value head, as two halves of 128, against tiles of 128 keys.  Four warps expand the tile once, its keys
// to fp16 and its values to bf16 (what eqat_cache_read gives); rows are the 128 lanes of both products, in steps of 64 keys:
//     S = Q K^T     128 x 64, operands in shared memory, fp16
//     O += P V      P in tensor memory beside S, bf16
// Eight warps, one thread a row, do the softmax: maximum, then weights, which go to tensor memory as bf16; a row's sums are
// rescaled only when its maximum rises by more than 2^8.  A warp for each half issues its products; while one half is in its
// softmax the other half's products run.
//
// Keys as fp16 are off by 2^-11 of themselves at most, as bf16 by 2^-8.  Queries and keys that fp16 holds badly are scaled by
// powers of two.  Error of the outputs against 64 bits (relative norm), and time, with keys as bf16 and as fp16:
//     4 prompts of up to 1500, 32 heads of 64               0.0033, 92 us     0.0023 to 0.0024, 101 us
//     1000 new behind 7192, 64/8 heads of 128               0.0020, 326 us    0.0018, 339 us
//     16 x 5 new, window 4000 (one tile of 40 rows)         0.0022, 72 us     0.0019, 76 us
// A maximum that passes NaN on made that 104, 335 and 77 us.
//
// What bounds it: the latency of a step's softmax, about 2500 cycles of which the exponentials and their chain are most (three
// of eight pairs are polynomials for that reason), and the last wave of CTAs: the second of these has 256 items for 148 SMs.
// It runs at 755 TFLOP/s there, masked products not counted.  Steps of 128 keys took 396 us for it where steps of 64 took 320.
#include <type_traits>

#include "attention.cuh"
#include "common.cuh"
#include "ptx.cuh"
#include "wait.cuh"

namespace eqat {
namespace {

constexpr int kHalfWarps = 4, kSpreadWarps = 4;
constexpr int kThreads = (2 * kHalfWarps + kSpreadWarps + 4) * 32;      // two of the last four issue the products
// Registers of a thread: 128 at launch, divided anew over the four groups of warps (184 + 184 + 88 + 56 = 4 * 128).
constexpr int kSoftmaxRegs = 184, kSpreadRegs = 88, kProductRegs = 56;
constexpr float kLazy = 8.0f;                        // a maximum may be exceeded by 2^8 before the sums are rescaled
constexpr float kInfiniteValue = 0x1.FFp127f;        // rounds to an infinity of bf16, and all above
constexpr int64_t kPromptTokens = 1 << 25;           // of the longest sequence
constexpr int kTile = 128, kStep = 64;               // keys that are expanded, that are multiplied at once

template <int D, int G>
struct Shape {
  static constexpr int kRows = 256, kUnit = kTile, kStageTokens = 16;
  static constexpr int kBoxes = D / 64;                                // blocks of 64 elements: 128 rows x 128 bytes
  static constexpr int kOperandBytes = kBoxes * 16384;                 // 128 rows of queries, keys or values
  static constexpr int kStages = 2;
  static constexpr int kSmemBytes = 1024 + (2 + 2 * kStages) * kOperandBytes;
  static constexpr int kLoads = D / 32;                                // 16-byte loads of a lane per tile, keys or values
  // tensor memory of a half: scores of a step, weights of two steps, outputs
  static constexpr int kAlloc = 512, kHalfCols = 256, kWeightCol = 64, kOutputCol = 128;
};

struct PromptCtl {
  uint64_t queries_full;
  uint64_t keys_full[2], keys_free[2], values_full[2], values_free[2];
  uint64_t scores_done[2], scores_read[2];
  uint64_t weights_full[2][2], sums_done[2][2];      // of a half's even and odd steps: either side may be two steps ahead
  uint32_t tmem;
  int abort;
  // Of the last tiles, written by the spreading warps before they arrive at keys_full (strange: at values_full), read by the softmax
  // warps once they have met the commit of a product that was issued behind that arrival.  A commit orders the tensor core's
  // accesses, not those of the warp that issues it; what makes the tables visible is that shared memory has no copies: a store
  // that came before an arrival which some warp of the CTA has seen is there for all loads that any of them makes later.
  // (The products' warp arriving at a barrier of its own, which the softmax waits for once a tile, cost 4 to 5 %: 1000 new
  // behind 7192 336 -> 349 us, 4 prompts with heads of 64 104 -> 109.5.)
  alignas(16) uint32_t strange[8][4];                // tokens of the last tiles with a group that bf16 cannot hold
  alignas(16) uint32_t large[8][4];                  // tokens of the last tiles whose keys were scaled, and by
  uint8_t scaled_by[8][kTile];                       // what power of two: its exponent's bits
  int64_t before[kThreads];                          // units of the sequences before a thread's
  int64_t total;
};

__device__ __forceinline__ uint32_t as_word(__nv_bfloat162 x) { return *reinterpret_cast<uint32_t*>(&x); }
__device__ __forceinline__ __nv_bfloat162 as_pair(uint32_t x) { return *reinterpret_cast<__nv_bfloat162*>(&x); }

__device__ __forceinline__ __half2 as_half_pair(uint32_t x) { return *reinterpret_cast<__half2*>(&x); }

// q s + m of the codes in nibbles I and I + 4, rounded once: as an fp16 pair, as a bf16 pair.
template <int I>
__device__ __forceinline__ uint32_t key_pair(uint32_t w, __half2 s, __half2 m) {
  const uint32_t codes = ((w >> (4 * I)) & 0x000F000Fu) | 0x64006400u;                     // 1024 + q
  const __half2 r = __hfma2(__hsub2(as_half_pair(codes), as_half_pair(0x64006400u)), s, m);
  return *reinterpret_cast<const uint32_t*>(&r);
}
template <int I>
__device__ __forceinline__ uint32_t value_pair(uint32_t w, __nv_bfloat162 s, __nv_bfloat162 m) {
  const uint32_t codes = ((w >> (4 * I)) & 0x000F000Fu) | 0x43004300u;
  return as_word(__hfma2(__hsub2(as_pair(codes), as_pair(0x43004300u)), s, m));
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{\n\t.reg .b64 x, y, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 w, x, y;\n\tmov.b64 {%0, %1}, w;\n\t}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}

// The largest of three; NaN if one is.
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// 2^x by the multiply-add pipes, for x <= 16 (a NaN becomes some number: the row's sum is made NaN by its maximum): 2^n p(f)
// with n the nearest integer and f in [-1/2, 1/2], p of degree 3 with the smallest relative error there (7.5e-5, from the exchange algorithm; a weight is rounded to bf16, 2^-8, right after).  Below
// -126 it stays at 2^-126.  The special function unit takes 8 cycles for the 32 exponentials of a warp, 1000 cycles for the two
// halves' steps; three of eight pairs go this way (1000 new tokens behind 7192, 64/8 heads: none 332 us, two 325, three 323,
// four 340).
constexpr int kPolyPairs = 3;
__device__ __forceinline__ float2 exp2_poly(float2 x) {
  x.x = fmaxf(x.x, -126.0f);
  x.y = fmaxf(x.y, -126.0f);
  const float2 t = add2(x, make_float2(12582912.0f, 12582912.0f));      // 1.5 * 2^23: the integer in the low bits
  const float2 f = add2(x, fma2(t, make_float2(-1.0f, -1.0f), make_float2(12582912.0f, 12582912.0f)));
  float2 p = fma2(f, make_float2(0.05517167f, 0.05517167f), make_float2(0.24261113f, 0.24261113f));
  p = fma2(f, p, make_float2(0.69326097f, 0.69326097f));
  p = fma2(f, p, make_float2(0.99992806f, 0.99992806f));
  return make_float2(__uint_as_float(__float_as_uint(p.x) + (__float_as_uint(t.x) << 23)),
                     __uint_as_float(__float_as_uint(p.y) + (__float_as_uint(t.y) << 23)));
}

template <int D, int G>
__global__ void __launch_bounds__(kThreads, 1) prompt_kernel(const AttentionArgs a) {
  using S = Shape<D, G>;
  constexpr int kChunks = D / 32, kGroupChunks = kChunks / G;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(16) PromptCtl ctl_block;
  PromptCtl* ctl = &ctl_block;
  volatile int* abort_flag = &ctl->abort;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw = ptx::smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t queries = base, keys = queries + 2 * S::kOperandBytes, values = keys + S::kStages * S::kOperandBytes;

  if (threadIdx.x == 0) {
    ptx::mbar_init(ptx::smem_addr(&ctl->queries_full), 2 * kHalfWarps + 2);      // also the products' warps: done with the item before
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(ptx::smem_addr(&ctl->keys_full[i]), kSpreadWarps);
      ptx::mbar_init(ptx::smem_addr(&ctl->values_full[i]), kSpreadWarps);
      ptx::mbar_init(ptx::smem_addr(&ctl->keys_free[i]), 2);
      ptx::mbar_init(ptx::smem_addr(&ctl->values_free[i]), 2);
      ptx::mbar_init(ptx::smem_addr(&ctl->scores_done[i]), 1);
      ptx::mbar_init(ptx::smem_addr(&ctl->scores_read[i]), kHalfWarps);
      ptx::mbar_init(ptx::smem_addr(&ctl->weights_full[i][0]), kHalfWarps);
      ptx::mbar_init(ptx::smem_addr(&ctl->weights_full[i][1]), kHalfWarps);
      ptx::mbar_init(ptx::smem_addr(&ctl->sums_done[i][0]), 1);
      ptx::mbar_init(ptx::smem_addr(&ctl->sums_done[i][1]), 1);
    }
    ctl->abort = 0;
    ptx::fence_mbar_init();
  }
  if (warp == 0) {
    take_columns(ptx::smem_addr(&ctl->tmem), S::kAlloc);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = ctl->tmem;
  ptx::grid_dependency_wait();

  // ---- the items (sequence, row tile, head), and how many come before each thread's sequences
  const CacheView& v = a.cache;
  const int each = (v.sequences + kThreads - 1) / kThreads;
  auto items_of = [&](int b, SequenceWork& w) {
    w = sequence_work<S>(a, b);
    return (int64_t)w.tiles * v.kv_heads;
  };
  {
    int64_t own = 0;
    SequenceWork w;
    for (int b = (int)threadIdx.x * each; b < min(((int)threadIdx.x + 1) * each, v.sequences); ++b) own += items_of(b, w);
    ctl->before[threadIdx.x] = own;
    __syncthreads();
    if (warp == 0) {                                                     // exclusive sums, 32 threads at a time
      int64_t sum = 0;
      for (int k = 0; k < kThreads; k += 32) {
        const int64_t n = ctl->before[k + lane];
        int64_t upto = n;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const int64_t o = __shfl_up_sync(0xFFFFFFFFu, upto, d);
          if (lane >= d) upto += o;
        }
        ctl->before[k + lane] = sum + upto - n;
        sum += __shfl_sync(0xFFFFFFFFu, upto, 31);
      }
      if (lane == 0) ctl->total = sum;
    }
    __syncthreads();
  }
  const int64_t total = ctl->total;
  struct Job {
    SequenceRows rows;
    Segment sg;
    int sequence, head, tiles, steps, halves;
  };
  auto job_of = [&](int64_t x) {                                         // whole warp
    int k = 0;
    for (int i = 0; i * each < v.sequences; i += 32) k += __popc(__ballot_sync(0xFFFFFFFFu, (i + lane) * each < v.sequences && ctl->before[i + lane] <= x));
    int b = (k - 1) * each;                                              // the last thread with no more than x before it
    int64_t before = ctl->before[k - 1];
    SequenceWork w;
    for (int64_t n; x >= before + (n = items_of(b, w)); ++b) before += n;
    const int in = (int)(x - before), tile = w.tiles - 1 - in / v.kv_heads;            // the longest rows first
    Job j;
    j.rows = w.rows;
    j.sequence = b;
    j.head = in % v.kv_heads;
    j.sg = segment_of<S>(a, w, tile);
    j.steps = j.sg.from < j.sg.high ? (j.sg.high - j.sg.from + kStep - 1) / kStep : 0;
    j.tiles = (j.steps + 1) / 2;
    j.halves = j.sg.rows > 128 ? 2 : 1;
    return j;
  };
  auto wait = [&](uint64_t& barrier, uint32_t phase) {
    bounded_wait_warp(ptx::smem_addr(&barrier), phase & 1u, abort_flag, WAIT_EPI_ACC_FULL);
  };
  auto arrive = [&](uint64_t& barrier) {                                 // a warp's
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(ptx::smem_addr(&barrier));
  };

  if (warp < 2 * kHalfWarps) {
    // ================================================================== softmax: thread `row` of half h
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    const int h = warp / kHalfWarps, row_in_half = threadIdx.x & 127;
    const uint32_t own = (uint32_t)((warp % kHalfWarps) * 32) << 16;
    const uint32_t scores = tmem + h * S::kHalfCols + own, outputs = scores + S::kOutputCol;
    const uint32_t query_row = queries + h * S::kOperandBytes + row_in_half * 128;
    float c = 1.0f;                                                      // the row's factor: its query is scaled too
    auto wait_sums = [&](uint32_t step) { wait(ctl->sums_done[h][step & 1u], step >> 1); };
    const uint32_t sign = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
    uint32_t n = 0, count = 0, items = 0;                                // steps of this half, tiles of all items, items so far
    for (int64_t x = blockIdx.x; x < total; x += gridDim.x) {
      const Job job = job_of(x);
      const int r = h * 128 + row_in_half, row = job.sg.first_row + r, new_token = token_of_row(a, row);
      const bool real = r < job.sg.rows;
      const int base_pos = job.rows.length - job.rows.count;
      const int64_t out_row = job.rows.first + new_token;
      const int q_head = job.head * a.ratio + row - new_token * a.ratio;
      // ---- the row's query, in the order of the codes (0 4 1 5 2 6 3 7 of each eight)
      if (job.tiles > 0) {
        if (h < job.halves) {
          const uint4* src = reinterpret_cast<const uint4*>(a.Q + out_row * a.q_pitch + (int64_t)q_head * D);
          // scaled by a power of two, so that the largest element lies in [1, 2), [2, 4) from 2^127 on, to fp16: exact down to
          // 2^-17, off by at most 2^-25 below; an infinity becomes NaN: no score of the row means anything
          uint4 e[D / 8];
          uint32_t most = 0;
#pragma unroll
          for (int p = 0; p < D / 8; ++p) {
            e[p] = make_uint4(0u, 0u, 0u, 0u);
            if (real) e[p] = ptx::ld_global(src + p);
            most = __vmaxu2(most, __vmaxu2(__vmaxu2(e[p].x & 0x7FFF7FFFu, e[p].y & 0x7FFF7FFFu), __vmaxu2(e[p].z & 0x7FFF7FFFu, e[p].w & 0x7FFF7FFFu)));
          }
          most = max(most & 0xFFFFu, most >> 16);
          const int up = most == 0 ? 0 : min(max(127 - (int)(most >> 7), -126), 100);
          const float scale = most >= 0x7F80u ? __int_as_float(0x7FC00000) : __int_as_float((127 + up) << 23);
          c = fmaxf(fabsf(a.scale_log2) * __int_as_float((127 - up) << 23), 1e-37f);      // (not 0: -infinity times 0 is NaN)
          auto two = [&](uint32_t lo, uint32_t hi) {                     // bf16 numbers in the high halves
            const __half2 r = __floats2half2_rn(__uint_as_float(lo) * scale, __uint_as_float(hi) * scale);
            return *reinterpret_cast<const uint32_t*>(&r) ^ sign;
          };
#pragma unroll
          for (int p = 0; p < D / 8; ++p)
            ptx::sts_128(query_row + p / 8 * 16384 + (((p % 8) ^ (row_in_half & 7)) << 4), two(e[p].x << 16, e[p].z << 16),
                         two(e[p].x & 0xFFFF0000u, e[p].z & 0xFFFF0000u), two(e[p].y << 16, e[p].w << 16), two(e[p].y & 0xFFFF0000u, e[p].w & 0xFFFF0000u));
          ptx::fence_proxy_async_smem();
        }
        ptx::tc_fence_before();                                          // the last item's outputs have been read
        arrive(ctl->queries_full);
      }
      const uint32_t first_count = count;
      count += job.tiles;
      if (h >= job.halves) {                                             // not ahead of the half that has rows
        if (job.tiles > 0) wait(ctl->queries_full, items++);
        continue;
      }
      if (job.tiles > 0) ++items;
      // keys that this row, and that every row of the half, sees
      const int high = real ? base_pos + new_token + 1 : 0, low = a.window > 0 ? base_pos + new_token + 1 - a.window : 0;
      const int last_row = min(job.sg.rows, (h + 1) * 128) - 1;
      const int all_high = base_pos + token_of_row(a, job.sg.first_row + h * 128) + 1;
      const int all_low = a.window > 0 ? base_pos + token_of_row(a, job.sg.first_row + last_row) + 1 - a.window : 0;
      float top = -INFINITY, sum = 0.0f;                                 // of the scores, before the scale; of the weights
      // Groups of values that bf16 cannot hold have been spread as zeros, since zero times NaN is not zero: a row that sees
      // one is NaN.
      bool strange = false;
      auto look = [&](int i) {                                           // at a tile whose values have been multiplied
        const uint4 y = *reinterpret_cast<const uint4*>(ctl->strange[(first_count + i) & 7u]);
        if ((y.x | y.y | y.z | y.w) == 0u) return;
        const uint32_t words[4] = {y.x, y.y, y.z, y.w};
        for (int t = 0; t < kTile; ++t) {
          const int token = job.sg.from + i * kTile + t;
          strange |= (words[t / 32] >> (t % 32) & 1u) != 0u && token < high && token >= low;
        }
      };
      for (int i = 0; i < job.steps; ++i, ++n) {
        const int t0 = job.sg.from + i * kStep;
        const bool edge = t0 < all_low || t0 + kStep > all_high;
        wait(ctl->scores_done[h], n);
        ptx::tc_fence_after();
        const uint2 large = *reinterpret_cast<const uint2*>(&ctl->large[(first_count + i / 2) & 7u][i & 1 ? 2 : 0]);
        float s[kStep];                                                  // the row's scores
#pragma unroll
        for (int k = 0; k < kStep; k += 32) ptx::tmem_ld_32x32(scores + k, *reinterpret_cast<uint32_t(*)[32]>(s + k));
        ptx::tmem_ld_wait();
        ptx::tc_fence_before();
        arrive(ctl->scores_read[h]);                                     // the next step's may come
        if ((large.x | large.y) != 0u) {                                 // keys that fp16 holds badly, each with its own scale
          const uint8_t* by = ctl->scaled_by[(first_count + i / 2) & 7u] + (i & 1) * kStep;
#pragma unroll
          for (int j = 0; j < kStep; ++j) {
            s[j] *= __int_as_float((int)by[j] << 23);
            if (!(fabsf(s[j]) < INFINITY)) s[j] = __int_as_float(0x7FC00000);          // (-infinity is what is masked)
          }
        }
        if (edge) {
          const int before = high - t0, from = low - t0;
#pragma unroll
          for (int j = 0; j < kStep; ++j) s[j] = j < before && j >= from ? s[j] : -INFINITY;
        }
        float m4[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
        for (int j = 4; j < kStep; j += 8)
#pragma unroll
          for (int k = 0; k < 4 && j + 2 * k < kStep; ++k) m4[k] = max_nan(m4[k], s[j + 2 * k], s[j + 2 * k + 1]);
        const float most = max_nan(max_nan(m4[0], m4[1], m4[2]), m4[3], m4[3]);
        const bool first = top == -INFINITY;
        const bool raise = first ? most > -INFINITY : (most - top) * c > kLazy;
        if (__any_sync(0xFFFFFFFFu, raise)) {
          const float to = raise ? most : top;
          const float f = first || !raise ? 1.0f : exp2_approx((top - to) * c);
          top = to;
          sum *= f;
          if (i > 0) {
            wait_sums(n - 1);
            ptx::tc_fence_after();
#pragma unroll 1
            for (int k = 0; k < D; k += 16) {
              uint32_t o[16];
              ptx::tmem_ld_32x16(outputs + k, o);
              ptx::tmem_ld_wait();
#pragma unroll
              for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
              ptx::tmem_st_32x16(outputs + k, o);
            }
          }
        }
        // a score that is NaN or, scaled, beyond fp32: so is everything of the row
        if (most != -INFINITY) sum = fmaf(0.0f, most * c, sum);
        // ---- weights, two a column, in the place of those of two steps ago: this step's scores were issued behind the
        // product with those
        if (i > 1 && (i & 1) == 0) look(i / 2 - 1);
        const float shift = top == -INFINITY ? 0.0f : top * c;
        const float2 c2 = make_float2(c, c), shift2 = make_float2(-shift, -shift);
        float2 parts[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
        auto weigh = [&](auto is_edge) {
#pragma unroll
          for (int k = 0; k < kStep; k += 32) {
            uint32_t p[16];
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
              float2 e = fma2(make_float2(s[k + j], s[k + j + 1]), c2, shift2);
              if (!decltype(is_edge)::value && j / 2 % 8 >= 8 - kPolyPairs) {
                e = exp2_poly(e);
              } else {
                e.x = exp2_approx(e.x);
                e.y = exp2_approx(e.y);
              }
              parts[j / 2 & 1] = add2(parts[j / 2 & 1], e);
              p[j / 2] = pack_bf16x2(e.x, e.y);
            }
            ptx::tmem_st_32x16(scores + S::kWeightCol + (n & 1u) * 32 + k / 2, p);
          }
        };
        if (edge) weigh(std::true_type());                               // what is masked weighs 0, not 2^-126
        else weigh(std::false_type());
        ptx::tmem_st_wait();
        ptx::tc_fence_before();
        arrive(ctl->weights_full[h][n & 1u]);
        parts[0] = add2(parts[0], parts[1]);
        sum += parts[0].x + parts[0].y;
      }
      // ---- outputs
      if (job.tiles > 0) {
        wait_sums(n - 1);
        ptx::tc_fence_after();
        if (job.tiles > 1) look(job.tiles - 2);
        look(job.tiles - 1);
      }
      const bool empty = top == -INFINITY && sum == 0.0f;                // (a row whose scores are all NaN is not)
      const float inv = strange ? __int_as_float(0x7FC00000) : 1.0f / sum;
      eqat_bf16* to = a.O + out_row * a.o_pitch + (int64_t)q_head * D;
#pragma unroll 1
      for (int k = 0; k < D / 32; ++k) {
        uint32_t o[32];
        if (job.tiles > 0) {
          ptx::tmem_ld_32x32(outputs + 32 * k, o);
          ptx::tmem_ld_wait();
        }
        if (real) {
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            float e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) e[j] = empty ? 0.0f : __uint_as_float(o[8 * p + j]) * inv;
            *reinterpret_cast<uint4*>(to + 32 * k + 8 * p) = make_uint4(pack_bf16x2(e[0], e[2]), pack_bf16x2(e[4], e[6]), pack_bf16x2(e[1], e[3]), pack_bf16x2(e[5], e[7]));
          }
        }
      }
      if (real && a.lse != nullptr)
        a.lse[out_row * a.q_heads + q_head] = empty ? -INFINITY : ((top == -INFINITY ? 0.0f : top * c) + log2f(sum)) * 0.69314718055994531f;
    }
  } else if (warp < 2 * kHalfWarps + kSpreadWarps) {
    // ================================================================== keys as fp16, values as bf16
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kSpreadRegs));
    const int w4 = warp - 2 * kHalfWarps;                                // 32 tokens of a tile
    const int token_in = lane / kChunks, chunk = lane % kChunks;         // of this lane's first chunk; tokens 32 / kChunks apart
    constexpr int kApart = 32 / kChunks;
    const uint32_t row_at = (32 * w4 + token_in) * 128 + chunk / 2 * 16384;
    uint32_t count = 0;                                                  // tiles so far
    for (int64_t x = blockIdx.x; x < total; x += gridDim.x) {
      const Job job = job_of(x);
      int page = 0;
      auto page_of = [&](int i) {
        const int token = job.sg.from + i * kTile + 32 * w4 + 16 * lane;
        return lane < 2 && token < job.sg.high ? ld_index(v.page_table + (int64_t)job.sequence * v.max_pages + page_index(a, token)) : 0;
      };
      struct Fetched { uint4 codes[S::kLoads]; uint32_t params[S::kLoads]; };
      uint32_t at[2] = {0, 0};
      auto find = [&](int i) {
        const int token = job.sg.from + i * kTile + 32 * w4 + 16 * lane;
        // a page number outside the pool counts as the nearest inside
        const uint32_t place = ((uint32_t)min(max(page, 0), v.pages - 1) * v.kv_heads + job.head) * v.page_size + (token - page_index(a, token) * v.page_size);
        at[0] = __shfl_sync(0xFFFFFFFFu, place, 0);
        at[1] = __shfl_sync(0xFFFFFFFFu, place, 1);
        page = page_of(i + 1);
      };
      auto fetch = [&](Fetched& f, const uint8_t* codes, const uint32_t* params, int i) {
        const int left = job.sg.high - (job.sg.from + i * kTile + 32 * w4);              // tokens from the warp's first on
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const uint4* from = reinterpret_cast<const uint4*>(codes + (uint64_t)at[p] * (D / 2)) + lane;
          const uint32_t* with = params + (uint64_t)at[p] * G + token_in * G + chunk / kGroupChunks;
#pragma unroll
          for (int j = 0; j < S::kLoads / 2; ++j) {
            const int k = p * (S::kLoads / 2) + j;
            f.codes[k] = make_uint4(0u, 0u, 0u, 0u);
            f.params[k] = 0u;                                            // behind the last key: zeros
            if (16 * p < left) f.codes[k] = ptx::ld_global(from + 32 * j);
            if (16 * p + j * kApart + token_in < left) f.params[k] = ptx::ld_global(with + j * kApart * G);
          }
        }
      };
      // Keys as fp16.  A token whose largest element may be 2^14 or more, or is below 2^-6, where the steps would lose bits to
      // fp16's least exponent, is scaled by a power of two of its own.
      // Whether there may be one is found for the warp's tokens at once: none where every step lies in [2^-8, 2^9), since 15
      // steps then reach 2^-6 on one side of zero or the other, and every minimum below 2^13.
      auto spread_keys = [&](const Fetched& f, uint32_t operand, uint32_t slot) {
        uint32_t most = 0, least = 0xFFFFFFFFu;
#pragma unroll
        for (int k = 0; k < S::kLoads; ++k) {
          const uint32_t size = f.params[k] & 0x7FFF7FFFu;
          most = __vmaxu2(most, size);
          least = __vminu2(least, size);
        }
        const bool ordinary = (least & 0xFFFFu) >= (127 - 8) << 7 && (most & 0xFFFFu) < (127 + 9) << 7 && most >> 16 < (127 + 13) << 7;
        auto spread = [&](auto scaled) {
          uint32_t marks = 0;
#pragma unroll
          for (int k = 0; k < S::kLoads; ++k) {
            const int token = 32 * w4 + token_in + k * kApart;
            const uint32_t param = f.params[k];
            float down = 1.0f;
            if (decltype(scaled)::value) {
              const float bound = fmaf(15.0f, fabsf(param_step(param)), fabsf(param_low(param)));
              // not finite: the others count; a finite step and minimum may give an infinite bound
              const bool bad = (param & 0x7F80u) == 0x7F80u || (param & 0x7F800000u) == 0x7F800000u;
              uint32_t exponent = bad ? 0u : min(__float_as_uint(bound) >> 23, 254u);
#pragma unroll
              for (int d = 1; d < kChunks; d <<= 1) exponent = max(exponent, __shfl_xor_sync(0xFFFFFFFFu, exponent, d));
              const int by = exponent > 127 + 13 ? (int)exponent - (127 + 13) : exponent > 0 && exponent < 127 - 6 ? (int)exponent - 127 : 0;
              if (by != 0) marks |= 1u << (token & 31);
              if (chunk == 0) ctl->scaled_by[slot][token] = (uint8_t)(127 + by);
              down = bad ? __int_as_float(0x7FC00000) : __int_as_float((127 - by) << 23);      // NaN, not an infinity, in every score
            }
            const __half2 s2 = __float2half2_rn(param_step(param) * down), m2 = __float2half2_rn(param_low(param) * down);
            const uint32_t w[4] = {f.codes[k].x, f.codes[k].y, f.codes[k].z, f.codes[k].w};
#pragma unroll
            for (int p = 0; p < 4; ++p)
              ptx::sts_128(operand + row_at + k * kApart * 128 + (((chunk % 2 * 4 + p) ^ (token & 7)) << 4), key_pair<0>(w[p], s2, m2),
                           key_pair<1>(w[p], s2, m2), key_pair<2>(w[p], s2, m2), key_pair<3>(w[p], s2, m2));
          }
          if (decltype(scaled)::value) marks = __reduce_or_sync(0xFFFFFFFFu, marks);
          if (lane == 0) ctl->large[slot][w4] = marks;
        };
        if (__all_sync(0xFFFFFFFFu, ordinary)) {
          ctl->scaled_by[slot][32 * w4 + lane] = 127;                    // (the step's other warp may have some)
          spread(std::false_type());
        } else {
          spread(std::true_type());
        }
      };
      // Values as bf16.  A group that is not finite, or whose largest value would round to an infinity, is marked.
      auto spread_values = [&](const Fetched& f, uint32_t operand, uint32_t* strange) {
        uint32_t marks = 0;
#pragma unroll
        for (int k = 0; k < S::kLoads; ++k) {
          const int token = 32 * w4 + token_in + k * kApart;
          uint32_t param = f.params[k];
          if (!(fabsf(fmaf(15.0f, param_step(param), param_low(param))) < kInfiniteValue)) {
            param = 0u;
            marks |= 1u << (token & 31);
          }
          const __nv_bfloat162 s2 = as_pair(__byte_perm(param, 0, 0x1010)), m2 = as_pair(__byte_perm(param, 0, 0x3232));
          const uint32_t w[4] = {f.codes[k].x, f.codes[k].y, f.codes[k].z, f.codes[k].w};
#pragma unroll
          for (int p = 0; p < 4; ++p)
            ptx::sts_128(operand + row_at + k * kApart * 128 + (((chunk % 2 * 4 + p) ^ (token & 7)) << 4), value_pair<0>(w[p], s2, m2),
                         value_pair<1>(w[p], s2, m2), value_pair<2>(w[p], s2, m2), value_pair<3>(w[p], s2, m2));
        }
        marks = __reduce_or_sync(0xFFFFFFFFu, marks);
        if (lane == 0) strange[w4] = marks;
      };
      Fetched key, value;
      if (job.tiles > 0) {
        page = page_of(0);
        find(0);
        fetch(key, v.kq, v.kp, 0);
        fetch(value, v.vq, v.vp, 0);
      }
      for (int i = 0; i < job.tiles; ++i, ++count) {
        const uint32_t stage = count & 1u, use = count >> 1;
        if (use > 0) wait(ctl->keys_free[stage], use - 1);
        spread_keys(key, keys + stage * S::kOperandBytes, count & 7u);
        ptx::fence_proxy_async_smem();
        arrive(ctl->keys_full[stage]);
        if (i + 1 < job.tiles) {
          find(i + 1);
          fetch(key, v.kq, v.kp, i + 1);
        }
        if (use > 0) wait(ctl->values_free[stage], use - 1);
        spread_values(value, values + stage * S::kOperandBytes, ctl->strange[count & 7u]);
        ptx::fence_proxy_async_smem();
        arrive(ctl->values_full[stage]);
        if (i + 1 < job.tiles) fetch(value, v.vq, v.vp, i + 1);
      }
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kProductRegs));
    const int h = warp - (2 * kHalfWarps + kSpreadWarps);                // a warp for each half
    if (h < 2) {
      // ================================================================ the products
      constexpr uint32_t kScoreDesc = (1u << 4) | ((uint32_t)(kStep / 8) << 17) | (8u << 24);      // fp16 operands
      constexpr uint32_t kSumDesc = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D / 8) << 17) | (8u << 24);
      const uint64_t query_desc = ptx::smem_desc(queries + h * S::kOperandBytes);
      const uint64_t key_desc = ptx::smem_desc(keys), value_desc = ptx::smem_desc(values, 16384);
      const uint32_t scores = tmem + h * S::kHalfCols, outputs = scores + S::kOutputCol;
      uint32_t count = 0, items = 0, n = 0;                              // tiles, items with any, steps of this half
      for (int64_t x = blockIdx.x; x < total; x += gridDim.x) {
        const Job job = job_of(x);
        if (job.tiles == 0) continue;
        if (lane == 0) ptx::mbar_arrive(ptx::smem_addr(&ctl->queries_full));
        wait(ctl->queries_full, items++);
        const bool own = h < job.halves;
        if (!own) {                                                      // a half without rows hands back what it does not read
          for (int i = 0; i < job.tiles; ++i, ++count) {
            wait(ctl->keys_full[count & 1u], count >> 1);
            if (lane == 0) ptx::mbar_arrive(ptx::smem_addr(&ctl->keys_free[count & 1u]));
            wait(ctl->values_full[count & 1u], count >> 1);
            if (lane == 0) ptx::mbar_arrive(ptx::smem_addr(&ctl->values_free[count & 1u]));
          }
          continue;
        }
        auto multiply_keys = [&](int i) {                                // scores of step i of the item
          const uint32_t tile = count + i / 2, stage = tile & 1u;
          if ((i & 1) == 0) wait(ctl->keys_full[stage], tile >> 1);
          ptx::tc_fence_after();
          if (ptx::elect_one()) {
            const uint64_t k = key_desc + (uint64_t)(stage * (S::kOperandBytes >> 4) + (i & 1) * (kStep * 128 >> 4));
#pragma unroll
            for (int e = 0; e < D / 16; ++e)
              ptx::mma_bf16_ss(scores, query_desc + ((e / 4 * 16384 + e % 4 * 32) >> 4), k + ((e / 4 * 16384 + e % 4 * 32) >> 4), kScoreDesc, e != 0);
            ptx::mma_commit(ptx::smem_addr(&ctl->scores_done[h]));
            if ((i & 1) != 0 || i + 1 == job.steps) ptx::mma_commit(ptx::smem_addr(&ctl->keys_free[stage]));
          }
          __syncwarp();
        };
        multiply_keys(0);
        for (int i = 0; i < job.steps; ++i, ++n) {
          wait(ctl->scores_read[h], n);
          if (i + 1 < job.steps) multiply_keys(i + 1);
          const uint32_t tile = count + i / 2, stage = tile & 1u;
          wait(ctl->weights_full[h][n & 1u], n >> 1);
          if ((i & 1) == 0) wait(ctl->values_full[stage], tile >> 1);
          ptx::tc_fence_after();
          if (ptx::elect_one()) {
            const uint64_t b = value_desc + (uint64_t)(stage * (S::kOperandBytes >> 4) + (i & 1) * (kStep * 128 >> 4));
#pragma unroll
            for (int e = 0; e < kStep / 16; ++e)
              ptx::mma_bf16_ts(outputs, scores + S::kWeightCol + (n & 1u) * 32 + e * 8, b + ((e * 2048) >> 4), kSumDesc, i != 0 || e != 0);
            ptx::mma_commit(ptx::smem_addr(&ctl->sums_done[h][n & 1u]));
            if ((i & 1) != 0 || i + 1 == job.steps) ptx::mma_commit(ptx::smem_addr(&ctl->values_free[stage]));
          }
          __syncwarp();
        }
        count += job.tiles;
      }
    }
  }
  ptx::grid_dependents_launch();
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(ctl->tmem, S::kAlloc);
  }
}

template <int D, int G>
int launch_shape(const AttentionArgs& a, int sms, cudaStream_t st) {
  using S = Shape<D, G>;
  static SmemOptIn opt;
  if (!opt.ensure(prompt_kernel<D, G>, S::kSmemBytes)) return EQAT_ERR_CUDA;
  return launch_overlapped(prompt_kernel<D, G>, dim3(sms), dim3(kThreads), S::kSmemBytes, st, a);
}

}  // namespace

bool prompt_attention_applies(const eqat_cache_desc& d, const eqat_attention_desc& a, int sms) {
  const int64_t ratio = a.q_heads / d.kv_heads;
  if (d.head_dim > 128 || a.max_new * ratio < kPromptRows) return false;
  // A CTA's idle half waits for as long as an item of the other half lasts, about 1.3 us for 64 keys: 0.7 s here, of the 2 s after
  // which a wait gives up.
  if ((int64_t)d.max_pages * d.page_size > kPromptTokens) return false;
  // Estimated cycles for 128 keys, if all sequences have the same number of rows or, where that is few, as many as possible have
  // the most and the others one.  Here an SM takes about 4500 for an item, of up to 256 rows, and the items are dealt out
  // whole.  The kernel for few rows takes 3700 for tiles of 32 rows, 2100 for 16 and 1000 + 100 a group for 8, and spreads any
  // number of tiles over all SMs.  (2000 tokens, 64/8 heads, 40 rows, groups of 128:
  // 32 sequences 78 us here, 110 there; 4 sequences of 8000 tokens 123 and 62.)
  const int64_t most = (int64_t)a.max_new * d.sequences, rows = d.rows < most ? d.rows : most;
  int64_t with = d.sequences < rows ? d.sequences : rows, each = (rows * ratio + with - 1) / with;
  if (each < kPromptRows) {
    each = a.max_new * ratio;
    with = (rows - with) / a.max_new > 1 ? (rows - with) / a.max_new : 1;
  }
  const int groups = d.head_dim / d.group, tile = groups >= 4 ? 8 : groups == 2 ? 16 : 32;
  const double here = (double)((with * d.kv_heads * ((each + 255) / 256) + sms - 1) / sms) * 4500.0;
  const double there = (double)(with * d.kv_heads * ((each + tile - 1) / tile)) / sms * (tile == 8 ? 1000 + 100 * groups : tile == 16 ? 2100 : 3700);
  return here < there;
}

int prompt_least_rows(const eqat_cache_desc& d, const eqat_attention_desc& a, int sms) {
  const int64_t ratio = a.q_heads / d.kv_heads;
  if (d.rows * ratio < (int64_t)d.sequences * kPromptRows) return kPromptRows;
  if ((d.rows - (int64_t)(d.sequences - 1) * a.max_new) * ratio >= kPromptRows) return 1;        // none can have fewer
  // Cycles where short sequences, as long as the table has room for and with one row, become items here, and where they go to
  // the kernel for few rows: an item takes 4500 for 128 keys, a tile there 1000, the two launches 17000 (9 us).  The long ones
  // are taken as whole prompts.  (64/8 heads, all here against divided: a prompt of 2000 and one token behind 32768 604 and 173 us,
  // and 31 such tokens 1182 and 408; four prompts of 640 to 1336 178 and 187.)
  const UnequalBatch u = unequal_batch(d, a);
  const double length = (double)d.max_pages * d.page_size, key = 4500.0 / 128;
  const double prompts = (double)(u.with * d.kv_heads * ((u.longest * ratio + 255) / 256)) * u.longest / 2 / sms;
  const double shorts = (double)(u.rest * d.kv_heads) * length / sms;
  const double together = (prompts + shorts > length ? prompts + shorts : length) * key;
  const double apart = (prompts > u.longest ? prompts : u.longest) * key + shorts / 128 * 1000 + 17000;
  return together <= apart ? 1 : kPromptRows;
}

int launch_prompt_attention(const eqat_cache_desc& d, AttentionArgs a, cudaStream_t st) {
  const int sms = sm_count(), g = d.head_dim / d.group;
  if (sms <= 0) return EQAT_ERR_CUDA;
  a.most_rows = INT32_MAX;
  if (d.head_dim == 64) return g == 1 ? launch_shape<64, 1>(a, sms, st) : launch_shape<64, 2>(a, sms, st);
  return g == 1 ? launch_shape<128, 1>(a, sms, st) : g == 2 ? launch_shape<128, 2>(a, sms, st) : launch_shape<128, 4>(a, sms, st);
}

int launch_wait_expiry_prompt(cudaStream_t st) { return launch_wait_expiry(st); }
int read_prompt_status(int* status, int* detail) { return read_wait_status(status, detail); }

}  // namespace eqat
