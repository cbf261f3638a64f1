// Attention of a few new tokens over the 4-bit cache: decoding, drafted tokens.
//
// A key/value head's codes are read once for up to 8 * NT query rows (new tokens x the query heads that share the head).
// With step s and minimum m of a group and q a code, K = q s + m and V likewise, so
//     Q . K_t  = sum over groups of  s_t (sum_d Q_d q_td) + m_t (sum_d Q_d)
//     sum_t p_t V_t = sum_t (p_t s_t) (q_t - 8) + sum_t p_t (m_t + 8 s_t):
// both products run on matrix instructions with codes as exact bf16 integers (128 + q for the keys, whose constant goes into
// the second term; q - 8 for the values, where a long even softmax adds up to far less than 128 times its terms), steps and
// minima multiply fp32 sums.  p_t s_t is rounded to bf16, as the softmax weights of any attention on these instructions are.
//
// Scores are computed transposed (16 tokens x 8 rows), so the codes are always the 16-row operand and one user's single
// query wastes nothing but columns.  The layout of the two operands:
//   keys    ldmatrix gives a thread the words of tokens g, g + 8 (g = lane / 4): eight codes of one token; the nibbles 4
//           apart are a register pair, so a word is two k-steps of one group.  The queries are put in that order once.
//   values  ldmatrix.trans gives a thread halfword g of a 16-byte chunk for two neighbouring tokens: again pairs.
//   p s     is transposed by movmatrix from the score layout to that of the second operand.
//
// Work is dealt out in units of one 4-warp CTA's stage (4096 / head_dim tokens per warp); the units of all (sequence, row
// tile, head) segments are laid end to end and every CTA takes an equal stretch, so batches of any lengths fill the device.
// A segment that several CTAs share is joined by a second small kernel in a fixed order.  Inside a CTA every warp has its
// own ring of stages, fed by its own lanes with tensor copies (codes, 128-byte swizzle: ldmatrix without conflicts) and bulk
// copies (steps and minima), its own maximum, sum and accumulators; warps meet at the end of a segment.
#include <cuda.h>

#include <type_traits>

#include "cache.cuh"
#include "common.cuh"
#include "gemm.cuh"
#include "ptx.cuh"
#include "wait.cuh"

namespace eqat {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazy = 8.0f;                        // a maximum may be exceeded by 2^8 before the sums are rescaled

template <int D, int G, int NT>
struct Shape {
  static constexpr int kStageTokens = 4096 / D;                        // per warp
  static constexpr int kSteps = kStageTokens / 16;
  static constexpr int kUnit = kWarps * kStageTokens;
  static constexpr int kRows = 8 * NT;
  static constexpr int kParamBytes = kStageTokens * G * 4;
  static constexpr int kMergeFloats = kRows * D;                       // of a warp, in its ring
  static constexpr int kStages = kMergeFloats * 4 > 3 * 4096 ? 4 : 3;
  static constexpr int kRingBytes = kStages * 4096;                    // codes of a warp (1024-byte aligned)
  static constexpr int kParamRing = kStages * 2 * kParamBytes;
  static constexpr int kWarpBytes = kRingBytes + kParamRing;
  static constexpr int kSmemBytes = 1024 + kWarps * kWarpBytes;
  static constexpr int kRegCtas = NT * D <= 128 ? 4 : NT * D <= 256 ? 3 : 2;
  static constexpr int kSmemCtas = 227 * 1024 / (kSmemBytes + 1024 + 512);
  static constexpr int kCtas = kRegCtas < kSmemCtas ? kRegCtas : kSmemCtas;
  static_assert(kMergeFloats * 4 <= kRingBytes, "the accumulators of a warp are exchanged through its ring");
};

struct AttentionArgs {
  CacheView cache;
  const eqat_bf16* Q;
  int64_t q_pitch, o_pitch;
  eqat_bf16* O;
  float* lse;
  float* partial;              // [2 * workers][rows of a tile][D + 2]
  int q_heads, ratio, max_new, window;
  float scale_log2;            // scale * log2(e)
  int box_tokens;              // tokens of one copy of codes
  int min_units;               // least number of units of a worker
};

// ------------------------------------------------------------------ the work and its division
// All segments of a sequence have the same number of units, so that a unit is found by division; early row tiles of a long
// prompt and rows at the edge of a window leave some empty.
struct SequenceWork {
  SequenceRows rows;
  int tiles, units;            // row tiles; units of a segment
};
template <typename S>
__device__ __forceinline__ SequenceWork sequence_work(const AttentionArgs& a, int b) {
  SequenceWork w;
  w.rows = sequence_rows(a.cache, b);
  const int64_t rows = (int64_t)min(w.rows.count, a.max_new) * a.ratio;
  w.tiles = (int)((rows + S::kRows - 1) / S::kRows);
  int span = w.rows.length;
  if (a.window > 0) span = (int)min((int64_t)span, (int64_t)a.window + S::kRows / a.ratio + 1 + S::kStageTokens);
  w.units = max(1, (span + S::kUnit - 1) / S::kUnit);
  return w;
}
__device__ __forceinline__ int64_t work_units(const CacheView& v, const SequenceWork& w) {
  return (int64_t)w.tiles * v.kv_heads * w.units;
}

struct WorkPlace {
  int64_t total, per;          // units of the call, of a worker
  int64_t before;              // units of the sequences before `sequence`
  int sequence;                // that holds unit `x` (or sequences, if none does)
};
// Whole CTA: finds the sequence of unit x, which may depend on the total (x = f(per)).
template <typename S, typename F>
__device__ __forceinline__ WorkPlace find_work(const AttentionArgs& a, int workers, F&& f, int64_t* scratch) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int each = (a.cache.sequences + kThreads - 1) / kThreads;
  const int b0 = min(tid * each, a.cache.sequences), b1 = min(b0 + each, a.cache.sequences);
  int64_t own = 0;
  for (int b = b0; b < b1; ++b) own += work_units(a.cache, sequence_work<S>(a, b));
  int64_t upto = own;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t o = __shfl_up_sync(0xFFFFFFFFu, upto, d);
    if (lane >= d) upto += o;
  }
  if (lane == 31) scratch[warp] = upto;
  if (tid == 0) scratch[kWarps + 1] = a.cache.sequences;
  __syncthreads();
  int64_t total = 0, before = upto - own;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += scratch[w];
    total += scratch[w];
  }
  WorkPlace p;
  p.total = total;
  p.per = max((total + workers - 1) / workers, (int64_t)a.min_units);
  const int64_t x = f(p.per);
  if (x >= before && x < before + own) {
    int b = b0;
    for (;; ++b) {
      const int64_t n = work_units(a.cache, sequence_work<S>(a, b));
      if (x < before + n) break;
      before += n;
    }
    scratch[kWarps] = before;
    scratch[kWarps + 1] = b;
  }
  __syncthreads();
  p.before = scratch[kWarps];
  p.sequence = (int)scratch[kWarps + 1];
  return p;
}

// A segment: one row tile of one sequence over one key/value head.
struct Segment {
  int first_row, rows;         // of the tile, counted in (new token, query head of this key/value head)
  int low, high;               // keys that any row of the tile sees: [low, high)
  int from;                    // low, rounded down to a stage
};
template <typename S>
__device__ __forceinline__ Segment segment_of(const AttentionArgs& a, const SequenceWork& w, int tile) {
  Segment s;
  const int n = min(w.rows.count, a.max_new);
  s.first_row = tile * S::kRows;
  s.rows = min(S::kRows, n * a.ratio - s.first_row);
  const int base = w.rows.length - w.rows.count;
  s.high = max(base + (s.first_row + s.rows - 1) / a.ratio + 1, 0);
  s.low = a.window > 0 ? max(base + s.first_row / a.ratio + 1 - a.window, 0) : 0;
  s.from = s.low & ~(S::kStageTokens - 1);
  return s;
}

// ------------------------------------------------------------------ instructions
__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
// D (16 x 8, fp32) += A (16 x 16, bf16) * B (16 x 8, bf16)
__device__ __forceinline__ void mma_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// Two codes of a word, nibbles I and I + 4, as bf16 128 + q.
template <int I>
__device__ __forceinline__ uint32_t codes_128(uint32_t w) { return ((w >> (4 * I)) & 0x000F000Fu) | 0x43004300u; }
// The same as q - 8.
template <int I>
__device__ __forceinline__ uint32_t codes_centred(uint32_t w) {
  const uint32_t x = codes_128<I>(w);
  const uint32_t off = 0x43084308u;                                    // 136
  const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&x), *reinterpret_cast<const __nv_bfloat162*>(&off));
  return *reinterpret_cast<const uint32_t*>(&r);
}
template <int G>
__device__ __forceinline__ void load_params(uint32_t (&r)[G], uint32_t addr) {
  if constexpr (G == 1) {
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r[0]) : "r"(addr) : "memory");
  } else if constexpr (G == 2) {
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr) : "memory");
  } else {
#pragma unroll
    for (int i = 0; i < G; i += 4) {
      const uint4 v = ptx::lds_128(addr + 4 * i);
      r[i] = v.x; r[i + 1] = v.y; r[i + 2] = v.z; r[i + 3] = v.w;
    }
  }
}

// ------------------------------------------------------------------ the kernel
struct AttentionCtl {
  uint64_t full[kWarps][4];
  float top[kWarps][16], sum[kWarps][16];
  int64_t scratch[kWarps + 2];
  int abort;
};

template <int D, int G, int NT>
__global__ void __launch_bounds__(kThreads, (Shape<D, G, NT>::kCtas))
attention_kernel(const AttentionArgs a, const __grid_constant__ CUtensorMap keys_map, const __grid_constant__ CUtensorMap values_map) {
  using S = Shape<D, G, NT>;
  constexpr int kChunks = D / 32;                                      // 16-byte chunks of a row of codes
  constexpr int kGroupChunks = kChunks / G;
  extern __shared__ uint8_t smem_raw[];
  __shared__ AttentionCtl ctl_block;
  AttentionCtl* ctl = &ctl_block;
  volatile int* abort_flag = &ctl->abort;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
  const uint32_t raw = ptx::smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t ring = base + warp * S::kRingBytes;
  const uint32_t param_ring = base + kWarps * S::kRingBytes + warp * S::kParamRing;
  float* merge = reinterpret_cast<float*>(smem_raw + (base - raw));
  if (lane == 0)
    for (int i = 0; i < S::kStages; ++i) ptx::mbar_init(ptx::smem_addr(&ctl->full[warp][i]), 1);
  if (tid == 0) {
    ctl->abort = 0;
    ptx::tma_prefetch_desc(&keys_map);
    ptx::tma_prefetch_desc(&values_map);
  }
  ptx::fence_mbar_init();
  __syncthreads();
  ptx::grid_dependency_wait();

  const CacheView& v = a.cache;
  const WorkPlace wp = find_work<S>(a, gridDim.x, [&](int64_t per) { return (int64_t)blockIdx.x * per; }, ctl->scratch);
  int64_t x = (int64_t)blockIdx.x * wp.per;
  const int64_t x_end = min(x + wp.per, wp.total);
  int b = wp.sequence;
  int64_t seq_before = wp.before;
  uint32_t issued = 0, taken = 0;                                      // stages of this warp over all segments
  bool alive = true;

  // per-lane ldmatrix offset inside 16 tokens of codes: matrices (tokens 0-7, chunk j), (8-15, j), (0-7, j+1), (8-15, j+1)
  const uint32_t mat_token = ((lane >> 3) & 1) * 8 + (lane & 7);
  const uint32_t mat_linear = mat_token * (D / 2) + (lane >> 4) * 16;
  const uint32_t mat_offset = mat_linear ^ (((mat_linear >> 7) & 7u) << 4);

  while (x < x_end) {
    SequenceWork w = sequence_work<S>(a, b);
    int64_t have = work_units(v, w);
    while (x >= seq_before + have) {                                   // sequences without rows have no units
      seq_before += have;
      w = sequence_work<S>(a, ++b);
      have = work_units(v, w);
    }
    const int64_t in_seq = x - seq_before;
    const int seg = (int)(in_seq / w.units), u0 = (int)(in_seq % w.units);
    const int u1 = (int)min((int64_t)w.units, u0 + (x_end - x));
    const int head = seg % v.kv_heads;
    const Segment sg = segment_of<S>(a, w, seg / v.kv_heads);
    const bool whole = u0 == 0 && u1 == w.units;

    // ---- the stages of this warp: tokens from + (4 (u0 + i) + warp) * kStageTokens
    const int first_token = sg.from + (u0 * kWarps + warp) * S::kStageTokens;
    int stages = 0;
    if (alive && first_token < sg.high)
      stages = min(u1 - u0, (sg.high - first_token + S::kUnit - 1) / S::kUnit);
    auto page_of = [&](int token) {                                    // of this lane's piece of a stage
      if (token >= sg.high) return 0;
      const int page = ld_index(v.page_table + (int64_t)b * v.max_pages + token / v.page_size);
      return min(max(page, 0), v.pages - 1);
    };
    // Lanes 4 p .. 4 p + 3 fetch piece p of a stage: codes of keys and values, parameters of keys and values.
    const int piece_token = (lane >> 2) * a.box_tokens;
    int page = 0;
    if (stages > 0 && piece_token < S::kStageTokens) page = page_of(first_token + piece_token);
    auto issue = [&](int i) {                                          // page: of stage i, already fetched
      const int slot = (int)(issued % S::kStages);
      const uint32_t full = ptx::smem_addr(&ctl->full[warp][slot]);
      const int t = first_token + i * S::kUnit;
      const int pieces = min(S::kStageTokens / a.box_tokens, (sg.high - t + a.box_tokens - 1) / a.box_tokens);
      if (lane == 0) ptx::mbar_expect_tx(full, pieces * a.box_tokens * (D + 8 * G));
      __syncwarp();
      if (lane < 4 * pieces) {
        const int tok = t + piece_token;
        const int64_t at = ((int64_t)page * v.kv_heads + head) * v.page_size + tok % v.page_size;
        const int what = lane & 3;
        if (what < 2) {
          ptx::tma_load_2d(ring + slot * 4096 + what * 2048 + piece_token * (D / 2), what == 0 ? &keys_map : &values_map, 0,
                           (int)(at * (D / 2) / 128), full);
        } else {
          ptx::bulk_load(param_ring + slot * 2 * S::kParamBytes + (what - 2) * S::kParamBytes + piece_token * G * 4,
                         (what == 2 ? v.kp : v.vp) + at * G, a.box_tokens * G * 4, full);
        }
      }
      ++issued;
      if (i + 1 < stages && piece_token < S::kStageTokens) page = page_of(t + S::kUnit + piece_token);
    };
    int next_issue = 0;
    for (; next_issue < min(stages, S::kStages); ++next_issue) issue(next_issue);

    // ---- the queries, in the order of the codes, and their sums per group
    uint32_t q[NT][kChunks][4];
    float q_sum[NT][G][2];
    int row_low[NT][2], row_high[NT][2];                               // keys that the rows of this lane's columns see
    const int base_pos = w.rows.length - w.rows.count;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int r = n * 8 + g;
      float sums[G];
#pragma unroll
      for (int k = 0; k < G; ++k) sums[k] = 0.0f;
      const int row = sg.first_row + r;
      const eqat_bf16* src = a.Q + (int64_t)(w.rows.first + row / a.ratio) * a.q_pitch + (int64_t)(head * a.ratio + row % a.ratio) * D;
#pragma unroll
      for (int j = 0; j < kChunks; ++j) {
        uint4 e = make_uint4(0u, 0u, 0u, 0u);
        if (r < sg.rows) e = ptx::ld_global(reinterpret_cast<const uint4*>(src + j * 32 + c * 8));
        q[n][j][0] = __byte_perm(e.x, e.z, 0x5410);                    // elements 0, 4
        q[n][j][1] = __byte_perm(e.x, e.z, 0x7632);                    // 1, 5
        q[n][j][2] = __byte_perm(e.y, e.w, 0x5410);                    // 2, 6
        q[n][j][3] = __byte_perm(e.y, e.w, 0x7632);                    // 3, 7
        sums[j / kGroupChunks] += ((param_step(e.x) + param_low(e.x)) + (param_step(e.y) + param_low(e.y))) +
                                  ((param_step(e.z) + param_low(e.z)) + (param_step(e.w) + param_low(e.w)));
      }
#pragma unroll
      for (int k = 0; k < G; ++k) {
        sums[k] += __shfl_xor_sync(0xFFFFFFFFu, sums[k], 1);
        sums[k] += __shfl_xor_sync(0xFFFFFFFFu, sums[k], 2);
        q_sum[n][k][0] = __shfl_sync(0xFFFFFFFFu, sums[k], 8 * c);     // of rows 2 c, 2 c + 1
        q_sum[n][k][1] = __shfl_sync(0xFFFFFFFFu, sums[k], 8 * c + 4);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int rr = n * 8 + 2 * c + i;
        const int pos = base_pos + (sg.first_row + rr) / a.ratio;
        row_high[n][i] = rr < sg.rows ? pos + 1 : 0;
        row_low[n][i] = a.window > 0 ? pos + 1 - a.window : 0;
      }
    }
    // every row of the tile sees the keys [all_low, all_high)
    const int all_high = base_pos + sg.first_row / a.ratio + 1;
    const int all_low = a.window > 0 ? base_pos + (sg.first_row + sg.rows - 1) / a.ratio + 1 - a.window : 0;

    float o[NT][kChunks * 2][4] = {};
    float low_sum[NT][G][2] = {};                                      // sum of p (m + 8 s)
    float total[NT][2] = {}, top[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) top[n][0] = top[n][1] = -INFINITY;

    for (int i = 0; i < stages; ++i) {
      const int slot = (int)(taken % S::kStages);
      if (!bounded_wait_warp(ptx::smem_addr(&ctl->full[warp][slot]), (taken / S::kStages) & 1u, abort_flag, WAIT_STREAM_FULL)) {
        alive = false;
        break;
      }
      ++taken;
      const int t0 = first_token + i * S::kUnit;
      const bool edge = t0 < all_low || t0 + S::kStageTokens > all_high;
      const uint32_t kc = ring + slot * 4096, vc = kc + 2048;
      const uint32_t kp = param_ring + slot * 2 * S::kParamBytes, vp = kp + S::kParamBytes;

      // ---- scores, in units of log2
      float z[S::kSteps][NT][4];
#pragma unroll
      for (int st = 0; st < S::kSteps; ++st) {
        uint32_t words[kChunks][2];
#pragma unroll
        for (int j = 0; j < kChunks; j += 2) {
          uint32_t r[4];
          const uint32_t off = (st * 8 * D + (mat_offset ^ (j * 16))) ^ (D == 64 && (st & 1) ? 64u : 0u);
          ldmatrix_x4(r, kc + off);
          words[j][0] = r[0]; words[j][1] = r[1]; words[j + 1][0] = r[2]; words[j + 1][1] = r[3];
        }
        uint32_t pa[G], pb[G];
        load_params<G>(pa, kp + (st * 16 + g) * G * 4);
        load_params<G>(pb, kp + (st * 16 + 8 + g) * G * 4);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int k = 0; k < 4; ++k) z[st][n][k] = 0.0f;
#pragma unroll
        for (int k = 0; k < G; ++k) {
          float acc[NT][4] = {};
#pragma unroll
          for (int jj = 0; jj < kGroupChunks; ++jj) {
            const int j = k * kGroupChunks + jj;
            const uint32_t a00 = codes_128<0>(words[j][0]), a01 = codes_128<0>(words[j][1]);
            const uint32_t a10 = codes_128<1>(words[j][0]), a11 = codes_128<1>(words[j][1]);
            const uint32_t a20 = codes_128<2>(words[j][0]), a21 = codes_128<2>(words[j][1]);
            const uint32_t a30 = codes_128<3>(words[j][0]), a31 = codes_128<3>(words[j][1]);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              mma_16816(acc[n], a00, a01, a10, a11, q[n][j][0], q[n][j][1]);
              mma_16816(acc[n], a20, a21, a30, a31, q[n][j][2], q[n][j][3]);
            }
          }
          const float sa = param_step(pa[k]) * a.scale_log2, sb = param_step(pb[k]) * a.scale_log2;
          const float ma = fmaf(param_low(pa[k]), a.scale_log2, -128.0f * sa), mb = fmaf(param_low(pb[k]), a.scale_log2, -128.0f * sb);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            z[st][n][0] += fmaf(acc[n][0], sa, q_sum[n][k][0] * ma);
            z[st][n][1] += fmaf(acc[n][1], sa, q_sum[n][k][1] * ma);
            z[st][n][2] += fmaf(acc[n][2], sb, q_sum[n][k][0] * mb);
            z[st][n][3] += fmaf(acc[n][3], sb, q_sum[n][k][1] * mb);
          }
        }
      }
      if (edge) {
#pragma unroll
        for (int st = 0; st < S::kSteps; ++st) {
          const int ta = t0 + st * 16 + g, tb = ta + 8;
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              if (ta < row_low[n][k] || ta >= row_high[n][k]) z[st][n][k] = -INFINITY;
              if (tb < row_low[n][k] || tb >= row_high[n][k]) z[st][n][2 + k] = -INFINITY;
            }
        }
      }

      // ---- running maximum: raised only when some score is 2^kLazy above it (or nothing has been seen)
      float most[NT][2];
      bool raise = false;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float m = z[0][n][k];
#pragma unroll
          for (int st = 0; st < S::kSteps; ++st) m = fmaxf(m, fmaxf(z[st][n][k], z[st][n][2 + k]));
          most[n][k] = m;
          raise |= m > top[n][k] + kLazy;
        }
      if (__any_sync(0xFFFFFFFFu, raise)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float m = most[n][k];
            m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 4));
            m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 8));
            m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 16));
            m = fmaxf(m, top[n][k]);
            const float f = m == -INFINITY ? 1.0f : exp2_approx(top[n][k] - m);
            top[n][k] = m;
            total[n][k] *= f;
#pragma unroll
            for (int e = 0; e < G; ++e) low_sum[n][e][k] *= f;
#pragma unroll
            for (int u = 0; u < kChunks * 2; ++u) {
              o[n][u][k] *= f;
              o[n][u][2 + k] *= f;
            }
          }
      }

      // ---- softmax weights and the values
#pragma unroll
      for (int st = 0; st < S::kSteps; ++st) {
        uint32_t pa[G], pb[G];
        load_params<G>(pa, vp + (st * 16 + g) * G * 4);
        load_params<G>(pb, vp + (st * 16 + 8 + g) * G * 4);
        uint32_t ps[NT][G][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float p[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float m = top[n][k & 1];
            p[k] = exp2_approx(z[st][n][k] - (m == -INFINITY ? 0.0f : m));
          }
          total[n][0] += p[0] + p[2];
          total[n][1] += p[1] + p[3];
#pragma unroll
          for (int e = 0; e < G; ++e) {
            const float sa = param_step(pa[e]), sb = param_step(pb[e]);
            const float ma = fmaf(8.0f, sa, param_low(pa[e])), mb = fmaf(8.0f, sb, param_low(pb[e]));
            float wa0 = p[0] * sa, wa1 = p[1] * sa, wb0 = p[2] * sb, wb1 = p[3] * sb;
            float la0 = p[0] * ma, la1 = p[1] * ma, lb0 = p[2] * mb, lb1 = p[3] * mb;
            if (edge) {                                                // what a row does not see counts nothing, NaN or not
              const bool ha0 = z[st][n][0] == -INFINITY, ha1 = z[st][n][1] == -INFINITY;
              const bool hb0 = z[st][n][2] == -INFINITY, hb1 = z[st][n][3] == -INFINITY;
              wa0 = ha0 ? 0.0f : wa0; la0 = ha0 ? 0.0f : la0;
              wa1 = ha1 ? 0.0f : wa1; la1 = ha1 ? 0.0f : la1;
              wb0 = hb0 ? 0.0f : wb0; lb0 = hb0 ? 0.0f : lb0;
              wb1 = hb1 ? 0.0f : wb1; lb1 = hb1 ? 0.0f : lb1;
            }
            low_sum[n][e][0] += la0 + lb0;
            low_sum[n][e][1] += la1 + lb1;
            ps[n][e][0] = transpose_8x8(pack_bf16x2(wa0, wa1));
            ps[n][e][1] = transpose_8x8(pack_bf16x2(wb0, wb1));
          }
        }
#pragma unroll
        for (int j = 0; j < kChunks; j += 2) {
          uint32_t r[4];
          const uint32_t off = (st * 8 * D + (mat_offset ^ (j * 16))) ^ (D == 64 && (st & 1) ? 64u : 0u);
          ldmatrix_x4_trans(r, vc + off);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t ra = r[2 * h], rb = r[2 * h + 1];
            const uint32_t a0 = codes_centred<0>(ra), a1 = codes_centred<1>(ra), a2 = codes_centred<0>(rb), a3 = codes_centred<1>(rb);
            const uint32_t b0 = codes_centred<2>(ra), b1 = codes_centred<3>(ra), b2 = codes_centred<2>(rb), b3 = codes_centred<3>(rb);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const uint32_t* p = ps[n][(j + h) / kGroupChunks];
              mma_16816(o[n][2 * (j + h)], a0, a1, a2, a3, p[0], p[1]);
              mma_16816(o[n][2 * (j + h) + 1], b0, b1, b2, b3, p[0], p[1]);
            }
          }
        }
      }
      // the copy that takes this slot next must not overtake the reads
      ptx::fence_proxy_async_smem();
      __syncwarp();
      if (next_issue < stages) {
        issue(next_issue);
        ++next_issue;
      }
    }

    // ---- the four warps of the segment meet
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
          total[n][k] += __shfl_xor_sync(0xFFFFFFFFu, total[n][k], d);
#pragma unroll
          for (int e = 0; e < G; ++e) low_sum[n][e][k] += __shfl_xor_sync(0xFFFFFFFFu, low_sum[n][e][k], d);
        }
        if (g == 0) {
          ctl->top[warp][n * 8 + 2 * c + k] = top[n][k];
          ctl->sum[warp][n * 8 + 2 * c + k] = total[n][k];
        }
      }
    __syncthreads();
    {
      float* mine = merge + warp * (S::kRingBytes / 4);
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int r = n * 8 + 2 * c + k;
          const float m = fmaxf(fmaxf(ctl->top[0][r], ctl->top[1][r]), fmaxf(ctl->top[2][r], ctl->top[3][r]));
          const float f = m == -INFINITY ? 0.0f : exp2_approx(top[n][k] - m);
#pragma unroll
          for (int j = 0; j < kChunks; ++j) {
            const float low = low_sum[n][j / kGroupChunks][k];
            // elements 32 j + 4 g .. + 3 of row r; the 16-byte piece is turned by the row against bank conflicts
            const float4 e = make_float4((o[n][2 * j][k] + low) * f, (o[n][2 * j][2 + k] + low) * f,
                                         (o[n][2 * j + 1][k] + low) * f, (o[n][2 * j + 1][2 + k] + low) * f);
            *reinterpret_cast<float4*>(mine + r * D + (((j * 8 + g) ^ (r & 7)) << 2)) = e;
          }
        }
    }
    __syncthreads();
    // a piece that starts inside the segment goes to the worker's first slot, one that ends inside it to the second
    const int64_t part_slot = 2 * (int64_t)blockIdx.x + (u0 == 0 ? 1 : 0);
    for (int item = tid; item < S::kRows * (D / 4); item += kThreads) {
      const int r = item / (D / 4), p = item % (D / 4);
      if (r >= sg.rows) break;
      float m = ctl->top[0][r], l = 0.0f;
#pragma unroll
      for (int k = 1; k < kWarps; ++k) m = fmaxf(m, ctl->top[k][r]);
      float4 e = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
      for (int k = 0; k < kWarps; ++k) {
        const float4 y = *reinterpret_cast<const float4*>(merge + k * (S::kRingBytes / 4) + r * D + ((p ^ (r & 7)) << 2));
        e.x += y.x; e.y += y.y; e.z += y.z; e.w += y.w;
        l += m == -INFINITY ? 0.0f : ctl->sum[k][r] * exp2_approx(ctl->top[k][r] - m);
      }
      const int row = sg.first_row + r;
      const int64_t token = w.rows.first + row / a.ratio;
      const int q_head = head * a.ratio + row % a.ratio;
      if (whole) {
        const float inv = m == -INFINITY ? 0.0f : 1.0f / l;
        uint2 packed = make_uint2(pack_bf16x2(e.x * inv, e.y * inv), pack_bf16x2(e.z * inv, e.w * inv));
        *reinterpret_cast<uint2*>(a.O + token * a.o_pitch + (int64_t)q_head * D + p * 4) = packed;
        if (p == 0 && a.lse != nullptr)
          a.lse[token * a.q_heads + q_head] = m == -INFINITY ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
      } else {
        float* to = a.partial + (part_slot * S::kRows + r) * (D + 4);
        *reinterpret_cast<float4*>(to + p * 4) = e;
        if (p == 0) *reinterpret_cast<float2*>(to + D) = make_float2(m, l);
      }
    }
    ptx::fence_proxy_async_smem();                                     // the rings are filled by copies again
    __syncthreads();
    x += u1 - u0;
  }
  ptx::grid_dependents_launch();
  // a warp that gave up waits for its copies in flight before its shared memory goes
  for (; taken < issued; ++taken) {
    const uint64_t t = ptx::globaltimer_ns();
    while (!ptx::mbar_try_wait(ptx::smem_addr(&ctl->full[warp][taken % S::kStages]), (taken / S::kStages) & 1u))
      if (ptx::globaltimer_ns() - t > 50000000ull) break;
  }
}

// Joins the segments that workers share: the CTA of the first worker boundary inside a segment adds up the pieces, in the
// order of the workers.
template <int D, int G, int NT>
__global__ void __launch_bounds__(kThreads) attention_join_kernel(const AttentionArgs a, int workers) {
  using S = Shape<D, G, NT>;
  __shared__ int64_t scratch[kWarps + 2];
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  const int w = blockIdx.x + 1, r = blockIdx.y;
  const WorkPlace wp = find_work<S>(a, workers, [&](int64_t per) { return (int64_t)w * per; }, scratch);
  const int64_t x = (int64_t)w * wp.per;
  if (x >= wp.total) return;
  const SequenceWork sw = sequence_work<S>(a, wp.sequence);
  const int64_t in_seq = x - wp.before;
  const int seg = (int)(in_seq / sw.units);
  const int64_t start = wp.before + (int64_t)seg * sw.units, end = start + sw.units;
  if (start == x || start / wp.per != w - 1) return;
  const int head = seg % a.cache.kv_heads;
  const Segment sg = segment_of<S>(a, sw, seg / a.cache.kv_heads);
  if (r >= sg.rows) return;
  const int first = w - 1, last = (int)((end - 1) / wp.per);
  auto part = [&](int worker) {                                        // only the first worker's piece starts the segment
    return a.partial + ((2 * (int64_t)worker + (worker == first ? 1 : 0)) * S::kRows + r) * (D + 4);
  };
  float m = -INFINITY;
  for (int k = first; k <= last; ++k) m = fmaxf(m, ptx::ld_global(static_cast<const float*>(part(k) + D)));
  float l = 0.0f;
  float e[(D + kThreads - 1) / kThreads] = {};
  for (int k = first; k <= last; ++k) {
    const float* p = part(k);
    const float f = m == -INFINITY ? 0.0f : exp2_approx(ptx::ld_global(p + D) - m);
    l += f * ptx::ld_global(p + D + 1);
#pragma unroll
    for (int i = 0; i < (D + kThreads - 1) / kThreads; ++i)
      if (threadIdx.x + i * kThreads < D) e[i] += f * ptx::ld_global(p + threadIdx.x + i * kThreads);
  }
  const int row = sg.first_row + r;
  const int64_t token = sw.rows.first + row / a.ratio;
  const int q_head = head * a.ratio + row % a.ratio;
  const float inv = m == -INFINITY ? 0.0f : 1.0f / l;
#pragma unroll
  for (int i = 0; i < (D + kThreads - 1) / kThreads; ++i)
    if (threadIdx.x + i * kThreads < D)
      a.O[token * a.o_pitch + (int64_t)q_head * D + threadIdx.x + i * kThreads] = __bfloat16_as_ushort(__float2bfloat16_rn(e[i] * inv));
  if (threadIdx.x == 0 && a.lse != nullptr)
    a.lse[token * a.q_heads + q_head] = m == -INFINITY ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

// ------------------------------------------------------------------ host side
int row_tiles(const eqat_cache_desc& d, const eqat_attention_desc& a) {
  return (int64_t)a.max_new * (a.q_heads / d.kv_heads) <= 8 ? 1 : 2;
}

template <typename F>
int with_shape(const eqat_cache_desc& d, int nt, F&& f) {
  const int g = d.head_dim / d.group;
#define EQAT_SHAPE(DD, GG)                                                        \
  if (d.head_dim == DD && g == GG)                                                \
    return nt == 1 ? f(std::integral_constant<int, DD>(), std::integral_constant<int, GG>(), std::integral_constant<int, 1>()) \
                   : f(std::integral_constant<int, DD>(), std::integral_constant<int, GG>(), std::integral_constant<int, 2>());
  EQAT_SHAPE(64, 1)
  EQAT_SHAPE(64, 2)
  EQAT_SHAPE(128, 1)
  EQAT_SHAPE(128, 2)
  EQAT_SHAPE(128, 4)
  EQAT_SHAPE(256, 2)
  EQAT_SHAPE(256, 4)
  EQAT_SHAPE(256, 8)
#undef EQAT_SHAPE
  return EQAT_ERR_UNSUPPORTED;
}

constexpr int kMinUnits = 2;

// Units that a call can have at most, as far as the host knows.
template <typename S>
int64_t most_units(const eqat_cache_desc& d, const eqat_attention_desc& a) {
  const int64_t ratio = a.q_heads / d.kv_heads;
  const int64_t rows = (d.rows < (int64_t)a.max_new * d.sequences ? d.rows : (int64_t)a.max_new * d.sequences) * ratio;
  const int64_t tiles = rows / S::kRows + (d.sequences < d.rows ? d.sequences : d.rows);
  const int64_t units = ((int64_t)d.max_pages * d.page_size + S::kUnit - 1) / S::kUnit;
  const double total = (double)tiles * d.kv_heads * (double)(units > 0 ? units : 1);
  return total > 1e15 ? (int64_t)1e15 : (int64_t)total;
}

template <typename S>
int workers_of(const eqat_cache_desc& d, const eqat_attention_desc& a, int sms) {
  const int64_t want = (most_units<S>(d, a) + kMinUnits - 1) / kMinUnits;
  const int64_t most = (int64_t)sms * S::kCtas;
  return (int)(want < 1 ? 1 : want < most ? want : most);
}

}  // namespace

size_t cache_attention_workspace(const eqat_cache_desc& d, const eqat_attention_desc& a) {
  const int sms = sm_count();
  size_t bytes = (size_t)-1;
  with_shape(d, row_tiles(d, a), [&](auto D, auto G, auto NT) {
    using S = Shape<decltype(D)::value, decltype(G)::value, decltype(NT)::value>;
    const int w = workers_of<S>(d, a, sms > 0 ? sms : 148);
    bytes = w > 1 ? (size_t)2 * w * S::kRows * (decltype(D)::value + 4) * sizeof(float) : 0;
    return EQAT_OK;
  });
  return bytes;
}

int launch_cache_attention(const eqat_cache_desc& d, const eqat_attention_desc& at, const eqat_bf16* Q, int64_t q_pitch,
                           const CacheView& view, eqat_bf16* O, int64_t o_pitch, float* lse, void* workspace, cudaStream_t st) {
  const int sms = sm_count();
  if (sms <= 0) return EQAT_ERR_CUDA;
  return with_shape(d, row_tiles(d, at), [&](auto DD, auto GG, auto NN) {
    constexpr int D = decltype(DD)::value, G = decltype(GG)::value, NT = decltype(NN)::value;
    using S = Shape<D, G, NT>;
    AttentionArgs a{};
    a.cache = view;
    a.Q = Q;
    a.q_pitch = q_pitch;
    a.O = O;
    a.o_pitch = o_pitch;
    a.lse = lse;
    a.partial = static_cast<float*>(workspace);
    a.q_heads = at.q_heads;
    a.ratio = at.q_heads / d.kv_heads;
    a.max_new = at.max_new;
    a.window = at.window < view.max_length ? at.window : 0;              // a window of the longest sequence hides nothing
    a.scale_log2 = at.scale * kLog2e;
    a.box_tokens = d.page_size % S::kStageTokens == 0 ? S::kStageTokens : 16;
    a.min_units = kMinUnits;
    CUtensorMap km, vm;
    const uint64_t lines = (uint64_t)d.pages * d.kv_heads * d.page_size * (D / 2) / 128;
    const uint32_t box = a.box_tokens * (D / 2) / 128;
    if (!make_tmap_u8(&km, view.kq, 128, lines, 128, box, 128) || !make_tmap_u8(&vm, view.vq, 128, lines, 128, box, 128))
      return (int)EQAT_ERR_CUDA;
    static SmemOptIn opt;
    if (!opt.ensure(attention_kernel<D, G, NT>, S::kSmemBytes)) return (int)EQAT_ERR_CUDA;
    const int workers = workers_of<S>(d, at, sms);
    const int rc = launch_overlapped(attention_kernel<D, G, NT>, dim3(workers), dim3(kThreads), S::kSmemBytes, st, a, km, vm);
    if (rc != EQAT_OK || workers == 1) return rc;
    return launch_overlapped(attention_join_kernel<D, G, NT>, dim3(workers - 1, S::kRows), dim3(kThreads), 0, st, a, workers);
  });
}

int launch_wait_expiry_attention(cudaStream_t st) { return launch_wait_expiry(st); }
int read_attention_status(int* status, int* detail) { return read_wait_status(status, detail); }

}  // namespace eqat
