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
#include <type_traits>

#include "cache.cuh"
#include "common.cuh"
#include "ptx.cuh"

namespace eqat {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLazy = 8.0f;                        // a maximum may be exceeded by 2^8 before the sums are rescaled

template <int D, int G, int NT>
struct Shape {
  static constexpr int kStageTokens = 4096 / D;                 // per warp
  static constexpr int kCodeBytes = kStageTokens * D / 2;              // codes of the keys or of the values
  static constexpr int kSteps = kStageTokens / 16;
  static constexpr int kPieces = kSteps;                               // of 16 tokens, each in one page
  static constexpr int kUnit = kWarps * kStageTokens;
  static constexpr int kRows = 8 * NT;
  static constexpr int kParamBytes = kStageTokens * G * 4;
  static constexpr int kMergeFloats = kRows * D;                       // of a warp, in its ring
  static constexpr int kStages = kMergeFloats * 4 > 6 * kCodeBytes ? 4 : 3;
  static constexpr int kRingBytes = kStages * 2 * kCodeBytes;                    // codes of a warp (1024-byte aligned)
  static constexpr int kParamCopies = kPieces * 8 * G > 32 ? kPieces * 8 * G / 32 : 1;    // 16-byte copies of a lane
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
  uint32_t page_mul;           // n / (page_size / 16) = n * page_mul >> page_shift for n < 2^26
  int page_shift;
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

// Page of a token, counted in the sequence: page_size / 16 = n < 2^26 pieces, m = ceil(2^s / n) with s = 26 + ceil(log2 n):
// m n exceeds 2^s by less than n <= 2^(s - 26), so t m >> s is exact for t < 2^26.
__device__ __forceinline__ int page_index(const AttentionArgs& a, int token) {
  return (int)(((uint64_t)(uint32_t)(token >> 4) * a.page_mul) >> a.page_shift);
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
// D (16 x 8, fp32) += A (16 x 16, fp16) * B (16 x 8, fp16)
__device__ __forceinline__ void mma_fp16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// 16 bytes from global to shared memory, asynchronously; groups of copies are waited for by the thread that made them.
__device__ __forceinline__ void copy_16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int PENDING>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }
// q - 8 of the low nibbles of two bytes, times 2^-24, and of the high ones, times 2^-20: exact in fp16.
__device__ __forceinline__ uint32_t add_fp16x2(uint32_t x, uint32_t y) {
  const __half2 r = __hadd2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&y));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t centred_low(uint32_t w) { return add_fp16x2(w & 0x000F000Fu, 0x80088008u); }
__device__ __forceinline__ uint32_t centred_high(uint32_t w) { return add_fp16x2(w & 0x00F000F0u, 0x80808080u); }
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

__device__ __forceinline__ uint32_t pack_fp16x2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// ------------------------------------------------------------------ the kernel
struct AttentionCtl {
  float top[kWarps][16], sum[kWarps][16], most[16];
  int64_t scratch[kWarps + 2];
};

template <int D, int G, int NT>
__global__ void __launch_bounds__(kThreads, (Shape<D, G, NT>::kCtas))
attention_kernel(const AttentionArgs a) {
  using S = Shape<D, G, NT>;
  constexpr int kChunks = D / 32;                                      // 16-byte chunks of a row of codes
  constexpr int kGroupChunks = kChunks / G;
  extern __shared__ uint8_t smem_raw[];
  __shared__ AttentionCtl ctl_block;
  AttentionCtl* ctl = &ctl_block;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
  const uint32_t raw = ptx::smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t ring = base + warp * S::kRingBytes;
  const uint32_t param_ring = base + kWarps * S::kRingBytes + warp * S::kParamRing;
  float* merge = reinterpret_cast<float*>(smem_raw + (base - raw));
  ptx::grid_dependency_wait();

  const CacheView& v = a.cache;
  const WorkPlace wp = find_work<S>(a, gridDim.x, [&](int64_t per) { return (int64_t)blockIdx.x * per; }, ctl->scratch);
  int64_t x = (int64_t)blockIdx.x * wp.per;
  const int64_t x_end = min(x + wp.per, wp.total);
  int b = wp.sequence;
  int64_t seq_before = wp.before;

  // per-lane ldmatrix offset inside 16 tokens of codes: matrices (tokens 0-7, chunk j), (8-15, j), (0-7, j+1), (8-15, j+1)
  const uint32_t mat_token = ((lane >> 3) & 1) * 8 + (lane & 7);
  const uint32_t mat_linear = mat_token * (D / 2) + (lane >> 4) * 16;
  const uint32_t mat_offset = mat_linear ^ (((mat_linear >> 7) & 7u) << 4);
  const uint32_t copy_offset = (lane * 16) ^ (((lane * 16) >> 3) & 0x70u);

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
    const int stages = first_token < sg.high ? min(u1 - u0, (sg.high - first_token + S::kUnit - 1) / S::kUnit) : 0;
    // Lane p < kPieces holds the page of piece p of the stage that is fetched next, as it was read: what is done with it
    // waits until then.
    auto page_of = [&](int token) {
      return lane < S::kPieces && token < sg.high ? ld_index(v.page_table + (int64_t)b * v.max_pages + page_index(a, token)) : 0;
    };
    int page = page_of(first_token + 16 * lane);
    auto fetch = [&](int i, int slot) {
      if (i < stages) {
        const int t = first_token + i * S::kUnit;
        const int pieces = min(S::kPieces, (sg.high - t + 15) >> 4);
        // token slots of the pool, which are less than 2^32; a page number outside counts as the nearest inside
        const int token = t + 16 * lane;
        const uint32_t place = ((uint32_t)min(max(page, 0), v.pages - 1) * v.kv_heads + head) * v.page_size +
                               (token - page_index(a, token) * v.page_size);
        uint32_t from[S::kPieces];
#pragma unroll
        for (int p = 0; p < S::kPieces; ++p) from[p] = __shfl_sync(0xFFFFFFFFu, place, p);
#pragma unroll
        for (int p = 0; p < S::kPieces; ++p)
          if (p < pieces) {
            const uint8_t *ks = v.kq + (uint64_t)from[p] * (D / 2) + lane * 16, *vs = v.vq + (uint64_t)from[p] * (D / 2) + lane * 16;
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {                         // 512 bytes a time; copy_offset: 16-byte chunks swizzled
              const uint32_t dst = ring + slot * 2 * S::kCodeBytes + p * (8 * D) + j * 512 + (copy_offset ^ (((p * 8 * D + j * 512) >> 3) & 0x70u));
              copy_16(dst, ks + j * 512);
              copy_16(dst + S::kCodeBytes, vs + j * 512);
            }
          }
        // 4 G chunks of parameters for each piece, of the keys and of the values
#pragma unroll
        for (int e = 0; e < S::kParamCopies; ++e) {
          const int chunk = e * 32 + lane, p = chunk / (8 * G), part = chunk % (4 * G);
          const bool keys = chunk % (8 * G) < 4 * G;
          const uint32_t at = __shfl_sync(0xFFFFFFFFu, place, p);
          if (p < pieces)
            copy_16(param_ring + slot * 2 * S::kParamBytes + (keys ? 0 : S::kParamBytes) + p * 64 * G + part * 16,
                    (keys ? v.kp : v.vp) + (uint64_t)at * G + part * 4);
        }
        page = page_of(t + S::kUnit + 16 * lane);
      }
      copies_commit();
    };
    __syncwarp();
#pragma unroll
    for (int i = 0; i < S::kStages; ++i) fetch(i, i);

    // ---- the queries, in the order of the codes, and their sums per group.  A row is scaled by 2^k, so that its largest
    // element lies in [2^14, 2^15), and rounded to fp16, which holds a bf16 number exactly down to 2^-28 of the largest; `back`
    // undoes that and the 2^-24 of the codes.  (Rows beyond 2^115 become infinite.)
    uint32_t q[NT][kChunks][4];
    float q_sum[NT][G][2], back[NT][2];
    int row_low[NT][2], row_high[NT][2];                               // keys that the rows of this lane's columns see
    const int base_pos = w.rows.length - w.rows.count;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int r = n * 8 + g, row = sg.first_row + r;
      const eqat_bf16* src = a.Q + (int64_t)(w.rows.first + row / a.ratio) * a.q_pitch + (int64_t)(head * a.ratio + row % a.ratio) * D;
      uint4 e[kChunks];
      uint32_t most = 0;
#pragma unroll
      for (int j = 0; j < kChunks; ++j) {
        e[j] = make_uint4(0u, 0u, 0u, 0u);
        if (r < sg.rows) e[j] = ptx::ld_global(reinterpret_cast<const uint4*>(src + j * 32 + c * 8));
        // bf16 bit patterns without the sign compare like the numbers
        most = __vmaxu2(most, __vmaxu2(__vmaxu2(e[j].x & 0x7FFF7FFFu, e[j].y & 0x7FFF7FFFu), __vmaxu2(e[j].z & 0x7FFF7FFFu, e[j].w & 0x7FFF7FFFu)));
      }
      most = max(most & 0xFFFFu, most >> 16);
      most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
      most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
      const int k2 = most == 0 ? 0 : min(max(14 - ((int)(most >> 7) - 127), -100), 100);
      const float up = __int_as_float((127 + k2) << 23), up16 = up * 0.0625f;
      float sums[G];
#pragma unroll
      for (int k = 0; k < G; ++k) sums[k] = 0.0f;
#pragma unroll
      for (int j = 0; j < kChunks; ++j) {
        const float x0 = param_step(e[j].x), x1 = param_low(e[j].x), x2 = param_step(e[j].y), x3 = param_low(e[j].y);
        const float x4 = param_step(e[j].z), x5 = param_low(e[j].z), x6 = param_step(e[j].w), x7 = param_low(e[j].w);
        q[n][j][0] = pack_fp16x2(x0 * up, x4 * up);                    // the codes of nibbles 1 and 3 count 16-fold
        q[n][j][1] = pack_fp16x2(x1 * up16, x5 * up16);
        q[n][j][2] = pack_fp16x2(x2 * up, x6 * up);
        q[n][j][3] = pack_fp16x2(x3 * up16, x7 * up16);
        sums[j / kGroupChunks] += ((x0 + x1) + (x2 + x3)) + ((x4 + x5) + (x6 + x7));
      }
      const float down = __int_as_float((127 + 24 - k2) << 23);
#pragma unroll
      for (int i = 0; i < 2; ++i) back[n][i] = __shfl_sync(0xFFFFFFFFu, down, 8 * c + 4 * i);
#pragma unroll
      for (int k = 0; k < G; ++k) {
        sums[k] += __shfl_xor_sync(0xFFFFFFFFu, sums[k], 1);
        sums[k] += __shfl_xor_sync(0xFFFFFFFFu, sums[k], 2);
        sums[k] *= __int_as_float((127 - 24 + k2) << 23);              // in the units of the products
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
    // Weights are p = 2^(z - shift), z the score in log2: with the shift at the largest score (as of its last raise) plus
    // log2(unit) - 6, unit a power of two above all steps that the column has counted, p s lies below 2^14, in fp16's
    // range, and is exact to 2^-12 of itself from the largest (about 2^6) down to 2^-20 of it, to 2^-31 of it below.
    float total[NT][2] = {}, shift[NT][2], minus[NT][2] = {}, limit[NT][2], unit[NT][2] = {}, most[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) shift[n][0] = shift[n][1] = limit[n][0] = limit[n][1] = -INFINITY;

    int slot = 0;
    for (int i = 0; i < stages; ++i) {
      copies_wait<S::kStages - 1>();
      __syncwarp();
      const int t0 = first_token + i * S::kUnit;
      const bool edge = t0 < all_low || t0 + S::kStageTokens > all_high;
      const uint32_t kc = ring + slot * 2 * S::kCodeBytes, vc = kc + S::kCodeBytes;
      const uint32_t kp = param_ring + slot * 2 * S::kParamBytes, vp = kp + S::kParamBytes;

      // ---- scores, in units of log2 divided by `back`
      float z[S::kSteps][NT][4], acc[S::kSteps][NT][4];
      constexpr int kPairChunks = kChunks < 2 ? 1 : 2;                 // one ldmatrix
#pragma unroll
      for (int j0 = 0; j0 < kChunks; j0 += kPairChunks) {
        uint32_t words[S::kSteps][4];
#pragma unroll
        for (int st = 0; st < S::kSteps; ++st)
          ldmatrix_x4(words[st], kc + ((st * 8 * D + (mat_offset ^ (j0 * 16))) ^ (D == 64 && (st & 1) ? 64u : 0u)));
#pragma unroll
        for (int h = 0; h < kPairChunks; ++h) {
          // codes as fp16 numbers below the normal range: q 2^-24 in the low nibble of a byte, q 2^-20 in the high one
          const int j = j0 + h, k = j / kGroupChunks;
#pragma unroll
          for (int st = 0; st < S::kSteps; ++st) {
            if (j % kGroupChunks == 0)
#pragma unroll
              for (int n = 0; n < NT; ++n) acc[st][n][0] = acc[st][n][1] = acc[st][n][2] = acc[st][n][3] = 0.0f;
            const uint32_t wa = words[st][2 * h], wb = words[st][2 * h + 1];
#pragma unroll
            for (int n = 0; n < NT; ++n)
              mma_fp16(acc[st][n], wa & 0x000F000Fu, wb & 0x000F000Fu, wa & 0x00F000F0u, wb & 0x00F000F0u, q[n][j][0], q[n][j][1]);
          }
#pragma unroll
          for (int st = 0; st < S::kSteps; ++st) {
            const uint32_t xa = words[st][2 * h] >> 8, xb = words[st][2 * h + 1] >> 8;
#pragma unroll
            for (int n = 0; n < NT; ++n)
              mma_fp16(acc[st][n], xa & 0x000F000Fu, xb & 0x000F000Fu, xa & 0x00F000F0u, xb & 0x00F000F0u, q[n][j][2], q[n][j][3]);
          }
          if (j % kGroupChunks == kGroupChunks - 1) {
#pragma unroll
            for (int st = 0; st < S::kSteps; ++st) {
              const uint32_t pa = ptx::lds_32(kp + ((st * 16 + g) * G + k) * 4), pb = ptx::lds_32(kp + ((st * 16 + 8 + g) * G + k) * 4);
              const float sa = param_step(pa) * a.scale_log2, sb = param_step(pb) * a.scale_log2;
              const float ma = param_low(pa) * a.scale_log2, mb = param_low(pb) * a.scale_log2;
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                float* zz = z[st][n];
                zz[0] = fmaf(acc[st][n][0], sa, k == 0 ? q_sum[n][k][0] * ma : fmaf(q_sum[n][k][0], ma, zz[0]));
                zz[1] = fmaf(acc[st][n][1], sa, k == 0 ? q_sum[n][k][1] * ma : fmaf(q_sum[n][k][1], ma, zz[1]));
                zz[2] = fmaf(acc[st][n][2], sb, k == 0 ? q_sum[n][k][0] * mb : fmaf(q_sum[n][k][0], mb, zz[2]));
                zz[3] = fmaf(acc[st][n][3], sb, k == 0 ? q_sum[n][k][1] * mb : fmaf(q_sum[n][k][1], mb, zz[3]));
              }
            }
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

      // ---- steps and minima of the values, and the largest step that each column counts
      uint32_t vpar[S::kSteps][2][G];
      float widest[NT][2];
      {
        float all = 0.0f;
#pragma unroll
        for (int st = 0; st < S::kSteps; ++st)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            load_params<G>(vpar[st][h], vp + (st * 16 + 8 * h + g) * G * 4);
#pragma unroll
            for (int e = 0; e < G; ++e) all = fmaxf(all, param_step(vpar[st][h][e]));
          }
#pragma unroll
        for (int n = 0; n < NT; ++n) widest[n][0] = widest[n][1] = all;
      }
      if (edge) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float all = 0.0f;
#pragma unroll
            for (int st = 0; st < S::kSteps; ++st)
#pragma unroll
              for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < G; ++e)
                  all = fmaxf(all, z[st][n][2 * h + k] == -INFINITY ? 0.0f : param_step(vpar[st][h][e]));
            widest[n][k] = all;
          }
      }

      // ---- the columns' exponents are raised only when a score is 2^kLazy above the last maximum or a step above the last
      // unit (or nothing has been seen)
      bool raise = false;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float m = z[0][n][k];
#pragma unroll
          for (int st = 0; st < S::kSteps; ++st) m = fmaxf(m, fmaxf(z[st][n][k], z[st][n][2 + k]));
          most[n][k] = m;
          raise |= m * back[n][k] > limit[n][k] || widest[n][k] > unit[n][k];
        }
      if (__any_sync(0xFFFFFFFFu, raise)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float m = most[n][k], u = widest[n][k];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) {
              m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
              u = fmaxf(u, __shfl_xor_sync(0xFFFFFFFFu, u, d));
            }
            m = fmaxf(m * back[n][k], limit[n][k] - kLazy);
            if (u > unit[n][k])                                        // the next power of two
              unit[n][k] = __uint_as_float((uint32_t)min(max((int)(__float_as_uint(u) >> 23) + 1, 127 - 60), 254) << 23);
            const float to = m == -INFINITY ? -INFINITY : m + (float)((int)(__float_as_uint(unit[n][k]) >> 23) - 127 - 6);
            const float f = to == -INFINITY ? 1.0f : exp2_approx(shift[n][k] - to);
            limit[n][k] = m + kLazy;
            shift[n][k] = to;
            minus[n][k] = to == -INFINITY ? 0.0f : -to;
            total[n][k] *= f;
#pragma unroll
            for (int e = 0; e < G; ++e) low_sum[n][e][k] *= f;
#pragma unroll
            for (int u2 = 0; u2 < kChunks * 2; ++u2) {
              o[n][u2][k] *= f;
              o[n][u2][2 + k] *= f;
            }
          }
      }

      // ---- softmax weights and the values
#pragma unroll
      for (int st = 0; st < S::kSteps; ++st) {
        uint32_t ps[NT][G][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float p[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) p[k] = exp2_approx(fmaf(z[st][n][k], back[n][k & 1], minus[n][k & 1]));
          total[n][0] += p[0] + p[2];
          total[n][1] += p[1] + p[3];
#pragma unroll
          for (int e = 0; e < G; ++e) {
            const float sa = param_step(vpar[st][0][e]), sb = param_step(vpar[st][1][e]);
            const float ma = fmaf(8.0f, sa, param_low(vpar[st][0][e])), mb = fmaf(8.0f, sb, param_low(vpar[st][1][e]));
            float wa0 = p[0] * sa, wa1 = p[1] * sa, wb0 = p[2] * sb, wb1 = p[3] * sb;
            if (!edge) {
              low_sum[n][e][0] = fmaf(p[0], ma, fmaf(p[2], mb, low_sum[n][e][0]));
              low_sum[n][e][1] = fmaf(p[1], ma, fmaf(p[3], mb, low_sum[n][e][1]));
            } else {                                                   // what a row does not see counts nothing, NaN or not
              const bool ha0 = z[st][n][0] == -INFINITY, ha1 = z[st][n][1] == -INFINITY;
              const bool hb0 = z[st][n][2] == -INFINITY, hb1 = z[st][n][3] == -INFINITY;
              wa0 = ha0 ? 0.0f : wa0; wa1 = ha1 ? 0.0f : wa1;
              wb0 = hb0 ? 0.0f : wb0; wb1 = hb1 ? 0.0f : wb1;
              low_sum[n][e][0] += (ha0 ? 0.0f : p[0] * ma) + (hb0 ? 0.0f : p[2] * mb);
              low_sum[n][e][1] += (ha1 ? 0.0f : p[1] * ma) + (hb1 ? 0.0f : p[3] * mb);
            }
            ps[n][e][0] = transpose_8x8(pack_fp16x2(wa0, wa1));
            ps[n][e][1] = transpose_8x8(pack_fp16x2(wb0, wb1));
          }
        }
#pragma unroll
        for (int j = 0; j < kChunks; j += 2) {
          uint32_t r[4];
          const uint32_t off = (st * 8 * D + (mat_offset ^ (j * 16))) ^ (D == 64 && (st & 1) ? 64u : 0u);
          ldmatrix_x4_trans(r, vc + off);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t ra = r[2 * h], rb = r[2 * h + 1], xa = ra >> 8, xb = rb >> 8;
            const uint32_t a0 = centred_low(ra), a1 = centred_high(ra), a2 = centred_low(rb), a3 = centred_high(rb);
            const uint32_t b0 = centred_low(xa), b1 = centred_high(xa), b2 = centred_low(xb), b3 = centred_high(xb);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              const uint32_t* p = ps[n][(j + h) / kGroupChunks];
              mma_fp16(o[n][2 * (j + h)], a0, a1, a2, a3, p[0], p[1]);
              mma_fp16(o[n][2 * (j + h) + 1], b0, b1, b2, b3, p[0], p[1]);
            }
          }
        }
      }
      __syncwarp();                                                    // the stage has been read
      fetch(i + S::kStages, slot);
      slot = slot + 1 == S::kStages ? 0 : slot + 1;
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
        if (g == 0) ctl->top[warp][n * 8 + 2 * c + k] = shift[n][k];
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
          const float f = m == -INFINITY ? 0.0f : exp2_approx(shift[n][k] - m);
          const float even = f * 0x1p24f, odd = f * 0x1p20f;           // the units of the codes
          if (g == 0) ctl->sum[warp][r] = total[n][k] * f;
#pragma unroll
          for (int j = 0; j < kChunks; ++j) {
            const float low = low_sum[n][j / kGroupChunks][k] * f;
            // elements 32 j + 4 g .. + 3 of row r; the 16-byte piece is turned by the row against bank conflicts
            const float4 e = make_float4(fmaf(o[n][2 * j][k], even, low), fmaf(o[n][2 * j][2 + k], odd, low),
                                         fmaf(o[n][2 * j + 1][k], even, low), fmaf(o[n][2 * j + 1][2 + k], odd, low));
            *reinterpret_cast<float4*>(mine + r * D + (((j * 8 + g) ^ (r & 7)) << 2)) = e;
          }
          if (g == 0 && warp == 0) ctl->most[r] = m;
        }
    }
    __syncthreads();
    // a piece that starts inside the segment goes to the worker's first slot, one that ends inside it to the second
    const int64_t part_slot = 2 * (int64_t)blockIdx.x + (u0 == 0 ? 1 : 0);
    for (int r = warp; r < sg.rows; r += kWarps) {
      const float m = ctl->most[r], l = (ctl->sum[0][r] + ctl->sum[1][r]) + (ctl->sum[2][r] + ctl->sum[3][r]);
      const int row = sg.first_row + r;
      const int64_t token = w.rows.first + row / a.ratio;
      const int q_head = head * a.ratio + row % a.ratio;
      const float inv = m == -INFINITY ? 0.0f : 1.0f / l;
      eqat_bf16* out = a.O + token * a.o_pitch + (int64_t)q_head * D;
      float* part = whole ? nullptr : a.partial + (part_slot * S::kRows + r) * (D + 4);
#pragma unroll
      for (int p = lane; p < D / 4; p += 32) {
        float4 e = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < kWarps; ++k) {
          const float4 y = *reinterpret_cast<const float4*>(merge + k * (S::kRingBytes / 4) + r * D + ((p ^ (r & 7)) << 2));
          e.x += y.x; e.y += y.y; e.z += y.z; e.w += y.w;
        }
        if (whole) *reinterpret_cast<uint2*>(out + p * 4) = make_uint2(pack_bf16x2(e.x * inv, e.y * inv), pack_bf16x2(e.z * inv, e.w * inv));
        else *reinterpret_cast<float4*>(part + p * 4) = e;
      }
      if (lane == 0) {
        if (!whole) *reinterpret_cast<float2*>(part + D) = make_float2(m, l);
        else if (a.lse != nullptr)
          a.lse[token * a.q_heads + q_head] = m == -INFINITY ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
      }
    }
    __syncthreads();                                                   // the rings may be filled again
    x += u1 - u0;
  }
  ptx::grid_dependents_launch();
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

int log2_up(int v) {
  int s = 0;
  while ((1 << s) < v) ++s;
  return s;
}

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
    a.page_shift = 26 + log2_up(d.page_size / 16);
    a.page_mul = (uint32_t)((((uint64_t)1 << a.page_shift) + d.page_size / 16 - 1) / (d.page_size / 16));
    a.min_units = kMinUnits;
    static SmemOptIn opt;
    if (!opt.ensure(attention_kernel<D, G, NT>, S::kSmemBytes)) return (int)EQAT_ERR_CUDA;
    const int workers = workers_of<S>(d, at, sms);
    const int rc = launch_overlapped(attention_kernel<D, G, NT>, dim3(workers), dim3(kThreads), S::kSmemBytes, st, a);
    if (rc != EQAT_OK || workers == 1) return rc;
    return launch_overlapped(attention_join_kernel<D, G, NT>, dim3(workers - 1, S::kRows), dim3(kThreads), 0, st, a, workers);
  });
}

}  // namespace eqat
