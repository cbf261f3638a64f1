// Attention of new tokens over the 4-bit cache, on the tensor cores without expanding a code to more than a byte.
//
// A CTA takes a tile of 128 tokens of one key/value head at a time, for 1 to 32 query rows (new tokens x the query heads
// that share the head).  With step s and minimum m of a group and q a code, K = q s + m and V likewise, so
//     Q . K_t       = sum over groups of  s_t (sum_d Q_d q_td) + m_t (sum_d Q_d)
//     sum_t p_t V_t = sum_t (p_t s_t) q_t + sum_t p_t m_t:
// the codes enter both products as they are, as bytes, and steps and minima multiply sums.  Tokens are the 128 rows of the
// first product and elements of the head those of the second, so eight query rows are eight columns and not an eighth of a
// 128-row tile; each code costs three operations per eight and one byte of shared memory.
//   scores   kind::f8f6f4: the byte q is the e4m3 number q 2^-9 (0..7 below the normal range, 8..15 in the first binade).
//            A query row is scaled by a power of two and split into two e4m3 numbers, the second one 2^-4 finer: exact for
//            bf16 down to 2^-13 of the row's largest element, to 2^-22 of it below.
//   values   kind::i8: p s as an integer of up to 23 bits, its three bytes as columns of their own, unsigned codes, sums exact
//            in 32 bits.  (In fp32 the sums of the uncentred codes would be rounded at some thousand times the size of a long
//            even softmax's output.)
// Groups of the keys are ranges of K with accumulators of their own, groups of the values have columns of their own.
//
// Every thread is one token of the tile in the softmax: scores arrive as columns of its lane of tensor memory, so no value
// is exchanged between threads but a vote: a row's exponent is changed only when a weight leaves the range of the 23 bits,
// then the integer sums are emptied into fp32 registers (a thread is one element of the head there).
//
// What bounds it: a tile costs the SM's shared-memory and L1 data path 256 cycles for writing the bytes, 256 for the tensor
// core's reads of them, about 150 for fetching the codes and some 100 for weights and constants, of 1000 that it takes (HBM
// would deliver one in 750); of the issue slots 51 % are taken.  8 x 65536 tokens, 64/8 heads, groups of 128: 142 us, 4.0 TB/s;
// with one query head per key/value head 122 us, 4.7 TB/s (single calls, nothing in the L2).  64 x 4096 tokens of uneven
// lengths, pages of 16: 59 us, 3.1 TB/s; there the ends of segments (queries, first raise, sums over the threads) take a fifth.
// Measured and not kept, beside 61 us for the last of these:
//   codes as fp16 operands of mma.sync m16n8k16, fed by ldmatrix (the first form)   64 x 4096: 63 us, 8 x 65536 slower by 12 %
//   four warps that fetch and spread beside four that weigh                         69 us: the same data path
//   scores of the next tile under this one's weights, one barrier a tile            73 us
//   five CTAs an SM in 96 registers                                                 99 us
// and kept: codes fetched past the L1 (64.8 -> 60.9 us).
//
// Work is dealt out in tiles: those of all (sequence, row tile, head) segments are laid end to end and every CTA takes an
// equal stretch, so batches of any lengths fill the device.  A segment that several CTAs share is joined by a second small
// kernel in a fixed order.
#include <type_traits>

#include "attention.cuh"
#include "common.cuh"
#include "ptx.cuh"
#include "wait.cuh"

namespace eqat {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32, kJoinThreads = 256;
// Weights are p = 2^(z - top), z the score in log2 and top the row's largest as of its last raise.  The integers are
// w = p s 2^E, rounded, with E of the row such that its largest p s so far, whichever token has it, lies in [2^20, 2^21): a
// token with large steps that the row hardly sees leaves the others their bits, and so does one that takes nearly all of the
// softmax and has small steps.  A raise makes both anew; it comes when some w would pass 2^23, or p 2^kLazy.
// w is rounded down after a number in [0, 1) has been added that depends on the token's position alone (the fractions of
// multiples of the golden ratio): a long tail of weights below half a unit then counts what it should in the mean.  Rounded to
// the nearest they would be lost from sum w q and not from sum p and sum p m, which pulled the outputs of rows with one
// dominant token to the minima of all others' groups.  What is a whole number already stays one.  The error of an output is
// about that of sqrt(tokens) / 3 units in its sum: 2^-12 of the largest p s q for a million tokens.
constexpr float kLazy = 8.0f, kTop = 20.0f;
constexpr int kLeastExponent = -115, kMostExponent = 118;              // of 2^E; p 2^E stays finite
constexpr float kWeightLimit = 8388608.0f * (1.0f - 0x1p-10f);

// D: elements of a head, G: groups in it, ROWS: query rows of a tile (1, 4, or a multiple of eight).
template <int D, int G, int ROWS>
struct Shape {
  static constexpr int NB = (ROWS + 7) / 8;                            // blocks of eight rows: columns come in sixteens
  static constexpr int kStageTokens = 16;                              // segments start at a multiple of this
  static constexpr int kUnit = 128;                                    // tokens of a tile
  static constexpr int kRows = ROWS;
  static constexpr int kBlocks = D > 128 ? D / 128 : 1;                // blocks of 128 elements
  static constexpr int kBlockGroups = G / kBlocks;
  // Columns come in eights.  Few rows share one eight over the groups of a block: slot = group * ROWS + row.
  static constexpr bool kShared = ROWS * G <= 8;
  static constexpr int kSlots = ROWS * kBlockGroups;                   // of a block, where they are shared
  static constexpr int kParts = kShared ? 1 : NB * kBlockGroups;       // eights of a block
  static constexpr int kWeightUnits = kParts == 1 ? 2 : kParts + kParts / 2;      // 16-byte units of a token's weights, per block
  static constexpr int kWeightCols = 16 * kWeightUnits;
  static constexpr int kScoreCols = kShared ? 16 : 16 * NB * G;
  static constexpr int kSumCols = kBlocks * kWeightCols;
  // tensor memory: sums, then scores; 160 columns are taken as 128 + 32, with the last two groups' scores in the 32
  static constexpr int kCols = kScoreCols + kSumCols;
  static constexpr bool kTwoParts = kCols > 128 && kCols <= 160 && G >= 2 && NB == 1 && !kShared;
  static constexpr int kAlloc = kCols <= 64 ? 64 : kCols <= 128 || kTwoParts ? 128 : kCols <= 256 ? 256 : 512;
  static constexpr int kOperandBytes = kBlocks * 128 * 128;            // of keys or values: 128 tokens x 128 bytes a block
  static constexpr int kWeightBytes = kBlocks * kWeightUnits * 2048;
  static constexpr int kQueryBytes = kBlocks * NB * 2048;
  static constexpr int kNeedBytes = 1024 + 2 * kOperandBytes + kWeightBytes + kQueryBytes;
  // Two CTAs that each hold one part and wait for the other must not fill the tensor memory: no more than three of them fit
  // on an SM (4 * 57 KB are more than it has).
  static constexpr int kSmemBytes = kTwoParts && kNeedBytes < 57 * 1024 ? 57 * 1024 : kNeedBytes;
  static constexpr int kTmemCtas = 512 / (kAlloc + (kTwoParts ? 32 : 0));
  static constexpr int kSmemCtas = 227 * 1024 / (kSmemBytes + 4096);
  static constexpr int kRegCtas = kRows * (1 + G + kBlocks) <= 40 && D <= 128 ? 4 : 3;
  static constexpr int kCtas = kTmemCtas < kSmemCtas ? (kTmemCtas < kRegCtas ? kTmemCtas : kRegCtas) : (kSmemCtas < kRegCtas ? kSmemCtas : kRegCtas);
  static constexpr int kLoads = D / 32;                                // 16-byte loads of a lane per tile, keys or values
  static_assert((1 + G) * kRows * 512 <= 2 * kOperandBytes && kRows * D * 4 <= 2 * kOperandBytes, "sums meet in the operands' memory");
  static_assert(kCols <= 512, "tensor memory");
};

struct WorkPlace {
  int64_t total, per;          // units of the call, of a worker
  int64_t before;              // units of the sequences before `sequence`
  int sequence;                // that holds unit `x` (or sequences, if none does)
};
// Whole CTA: finds the sequence of unit x, which may depend on the total (x = f(per)).
template <typename S, typename F>
__device__ __forceinline__ WorkPlace find_work(const AttentionArgs& a, int workers, F&& f, int64_t* scratch) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (a.cache.sequences <= 32) {                                         // every warp by itself
    SequenceWork w{};
    if (lane < a.cache.sequences) w = sequence_work<S>(a, lane);
    const int64_t own = work_units(a.cache, w);
    int64_t upto = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t o = __shfl_up_sync(0xFFFFFFFFu, upto, d);
      if (lane >= d) upto += o;
    }
    WorkPlace p;
    p.total = __shfl_sync(0xFFFFFFFFu, upto, 31);
    // A tile takes a worker about a microsecond, a piece of a segment the join 0.06: few tiles for a worker where a segment
    // is short, sqrt(tiles / 16) where it is cut into many pieces (one head, 30000 tokens: 27.8 us with one, 17.8 with four).
    // More than 32 sequences of such lengths have tiles enough for all workers.
    const unsigned longest = __reduce_max_sync(0xFFFFFFFFu, w.tiles > 0 ? (unsigned)w.units : 0u);
    p.per = max(quotient(p.total + workers - 1, workers), (int64_t)max(1, (int)sqrtf((float)longest * 0.0625f)));
    const uint32_t behind = __ballot_sync(0xFFFFFFFFu, upto > f(p.per));     // sequences that end behind unit x
    p.sequence = behind == 0u ? a.cache.sequences : __ffs(behind) - 1;
    p.before = __shfl_sync(0xFFFFFFFFu, upto - own, behind == 0u ? 0 : __ffs(behind) - 1);
    return p;
  }
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
  p.per = max(quotient(total + workers - 1, workers), (int64_t)1);
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

// ------------------------------------------------------------------ instructions
// D[tmem] (+)= A[smem] * B[smem], bytes: e4m3 numbers with fp32 sums, unsigned integers with 32-bit sums.
__device__ __forceinline__ void mma_e4m3(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_u8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
      ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
// Instruction descriptors: fp32 sums of e4m3, both operands K-major; 32-bit sums of u8, both MN-major.
constexpr uint32_t kScoreDesc = (1u << 4) | (8u << 24);
constexpr uint32_t kSumDesc = (2u << 4) | (1u << 15) | (1u << 16) | (8u << 24);
// Matrix descriptor of the weights: MN-major without swizzle, 16-byte units of columns 2048 bytes apart, 8 tokens 128.
__device__ __forceinline__ uint64_t weight_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(128u >> 4) << 16) | ((uint64_t)(2048u >> 4) << 32) | (1ull << 46);
}
// Two numbers as e4m3, low byte first, and back.
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 from_e4m3x2(uint32_t v) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)v));
  return __half22float2(*reinterpret_cast<const __half2*>(&r));
}
__device__ __forceinline__ void sts_8(uint32_t addr, uint32_t v) { asm volatile("st.shared.u8 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void sts_32(uint32_t addr, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(addr), "r"(v) : "memory"); }
__device__ __forceinline__ void sts_64(uint32_t addr, uint32_t a, uint32_t b) {
  asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(addr), "r"(a), "r"(b) : "memory");
}
template <int G>
__device__ __forceinline__ void load_params(uint32_t (&r)[G], const uint32_t* p) {
  if constexpr (G == 1) {
    r[0] = ptx::ld_global(p);
  } else if constexpr (G == 2) {
    const uint2 v = ptx::ld_global(reinterpret_cast<const uint2*>(p));
    r[0] = v.x; r[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < G; i += 4) {
      const uint4 v = ptx::ld_global(reinterpret_cast<const uint4*>(p) + i / 4);
      r[i] = v.x; r[i + 1] = v.y; r[i + 2] = v.z; r[i + 3] = v.w;
    }
  }
}
// ------------------------------------------------------------------ the kernel
template <int ROWS, int G>
struct AttentionCtl {
  uint64_t scores_done, sums_done;
  uint32_t tmem[2];
  int abort;
  // of the query rows
  alignas(16) float back[ROWS], minus[ROWS], limit[ROWS];      // score in log2 = z * back; minus = -top; arg above limit: raise
  alignas(16) float weight[ROWS], grain[ROWS];         // 2^E, 2^-E
  float top[ROWS], peak[ROWS], factor[ROWS], delta[ROWS];      // peak: log2 of the largest 2^z s
  alignas(16) float q_sum[G][ROWS];
  int low[ROWS], high[ROWS];                           // keys that the row sees
  float warp_top[kWarps][ROWS], warp_peak[kWarps][ROWS];
  float sums[1 + G][ROWS];
  int64_t scratch[kWarps + 2];
};

template <int D, int G, int ROWS>
__global__ void __launch_bounds__(kThreads, (Shape<D, G, ROWS>::kCtas))
attention_kernel(const AttentionArgs a) {
  using S = Shape<D, G, ROWS>;
  constexpr int kRows = ROWS, NB = S::NB, kGroup = D / G, kChunks = D / 32;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(16) AttentionCtl<8 * NB, G> ctl_block;
  AttentionCtl<8 * NB, G>* ctl = &ctl_block;
  volatile int* abort_flag = &ctl->abort;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t raw = ptx::smem_addr(smem_raw), base = (raw + 1023u) & ~1023u;
  const uint32_t keys = base, values = keys + S::kOperandBytes, weights = values + S::kOperandBytes, queries = weights + S::kWeightBytes;
  float* meet = reinterpret_cast<float*>(smem_raw + (base - raw));       // the operands' memory, between segments
  // where this lane's first chunk goes in `keys`, as even codes (the odd ones: the other of two 16-byte pieces), and its
  // token's weights
  const uint32_t chunk_at = keys + (lane % kChunks / 4) * 16384 + (32 * warp + lane / kChunks) * 128 +
                            (((lane % kChunks % 4 * 2) ^ (lane / kChunks & 7)) << 4);
  const uint32_t weight_at = weights + tid * 16;

  if (tid == 0) {
    ptx::mbar_init(ptx::smem_addr(&ctl->scores_done), 1);
    ptx::mbar_init(ptx::smem_addr(&ctl->sums_done), 1);
    ctl->abort = 0;
    ptx::fence_mbar_init();
  }
  if (warp == 0) {
    take_columns(ptx::smem_addr(&ctl->tmem[0]), S::kAlloc);
    if (S::kTwoParts) take_columns(ptx::smem_addr(&ctl->tmem[1]), 32);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  for (int i = tid; i < S::kWeightBytes / 16; i += kThreads) ptx::sts_128(weights + i * 16, 0u, 0u, 0u, 0u);   // rows beyond ROWS stay so
  const uint32_t sum_tmem = ctl->tmem[0], own_lanes = (uint32_t)(warp * 32) << 16;
  auto score_tmem = [&](int group) -> uint32_t {                         // of the 16 NB columns of a group
    if (S::kTwoParts && group >= G - 2) return ctl->tmem[1] + 16 * (group - (G - 2));
    return sum_tmem + S::kSumCols + group * 16 * NB;
  };
  const uint64_t keys_desc = ptx::smem_desc(keys), queries_desc = ptx::smem_desc(queries), values_desc = ptx::smem_desc(values),
                 weights_desc = weight_desc(weights);
  ptx::grid_dependency_wait();

  const CacheView& v = a.cache;
  const WorkPlace wp = find_work<S>(a, gridDim.x, [&](int64_t per) { return (int64_t)blockIdx.x * per; }, ctl->scratch);
  int64_t x = (int64_t)blockIdx.x * wp.per;
  const int64_t x_begin = x;
  const int64_t x_end = min(x + wp.per, wp.total);
  int b = wp.sequence;
  int64_t seq_before = wp.before;
  uint32_t scores_phase = 0, sums_phase = 0;
  if (tid == 0 && a.records != nullptr) a.records[blockIdx.x].workers = 0;

  // The segment, or the part of one, that starts with unit x.
  struct Job {
    SequenceRows rows;
    Segment sg;
    int sequence, head, u0, u1, first_token, tiles;
    bool whole;
  };
  auto next_job = [&] {
    SequenceWork w = sequence_work<S>(a, b);
    int64_t have = work_units(v, w);
    while (x >= seq_before + have) {                                     // sequences without rows have no units
      seq_before += have;
      w = sequence_work<S>(a, ++b);
      have = work_units(v, w);
    }
    const int64_t in_seq = x - seq_before;
    const int seg = (int)quotient(in_seq, w.units), tile = seg / v.kv_heads;
    Job j;
    j.rows = w.rows;
    j.sequence = b;
    j.head = seg - tile * v.kv_heads;
    j.sg = segment_of<S>(a, w, tile);
    j.u0 = (int)(in_seq - (int64_t)seg * w.units);
    j.u1 = (int)min((int64_t)w.units, j.u0 + (x_end - x));
    j.whole = j.u0 == 0 && j.u1 == w.units;
    j.first_token = j.sg.from + j.u0 * S::kUnit;
    j.tiles = j.first_token < j.sg.high ? min(j.u1 - j.u0, (j.sg.high - j.first_token + S::kUnit - 1) / S::kUnit) : 0;
    if (tid == 0 && j.u0 == 0 && !j.whole)                               // the worker's last segment
      a.records[blockIdx.x] = JoinRecord{j.rows.first, j.sg.first_row, j.sg.rows, j.head, (int)quotient(x + w.units - 1, wp.per) - (int)blockIdx.x + 1, {0, 0, 0}};
    x += j.u1 - j.u0;
    return j;
  };

  // ---- fetching: a warp has 32 tokens of the tile, two pieces of 16 that lie in one page each; lanes 0 and 1 hold the
  // pages of the next tile's pieces, as they were read
  const uint8_t *key_lane = v.kq + lane * 16, *value_lane = v.vq + lane * 16;
  const uint32_t *key_param_lane = v.kp + (lane & 15) * G, *value_param_lane = v.vp + (lane & 15) * G;
  int page = 0;
  struct Places { uint32_t at[2]; };                                     // token slots of the pool, less than 2^32
  auto page_of = [&](const Job& j, int i) {
    const int token = j.first_token + i * S::kUnit + 32 * warp + 16 * lane;
    return lane < 2 && token < j.sg.high ? ld_index(v.page_table + (int64_t)j.sequence * v.max_pages + page_index(a, token)) : 0;
  };
  auto find = [&](const Job& j, int i) {                                 // the places of tile i (called for 0, 1, 2 ...)
    const int token = j.first_token + i * S::kUnit + 32 * warp + 16 * lane;
    // a page number outside the pool counts as the nearest inside
    const uint32_t at = ((uint32_t)min(max(page, 0), v.pages - 1) * v.kv_heads + j.head) * v.page_size + (token - page_index(a, token) * v.page_size);
    page = page_of(j, i + 1);
    return Places{{__shfl_sync(0xFFFFFFFFu, at, 0), __shfl_sync(0xFFFFFFFFu, at, 1)}};
  };
  // 16-byte chunks i * 32 + lane of the warp's 32 tokens; what is not fetched keeps the codes of before
  auto fetch = [&](uint4 (&to)[S::kLoads], const uint8_t* from, const Places& place, int left) {
#pragma unroll
    for (int p = 0; p < 2; ++p)
      if (16 * p < left) {
        const uint4* at = reinterpret_cast<const uint4*>(from + (uint64_t)place.at[p] * (D / 2));
#pragma unroll
        for (int j = 0; j < S::kLoads / 2; ++j) to[p * (S::kLoads / 2) + j] = ptx::ld_global_once(at + 32 * j);
      }
  };
  auto fetch_params = [&](uint32_t (&to)[G], const uint32_t* from, const Places& place, int left) {      // of this thread's token
    if ((lane & 16) < left) load_params<G>(to, from + (uint64_t)(lane < 16 ? place.at[0] : place.at[1]) * G);
  };
  auto left_of = [&](const Job& j, int i) { return j.sg.high - (j.first_token + i * S::kUnit + 32 * warp); };      // tokens from the warp's first on
  // Codes of a chunk (32 j .. 32 j + 31 of a token) as bytes: the even ones are 16 bytes 2 j of the token's row, the odd
  // ones 16 bytes 2 j + 1; 16-byte pieces swizzled by the row.
  auto spread = [&](const uint4 (&from)[S::kLoads], int operand) {
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const uint32_t at = (kChunks == 8 && (i & 1) ? chunk_at ^ 64u : chunk_at) + operand + i * (32 / kChunks * 128), odd = at ^ 16u;
      const uint4 c = from[i];
      ptx::sts_128(at, c.x & 0x0F0F0F0Fu, c.y & 0x0F0F0F0Fu, c.z & 0x0F0F0F0Fu, c.w & 0x0F0F0F0Fu);
      ptx::sts_128(odd, (c.x >> 4) & 0x0F0F0F0Fu, (c.y >> 4) & 0x0F0F0F0Fu, (c.z >> 4) & 0x0F0F0F0Fu, (c.w >> 4) & 0x0F0F0F0Fu);
    }
  };
  uint4 key_codes[S::kLoads] = {}, value_codes[S::kLoads] = {};
  uint32_t next_key_params[G] = {}, next_value_params[G] = {};
  auto fetch_first = [&](const Job& j) {
    if (j.tiles > 0) {
      const Places place = find(j, 0);
      const int left = left_of(j, 0);
      fetch(key_codes, key_lane, place, left);
      fetch_params(next_key_params, key_param_lane, place, left);
      fetch(value_codes, value_lane, place, left);
      fetch_params(next_value_params, value_param_lane, place, left);
    }
  };

  Job job;
  if (x < x_end) {
    job = next_job();
    page = page_of(job, 0);
    fetch_first(job);
  }
  for (bool more = x_begin < x_end; more;) {
    const Segment& sg = job.sg;
    const int tiles = job.tiles;

    // ---- the queries: 16 threads a row, scaled so that the largest element lies in [128, 256), in the order of the codes
    const int base_pos = job.rows.length - job.rows.count;
#pragma unroll
    for (int rb = 0; rb < NB; ++rb) {
      constexpr int kEach = D / 16;                                      // elements of a thread
      // shared eights: the row once for each group, with zeros for the other groups
      const int slot = rb * 8 + tid / 16, part = tid % 16, r = S::kShared ? slot % kRows : slot, row = sg.first_row + r;
      const int new_token = token_of_row(a, row), group = slot / kRows;
      const bool real = r < sg.rows && (!S::kShared || group < G);
      uint32_t e[kEach / 2] = {};
      if (real) {
        const eqat_bf16* src = a.Q + (int64_t)(job.rows.first + new_token) * a.q_pitch + (int64_t)(job.head * a.ratio + row - new_token * a.ratio) * D + part * kEach;
#pragma unroll
        for (int j = 0; j < kEach / 2; j += 2) {
          const uint2 y = ptx::ld_global(reinterpret_cast<const uint2*>(src + 2 * j));
          e[j] = y.x; e[j + 1] = y.y;
        }
      }
      uint32_t most = 0;                                                 // bf16 patterns without the sign compare like the numbers
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < kEach / 2; ++j) {
        most = __vmaxu2(most, e[j] & 0x7FFF7FFFu);
        if (S::kShared && part * kEach / kGroup != group) e[j] = 0u;
        sum += (param_step(e[j]) + param_low(e[j])) * 0x1p-9f;           // (128 of the largest numbers stay finite)
      }
      most = max(most & 0xFFFFu, most >> 16);
#pragma unroll
      for (int d = 1; d < 16; d <<= 1) most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
#pragma unroll
      for (int d = 1; d < (S::kShared ? 16 : kGroup / kEach); d <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
      const int up = most == 0 ? 0 : min(7 - ((int)(most >> 7) - 127), 100);       // -120 at least
      const float scale = __int_as_float((127 + up) << 23);
      if (most >= 0x7F80u) sum = __int_as_float(0x7FC00000);             // a NaN or an infinity: so are all scores
      if (S::kShared ? part == 0 : part % (kGroup / kEach) == 0)
        ctl->q_sum[S::kShared ? 0 : part * kEach / kGroup][slot] = sum * __int_as_float((127 + up + 9) << 23);
      if (part == 0 && (!S::kShared || group == 0)) {
        ctl->back[r] = __int_as_float((127 - up) << 23);                 // undoes the scale
        ctl->minus[r] = 0.0f;
        ctl->top[r] = ctl->peak[r] = -INFINITY;
        ctl->limit[r] = r < sg.rows ? -INFINITY : INFINITY;
        ctl->weight[r] = ctl->grain[r] = 0.0f;
        const int pos = base_pos + new_token;
        ctl->high[r] = r < sg.rows ? pos + 1 : 0;
        ctl->low[r] = a.window > 0 ? pos + 1 - a.window : 0;
      }
      // two rows of the operand: the leading e4m3 numbers, and 16 times what they leave
      const int lead = rb * 16 + tid / 16, rest = lead + 8;
#pragma unroll
      for (int j = 0; j < kEach / 2; j += 2) {                           // four elements: two even, two odd
        const float x0 = param_step(e[j]) * scale, x1 = param_low(e[j]) * scale, x2 = param_step(e[j + 1]) * scale, x3 = param_low(e[j + 1]) * scale;
        const uint32_t even = to_e4m3x2(x0, x2), odd = to_e4m3x2(x1, x3);
        const float2 fe = from_e4m3x2(even), fo = from_e4m3x2(odd);
        const uint32_t even2 = to_e4m3x2((x0 - fe.x) * 16.0f, (x2 - fe.y) * 16.0f), odd2 = to_e4m3x2((x1 - fo.x) * 16.0f, (x3 - fo.y) * 16.0f);
        const int d = part * kEach + 2 * j, in = d % 32;                 // of the head, of its chunk
        const uint32_t at = queries + (d / 128) * (NB * 2048);
        const int piece = (d % 128) / 32 * 2;
        auto put = [&](int n, int half, uint32_t two) {
          const uint32_t to = at + n * 128 + (((piece + half) ^ (n & 7)) << 4) + in / 2;
          asm volatile("st.shared.u16 [%0], %1;" ::"r"(to), "h"((uint16_t)two) : "memory");
        };
        put(lead, 0, even);
        put(lead, 1, odd);
        put(rest, 0, even2);
        put(rest, 1, odd2);
      }
    }
    // every row of the tile sees the keys [all_low, all_high)
    const int all_high = base_pos + token_of_row(a, sg.first_row) + 1;
    const int all_low = a.window > 0 ? base_pos + token_of_row(a, sg.first_row + sg.rows - 1) + 1 - a.window : 0;

    float total[kRows] = {}, low_sum[G][kRows] = {};                     // of this thread's tokens
    float out[S::kBlocks][kRows] = {};                                   // of this thread's element of the head: sums of p s q
    int since = 0;                                                       // tiles in the integer sums

    // Adds the integer sums to the registers, in the rows' present units.  A warp's 32 lanes are the elements 32 warp .. of a
    // block: one group.
    auto empty_sums = [&] {
#pragma unroll
      for (int k = 0; k < S::kBlocks; ++k)
#pragma unroll
        for (int rb = 0; rb < NB; ++rb) {
          const int group = (warp * 32 * S::kBlockGroups / (D < 128 ? 64 : 128)) % S::kBlockGroups;
          const int part = S::kShared ? 0 : group * NB + rb;
          const uint32_t at = sum_tmem + own_lanes + k * S::kWeightCols;
          uint32_t low16[16], high8[8];
          ptx::tmem_ld_32x16(at + part * 16, low16);
          ptx::tmem_ld_32x8(at + 16 * S::kParts + part * 8, high8);
          ptx::tmem_ld_wait();
#pragma unroll
          for (int slot = 0; slot < 8; ++slot) {
            const float sum = fmaf((float)(int)high8[slot], 65536.0f, fmaf((float)(int)low16[8 + slot], 256.0f, (float)(int)low16[slot]));
            if (S::kShared) {
              if (slot < S::kSlots && slot / kRows == group) out[k][slot % kRows] = fmaf(sum, ctl->grain[slot % kRows], out[k][slot % kRows]);
            } else if (rb * 8 + slot < kRows) {
              out[k][rb * 8 + slot] = fmaf(sum, ctl->grain[rb * 8 + slot], out[k][rb * 8 + slot]);
            }
          }
        }
      since = 0;
    };

    Places place{};
    for (int i = 0; i < tiles; ++i) {
      const int t0 = job.first_token + i * S::kUnit, token = t0 + tid, left = left_of(job, i + 1);
      const bool edge = t0 < all_low || t0 + S::kUnit > all_high;
      uint32_t key_params[G], value_params[G];
#pragma unroll
      for (int e = 0; e < G; ++e) {
        key_params[e] = next_key_params[e];
        value_params[e] = next_value_params[e];
      }
      spread(key_codes, 0);
      if (i + 1 < tiles) {
        place = find(job, i + 1);
        fetch(key_codes, key_lane, place, left);
        fetch_params(next_key_params, key_param_lane, place, left);
        fetch_params(next_value_params, value_param_lane, place, left);
      }
      ptx::fence_proxy_async_smem();
      ptx::tc_fence_before();
      __syncthreads();
      if (warp == 0) {
        ptx::tc_fence_after();
        if (ptx::elect_one()) {
#pragma unroll
          for (int d = 0; d < D; d += 32) {                              // a group's scores have columns of their own
            const int block = d / 128, at = d % 128;
            mma_e4m3(score_tmem(S::kShared ? 0 : d / kGroup), keys_desc + ((block * 16384 + at) >> 4),
                     queries_desc + ((block * (NB * 2048) + at) >> 4), kScoreDesc | ((uint32_t)(2 * NB) << 17), (S::kShared ? d : d % kGroup) != 0);
          }
          ptx::mma_commit(ptx::smem_addr(&ctl->scores_done));
        }
        __syncwarp();
      }
      // Under the product: the values of this tile.
      if (i > 0) {                                                       // the last tile's values and weights have been read
        bounded_wait_warp(ptx::smem_addr(&ctl->sums_done), sums_phase, abort_flag, WAIT_EPI_ACC_FULL);
        sums_phase ^= 1u;
        if (since == 4096) {                                             // 15 * 255 * 128 * 4096 < 2^31
          ptx::tc_fence_after();
          empty_sums();
        }
      }
      spread(value_codes, S::kOperandBytes);
      if (i + 1 < tiles) fetch(value_codes, value_lane, place, left);
      bounded_wait_warp(ptx::smem_addr(&ctl->scores_done), scores_phase, abort_flag, WAIT_EPI_ACC_FULL);
      scores_phase ^= 1u;
      ptx::tc_fence_after();

      // ---- this token's scores
      float arg[kRows];
      float step = 0.0f;
      bool raise = i == 0;
      if constexpr (S::kShared) {
        uint32_t acc[16];
        ptx::tmem_ld_32x16(score_tmem(0) + own_lanes, acc);
        ptx::tmem_ld_wait();
        const float4 q0 = *reinterpret_cast<const float4*>(&ctl->q_sum[0][0]), q1 = *reinterpret_cast<const float4*>(&ctl->q_sum[0][4]);
        const float qv[8] = {q0.x, q0.y, q0.z, q0.w, q1.x, q1.y, q1.z, q1.w};
#pragma unroll
        for (int e = 0; e < G; ++e) {
          const float ks = param_step(key_params[e]) * (a.scale_log2 * 512.0f), km = param_low(key_params[e]) * a.scale_log2;
          step = fmaxf(step, param_step(value_params[e]));
#pragma unroll
          for (int r = 0; r < kRows; ++r) {
            const int slot = e * kRows + r;
            const float z = fmaf(__uint_as_float(acc[8 + slot]), 0.0625f, __uint_as_float(acc[slot]));
            arg[r] = fmaf(z, ks, e == 0 ? qv[slot] * km : fmaf(qv[slot], km, arg[r]));
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < G; ++e) {
          const float ks = param_step(key_params[e]) * (a.scale_log2 * 512.0f), km = param_low(key_params[e]) * a.scale_log2;
          step = fmaxf(step, param_step(value_params[e]));
#pragma unroll
          for (int rb = 0; rb < NB; ++rb) {
            uint32_t acc[16];
            ptx::tmem_ld_32x16(score_tmem(e) + own_lanes + rb * 16, acc);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int q4 = 0; q4 < 8 && q4 < kRows; q4 += 4) {
              const float4 qs = *reinterpret_cast<const float4*>(&ctl->q_sum[e][rb * 8 + q4]);
              const float qv[4] = {qs.x, qs.y, qs.z, qs.w};
#pragma unroll
              for (int r = 0; r < 4 && r < kRows; ++r) {
                const float z = fmaf(__uint_as_float(acc[8 + q4 + r]), 0.0625f, __uint_as_float(acc[q4 + r]));
                float& to = arg[rb * 8 + q4 + r];
                to = fmaf(z, ks, e == 0 ? qv[r] * km : fmaf(qv[r], km, to));
              }
            }
          }
        }
      }
      // Some rows of an edge tile do not see some of its tokens.
      auto weigh = [&](auto is_edge) {
        constexpr bool kEdge = decltype(is_edge)::value;
#pragma unroll
        for (int r0 = 0; r0 < kRows; r0 += 4) {
          const float4 bk = *reinterpret_cast<const float4*>(&ctl->back[r0]), mn = *reinterpret_cast<const float4*>(&ctl->minus[r0]);
          const float4 lm = *reinterpret_cast<const float4*>(&ctl->limit[r0]);
          const float bv[4] = {bk.x, bk.y, bk.z, bk.w}, mv[4] = {mn.x, mn.y, mn.z, mn.w}, lv[4] = {lm.x, lm.y, lm.z, lm.w};
#pragma unroll
          for (int r = 0; r < 4 && r < kRows; ++r) {
            arg[r0 + r] = fmaf(arg[r0 + r], bv[r], mv[r]);
            if (kEdge) {
              const bool seen = token >= ctl->low[r0 + r] && token < ctl->high[r0 + r];
              arg[r0 + r] = seen ? arg[r0 + r] : -INFINITY;
            }
            raise |= arg[r0 + r] > lv[r];
          }
        }
        // The weights are written before it is known whether some thread wants its row's exponent raised, which is rare
        // behind a segment's first tile.
        float p[kRows], w[kRows];
        float most = __fdividef(kWeightLimit, step);                     // of p 2^E: no w passes 2^23
        const float add = __uint_as_float(0x3F800000u | ((uint32_t)token * 0x9E3779B1u >> 9)) - 1.0f;
        for (bool unset = i == 0;; unset = false) {
#pragma unroll
          for (int r = 0; r < kRows; ++r) p[r] = exp2_approx(arg[r]);
          if (!unset) {
#pragma unroll
            for (int r0 = 0; r0 < kRows; r0 += 4) {
              const float4 we = *reinterpret_cast<const float4*>(&ctl->weight[r0]);
              const float wv[4] = {we.x, we.y, we.z, we.w};
#pragma unroll
              for (int r = 0; r < 4 && r < kRows; ++r) {
                w[r0 + r] = p[r0 + r] * wv[r];
                raise |= w[r0 + r] > most;
              }
            }
            // a weight as an integer: the low 23 bits of w + 2^23; unseen, zero, whatever the step
            auto bits_of = [&](int e, int r) {
              const uint32_t y = __float_as_uint(__fadd_rz(__fmaf_rz(w[r], param_step(value_params[e]), add), 8388608.0f));
              return kEdge && arg[r] == -INFINITY ? 0u : y;
            };
            // eight slots, their low and middle bytes in one 16-byte unit of the token, the high ones in half of another
            auto put = [&](const uint32_t (&y)[8], int slots, int block, int part) {
              const uint32_t at = weight_at + block * (S::kWeightUnits * 2048) + part * 2048;
              const uint32_t high_at = weight_at + block * (S::kWeightUnits * 2048) + (S::kParts == 1 ? 2048 : (S::kParts + part / 2) * 2048 + (part & 1) * 8);
              if (slots == 1) {
                sts_8(at, y[0]);
                sts_8(at + 8, y[0] >> 8);
                sts_8(high_at, y[0] >> 16);
                return;
              }
              uint32_t low[2], mid[2], high[2];
#pragma unroll
              for (int h = 0; h < 2; ++h) {
                const uint32_t t01 = __byte_perm(y[4 * h], y[4 * h + 1], 0x5140), t23 = __byte_perm(y[4 * h + 2], y[4 * h + 3], 0x5140);
                low[h] = __byte_perm(t01, t23, 0x5410);
                mid[h] = __byte_perm(t01, t23, 0x7632);
                high[h] = __byte_perm(__byte_perm(y[4 * h], y[4 * h + 1], 0x0062), __byte_perm(y[4 * h + 2], y[4 * h + 3], 0x0062), 0x5410);
              }
              if (slots <= 4) {
                sts_32(at, low[0]);
                sts_32(at + 8, mid[0]);
                sts_32(high_at, high[0]);
              } else {
                ptx::sts_128(at, low[0], low[1], mid[0], mid[1]);
                sts_64(high_at, high[0], high[1]);
              }
            };
            if constexpr (S::kShared) {
#pragma unroll
              for (int block = 0; block < S::kBlocks; ++block) {
                uint32_t y[8] = {};
#pragma unroll
                for (int slot = 0; slot < S::kSlots; ++slot) y[slot] = bits_of(block * S::kBlockGroups + slot / kRows, slot % kRows);
                put(y, S::kSlots, block, 0);
              }
            } else {
#pragma unroll
              for (int e = 0; e < G; ++e)
#pragma unroll
                for (int rb = 0; rb < NB; ++rb) {
                  uint32_t y[8] = {};
#pragma unroll
                  for (int r = 0; r < 8 && r < kRows; ++r) y[r] = bits_of(e, rb * 8 + r);
                  put(y, kRows < 8 ? kRows : 8, e / S::kBlockGroups, e % S::kBlockGroups * NB + rb);
                }
            }
          }
          ptx::fence_proxy_async_smem();
          ptx::tc_fence_before();
          if (!__syncthreads_or(raise)) break;
          raise = false;
          most = INFINITY;                                               // once a tile
          // the largest score and the largest p s that each row sees in the tile
          const float step_log2 = log2f(step);
#pragma unroll
          for (int r = 0; r < kRows; ++r) {
            const float m = warp_max(arg[r]), u = warp_max(arg[r] + step_log2);
            if (lane == 0) {
              ctl->warp_top[warp][r] = m;
              ctl->warp_peak[warp][r] = u;
            }
          }
          if (since > 0) {
            ptx::tc_fence_after();
            empty_sums();
          }
          __syncthreads();
          if (warp == 0 && lane < sg.rows) {
            const int r = lane;
            const float m = fmaxf(fmaxf(ctl->warp_top[0][r], ctl->warp_top[1][r]), fmaxf(ctl->warp_top[2][r], ctl->warp_top[3][r]));
            const float u = fmaxf(fmaxf(ctl->warp_peak[0][r], ctl->warp_peak[1][r]), fmaxf(ctl->warp_peak[2][r], ctl->warp_peak[3][r]));
            float factor = 1.0f, delta = 0.0f;
            if (m > -INFINITY) {
              const float was = ctl->top[r], minus = ctl->minus[r];
              const float top = fmaxf(was, m - minus), peak = fmaxf(ctl->peak[r], u - minus);
              // (no steps so far: whatever comes makes a raise)
              const int e = peak > -INFINITY ? min(max((int)(kTop - floorf(peak - top)), kLeastExponent), kMostExponent) : kMostExponent;
              factor = was == -INFINITY ? 0.0f : exp2_approx(was - top);
              delta = -top - minus;
              ctl->top[r] = top;
              ctl->peak[r] = peak;
              ctl->minus[r] = -top;
              ctl->limit[r] = kLazy;
              ctl->weight[r] = __int_as_float((127 + e) << 23);
              ctl->grain[r] = __int_as_float((127 - e) << 23);
            }
            ctl->factor[r] = factor;
            ctl->delta[r] = delta;
          }
          __syncthreads();
#pragma unroll
          for (int r = 0; r < kRows; ++r) {
            const bool own = r < sg.rows;
            const float f = own ? ctl->factor[r] : 1.0f;
            arg[r] += own ? ctl->delta[r] : 0.0f;
            total[r] *= f;
#pragma unroll
            for (int e = 0; e < G; ++e) low_sum[e][r] *= f;
#pragma unroll
            for (int k = 0; k < S::kBlocks; ++k) out[k][r] *= f;
          }
        }
        if (warp == 0) {
          ptx::tc_fence_after();
          if (ptx::elect_one()) {
#pragma unroll
            for (int k = 0; k < S::kBlocks; ++k)
#pragma unroll
              for (int t = 0; t < 4; ++t)                                  // 32 tokens each
                mma_u8(sum_tmem + k * S::kWeightCols, values_desc + ((k * 16384 + t * 4096) >> 4),
                       weights_desc + ((k * (S::kWeightUnits * 2048) + t * 512) >> 4), kSumDesc | ((uint32_t)(S::kWeightCols / 8) << 17),
                       since > 0 || t > 0);
            ptx::mma_commit(ptx::smem_addr(&ctl->sums_done));
          }
          __syncwarp();
        }
        ++since;
        // a step that is not finite makes its group NaN
#pragma unroll
        for (int r = 0; r < kRows; ++r) total[r] += p[r];
#pragma unroll
        for (int e = 0; e < G; ++e) {
          const float m = fmaf(0.0f, param_step(value_params[e]), param_low(value_params[e]));
#pragma unroll
          for (int r = 0; r < kRows; ++r) {
            if (kEdge) low_sum[e][r] += arg[r] == -INFINITY ? 0.0f : p[r] * m;
            else low_sum[e][r] = fmaf(p[r], m, low_sum[e][r]);
          }
        }
      };
      if (edge) weigh(std::true_type());
      else weigh(std::false_type());
    }
    if (tiles > 0) {
      bounded_wait_warp(ptx::smem_addr(&ctl->sums_done), sums_phase, abort_flag, WAIT_EPI_ACC_FULL);
      sums_phase ^= 1u;
      ptx::tc_fence_after();
      empty_sums();
    }

    // the next segment is on its way while this one is finished
    const Job done = job;
    more = x < x_end;
    if (more) {
      job = next_job();
      page = page_of(job, 0);
    }

    // ---- sums over the tokens: every thread's values side by side, then a warp per row of them
#pragma unroll
    for (int r = 0; r < kRows; ++r) {
      meet[r * 128 + tid] = total[r];
#pragma unroll
      for (int e = 0; e < G; ++e) meet[((1 + e) * kRows + r) * 128 + tid] = low_sum[e][r];
    }
    __syncthreads();
    for (int n = warp; n < (1 + G) * kRows; n += kWarps) {
      const float4 y = *reinterpret_cast<const float4*>(meet + n * 128 + lane * 4);
      float sum = (y.x + y.y) + (y.z + y.w);
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, d);
      if (lane == 0) ctl->sums[n / kRows][n % kRows] = sum;
    }
    if (more) fetch_first(job);
    __syncthreads();
    // elements to their places: byte tid of a row is element 32 (tid / 32) + 2 (tid % 16) + (tid / 16 % 2)
#pragma unroll
    for (int k = 0; k < S::kBlocks; ++k) {
      const int d = k * 128 + (tid & ~31) + 2 * (tid & 15) + ((tid >> 4) & 1);
      if (d < D) {
#pragma unroll
        for (int r = 0; r < kRows; ++r) meet[r * D + d] = out[k][r] + ctl->sums[1 + d / kGroup][r];
      }
    }
    __syncthreads();
    // a piece that starts inside the segment goes to the worker's first slot, one that ends inside it to the second
    const int64_t part_slot = 2 * (int64_t)blockIdx.x + (done.u0 == 0 ? 1 : 0);
    for (int r = warp; r < done.sg.rows; r += kWarps) {
      const float m = ctl->top[r], l = ctl->sums[0][r];
      const int row = done.sg.first_row + r, new_token = token_of_row(a, row);
      const int64_t out_row = done.rows.first + new_token;
      const int q_head = done.head * a.ratio + row - new_token * a.ratio;
      const bool empty = m == -INFINITY && l == 0.0f;                    // (a row whose scores are all NaN is not)
      const float inv = empty ? 0.0f : 1.0f / l;
      eqat_bf16* to = a.O + out_row * a.o_pitch + (int64_t)q_head * D;
      float* part = done.whole ? nullptr : a.partial + (part_slot * kRows + r) * (D + 4);
#pragma unroll
      for (int p = lane; p < D / 4; p += 32) {
        const float4 e = *reinterpret_cast<const float4*>(meet + r * D + p * 4);
        if (done.whole) *reinterpret_cast<uint2*>(to + p * 4) = make_uint2(pack_bf16x2(e.x * inv, e.y * inv), pack_bf16x2(e.z * inv, e.w * inv));
        else *reinterpret_cast<float4*>(part + p * 4) = e;
      }
      if (lane == 0) {
        if (!done.whole) *reinterpret_cast<float2*>(part + D) = make_float2(m, l);
        else if (a.lse != nullptr)
          a.lse[out_row * a.q_heads + q_head] = empty ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
      }
    }
    __syncthreads();                                                     // the operands may be written again
  }
  ptx::grid_dependents_launch();
  ptx::tc_fence_before();
  __syncthreads();
  if (warp == 0) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(ctl->tmem[0], S::kAlloc);
    if (S::kTwoParts) ptx::tmem_dealloc(ctl->tmem[1], 32);
  }
}

// Joins the segments that workers share: a CTA per worker that starts a segment and does not finish it.  A row's pieces are
// dealt out to 1 to 16 warps, each adds up its own in the order of the workers, and then theirs are added up.
template <int D, int G, int ROWS>
__global__ void __launch_bounds__(kJoinThreads) attention_join_kernel(const AttentionArgs a) {
  using S = Shape<D, G, ROWS>;
  constexpr int kFours = D / 128 > 0 ? D / 128 : 1;                      // float4 of a lane
  constexpr int kJoinWarps = kJoinThreads / 32, kSplit = kJoinWarps / (ROWS < kJoinWarps ? ROWS : kJoinWarps);       // warps of a row
  __shared__ __align__(16) float sums[kJoinWarps][D], weights[kJoinWarps];
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, first = blockIdx.x, split = warp % kSplit;
  const JoinRecord rec = a.records[first];
  if (rec.workers <= 1) return;
  for (int r0 = 0; r0 < rec.rows; r0 += kJoinWarps / kSplit) {
    const int r = r0 + warp / kSplit;
    auto part = [&](int k) {                                             // only the first worker's piece starts the segment
      return a.partial + ((2 * (int64_t)(first + k) + (k == 0 ? 1 : 0)) * S::kRows + r) * (D + 4);
    };
    float m = -INFINITY, l = 0.0f;
    float4 e[kFours] = {};
    if (r < rec.rows) {
      for (int k = lane; k < rec.workers; k += 32) m = fmaxf(m, ptx::ld_global(static_cast<const float*>(part(k) + D)));
      m = warp_max(m);
      const int each = (rec.workers + kSplit - 1) / kSplit, from = split * each, upto = min(from + each, rec.workers);
      for (int k0 = from; k0 < upto; k0 += 32) {
        float f = 0.0f;
        if (k0 + lane < upto) {
          const uint2 y = ptx::ld_global(reinterpret_cast<const uint2*>(part(k0 + lane) + D));
          f = m == -INFINITY ? 1.0f : exp2_approx(__uint_as_float(y.x) - m);
          l = fmaf(f, __uint_as_float(y.y), l);
        }
        const int n = min(32, upto - k0);
        for (int k = 0; k < n; k += 8) {
          uint4 y[8][kFours];
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int i = 0; i < kFours; ++i)
              y[j][i] = k + j < n && lane + 32 * i < D / 4 ? ptx::ld_global(reinterpret_cast<const uint4*>(part(k0 + k + j)) + lane + 32 * i) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float fj = __shfl_sync(0xFFFFFFFFu, f, k + j);
#pragma unroll
            for (int i = 0; i < kFours; ++i) {
              e[i].x = fmaf(fj, __uint_as_float(y[j][i].x), e[i].x);
              e[i].y = fmaf(fj, __uint_as_float(y[j][i].y), e[i].y);
              e[i].z = fmaf(fj, __uint_as_float(y[j][i].z), e[i].z);
              e[i].w = fmaf(fj, __uint_as_float(y[j][i].w), e[i].w);
            }
          }
        }
      }
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) l += __shfl_xor_sync(0xFFFFFFFFu, l, d);
    }
    if (kSplit > 1) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kFours; ++i)
        if (lane + 32 * i < D / 4) *reinterpret_cast<float4*>(&sums[warp][(lane + 32 * i) * 4]) = e[i];
      if (lane == 0) weights[warp] = l;
      __syncthreads();
      if (split == 0) {
        for (int k = 1; k < kSplit; ++k) {
          l += weights[warp + k];
#pragma unroll
          for (int i = 0; i < kFours; ++i)
            if (lane + 32 * i < D / 4) {
              const float4 y = *reinterpret_cast<const float4*>(&sums[warp + k][(lane + 32 * i) * 4]);
              e[i].x += y.x; e[i].y += y.y; e[i].z += y.z; e[i].w += y.w;
            }
        }
      }
    }
    if (split != 0 || r >= rec.rows) continue;
    const int row = rec.first_row + r, new_token = token_of_row(a, row);
    const int64_t out_row = rec.first + new_token;
    const int q_head = rec.head * a.ratio + row - new_token * a.ratio;
    const bool empty = m == -INFINITY && l == 0.0f;
    const float inv = empty ? 0.0f : 1.0f / l;
#pragma unroll
    for (int i = 0; i < kFours; ++i)
      if (lane + 32 * i < D / 4)
        *reinterpret_cast<uint2*>(a.O + out_row * a.o_pitch + (int64_t)q_head * D + (lane + 32 * i) * 4) =
            make_uint2(pack_bf16x2(e[i].x * inv, e[i].y * inv), pack_bf16x2(e[i].z * inv, e[i].w * inv));
    if (lane == 0 && a.lse != nullptr)
      a.lse[out_row * a.q_heads + q_head] = empty ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
  }
}

// ------------------------------------------------------------------ host side
// How a call is divided between the two kernels.
struct Division {
  bool prompts;                // the kernel for prompts takes part
  int least_rows;              // of the sequences that are its own
};
Division divide(const eqat_cache_desc& d, const eqat_attention_desc& a, int sms) {
  const bool prompts = prompt_attention_applies(d, a, sms);
  return {prompts, prompts ? prompt_least_rows(d, a, sms) : 0};
}

// Query rows that a tile of the cache is read for: as many as an ordinary sequence here has, as far as accumulators and a
// thread's sums have room (32 rows x groups).  Ordinary is the average, without those that are the other kernel's in a call
// that is divided: decoding beside a prompt has the rows of one token.  (255 tokens behind 2048 beside a prompt of 512, 64/8
// heads: tiles of 32 rows 366 us, of 8 194; 99 tokens behind 4096 beside four drafted ones: of 32 261 us, of 16 165.)
int tile_rows(const eqat_cache_desc& d, const eqat_attention_desc& a, const Division& div) {
  const int64_t ratio = a.q_heads / d.kv_heads, have = d.sequences < d.rows ? d.sequences : d.rows;
  int64_t each = (d.rows + have - 1) / have;
  if (div.prompts && div.least_rows > 1) each = unequal_batch(d, a).each;
  int64_t rows = (each < a.max_new ? each : a.max_new) * ratio;
  if (div.prompts && rows > kPromptRows - 1) rows = kPromptRows - 1;
  const int groups = d.head_dim / d.group, most = groups >= 4 || d.head_dim == 256 ? 8 : groups == 2 ? 16 : 32;
  if (rows == 1) return 1;
  int n = 4;
  while (n < most && n < rows) n *= 2;
  return n;
}

template <typename F>
int with_shape(const eqat_cache_desc& d, int rows, F&& f) {
  const int g = d.head_dim / d.group;
#define EQAT_SHAPE(DD, GG, RR)                            \
  if (d.head_dim == DD && g == GG && rows == RR)          \
    return f(std::integral_constant<int, DD>(), std::integral_constant<int, GG>(), std::integral_constant<int, RR>());
#define EQAT_SHAPES(DD, GG) EQAT_SHAPE(DD, GG, 1) EQAT_SHAPE(DD, GG, 4) EQAT_SHAPE(DD, GG, 8)
  EQAT_SHAPES(64, 1)
  EQAT_SHAPE(64, 1, 16)
  EQAT_SHAPE(64, 1, 32)
  EQAT_SHAPES(64, 2)
  EQAT_SHAPE(64, 2, 16)
  EQAT_SHAPES(128, 1)
  EQAT_SHAPE(128, 1, 16)
  EQAT_SHAPE(128, 1, 32)
  EQAT_SHAPES(128, 2)
  EQAT_SHAPE(128, 2, 16)
  EQAT_SHAPES(128, 4)
  EQAT_SHAPES(256, 2)
  EQAT_SHAPES(256, 4)
  EQAT_SHAPES(256, 8)
#undef EQAT_SHAPES
#undef EQAT_SHAPE
  return EQAT_ERR_UNSUPPORTED;
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
  const int64_t want = most_units<S>(d, a);
  const int64_t most = (int64_t)sms * S::kCtas;
  return (int)(want < 1 ? 1 : want < most ? want : most);
}

}  // namespace

AttentionArgs attention_args(const eqat_cache_desc& d, const eqat_attention_desc& at, const eqat_bf16* Q, int64_t q_pitch,
                             const CacheView& view, eqat_bf16* O, int64_t o_pitch, float* lse) {
  auto log2_up = [](int v) {
    int s = 0;
    while ((1 << s) < v) ++s;
    return s;
  };
  AttentionArgs a{};
  a.cache = view;
  a.Q = Q;
  a.q_pitch = q_pitch;
  a.O = O;
  a.o_pitch = o_pitch;
  a.lse = lse;
  a.q_heads = at.q_heads;
  a.ratio = at.q_heads / d.kv_heads;
  a.ratio_shift = (a.ratio & (a.ratio - 1)) == 0 ? log2_up(a.ratio) : -1;
  a.max_new = at.max_new;
  a.window = at.window < view.max_length ? at.window : 0;                // a window of the longest sequence hides nothing
  a.scale_log2 = at.scale * kLog2e;
  a.page_shift = 26 + log2_up(d.page_size / 16);
  a.page_mul = (uint32_t)((((uint64_t)1 << a.page_shift) + d.page_size / 16 - 1) / (d.page_size / 16));
  return a;
}

void cache_attention_plan(const eqat_cache_desc& d, const eqat_attention_desc& a, int sms, int* plan) {
  const Division div = divide(d, a, sms);
  plan[0] = tile_rows(d, a, div);
  plan[1] = div.least_rows;
}

size_t cache_attention_workspace(const eqat_cache_desc& d, const eqat_attention_desc& a) {
  const int sms = sm_count() > 0 ? sm_count() : 148;
  size_t bytes = (size_t)-1;
  with_shape(d, tile_rows(d, a, divide(d, a, sms)), [&](auto D, auto G, auto NT) {
    using S = Shape<decltype(D)::value, decltype(G)::value, decltype(NT)::value>;
    const int w = workers_of<S>(d, a, sms);
    bytes = w > 1 ? (size_t)w * (sizeof(JoinRecord) + (size_t)2 * S::kRows * (decltype(D)::value + 4) * sizeof(float)) : 0;
    return EQAT_OK;
  });
  return bytes;
}

int launch_cache_attention(const eqat_cache_desc& d, const eqat_attention_desc& at, const eqat_bf16* Q, int64_t q_pitch,
                           const CacheView& view, eqat_bf16* O, int64_t o_pitch, float* lse, void* workspace, cudaStream_t st) {
  const int sms = sm_count();
  if (sms <= 0) return EQAT_ERR_CUDA;
  AttentionArgs args = attention_args(d, at, Q, q_pitch, view, O, o_pitch, lse);
  args.most_rows = INT32_MAX;
  const Division div = divide(d, at, sms);
  if (div.prompts) {                                                     // long sequences there, short ones here
    args.least_rows = div.least_rows;
    const int rc = launch_prompt_attention(d, args, st);
    if (rc != EQAT_OK || args.least_rows == 1) return rc;
    args.most_rows = args.least_rows - 1;
    args.least_rows = 0;
  }
  return with_shape(d, tile_rows(d, at, div), [&](auto DD, auto GG, auto NN) {
    constexpr int D = decltype(DD)::value, G = decltype(GG)::value, NT = decltype(NN)::value;
    using S = Shape<D, G, NT>;
    AttentionArgs a = args;
    static SmemOptIn opt;
    if (!opt.ensure(attention_kernel<D, G, NT>, S::kSmemBytes)) return (int)EQAT_ERR_CUDA;
    const int workers = workers_of<S>(d, at, sms);
    if (workers > 1) {
      a.records = static_cast<JoinRecord*>(workspace);
      a.partial = reinterpret_cast<float*>(a.records + workers);
    }
    const int rc = launch_overlapped(attention_kernel<D, G, NT>, dim3(workers), dim3(kThreads), S::kSmemBytes, st, a);
    if (rc != EQAT_OK || workers == 1) return rc;
    return launch_overlapped(attention_join_kernel<D, G, NT>, dim3(workers - 1), dim3(kJoinThreads), 0, st, a);
  });
}

int launch_wait_expiry_attention(cudaStream_t st) { return launch_wait_expiry(st); }
int read_attention_status(int* status, int* detail) { return read_wait_status(status, detail); }

}  // namespace eqat
