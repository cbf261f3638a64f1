// Attention over the 4-bit cache: what its kernels share.
#pragma once
#include "cache.cuh"
#include "common.cuh"
#include "ptx.cuh"

namespace eqat {

constexpr float kLog2e = 1.4426950408889634f;

// What a worker leaves behind for the join: its last segment, if it starts there and other workers go on with it.
struct __align__(16) JoinRecord {
  int first, first_row, rows, head;    // first row of the sequence, and the tile's rows as in Segment
  int workers, unused[3];              // pieces; at most one: nothing to join
};

struct AttentionArgs {
  CacheView cache;
  const eqat_bf16* Q;
  int64_t q_pitch, o_pitch;
  eqat_bf16* O;
  float* lse;
  JoinRecord* records;         // [workers]
  float* partial;              // [2 * workers][rows of a tile][D + 4]: sums, then the exponent and the sum of weights
  int q_heads, ratio, max_new, window;
  int ratio_shift;             // log2(ratio), or -1
  float scale_log2;            // scale * log2(e)
  uint32_t page_mul;           // n / (page_size / 16) = n * page_mul >> page_shift for n < 2^26
  int page_shift;
  int least_rows, most_rows;   // sequences with fewer or more rows (new tokens x ratio) are another kernel's
};

#ifdef __CUDACC__
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
  w.tiles = rows < a.least_rows || rows > a.most_rows ? 0 : (int)((rows + S::kRows - 1) / S::kRows);
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

// a / b for a >= 0: the 64-bit division, a subroutine of a hundred instructions, only where it is needed.
__device__ __forceinline__ int64_t quotient(int64_t a, int b) { return (a >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b; }
// New token of a row of a tile (rows run over the query heads of a token first).
__device__ __forceinline__ int token_of_row(const AttentionArgs& a, int row) { return a.ratio_shift >= 0 ? row >> a.ratio_shift : row / a.ratio; }

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
  s.high = max(base + token_of_row(a, s.first_row + s.rows - 1) + 1, 0);
  s.low = a.window > 0 ? max(base + token_of_row(a, s.first_row) + 1 - a.window, 0) : 0;
  s.from = s.low & ~(S::kStageTokens - 1);
  return s;
}

// ------------------------------------------------------------------ instructions
__device__ __forceinline__ float exp2_approx(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ float warp_max(float x) {
  float r;
  asm("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;" : "=f"(r) : "f"(x));
  return r;
}
// A CTA's tensor memory (whole warp).
__device__ __forceinline__ void take_columns(uint32_t smem_dst, uint32_t cols) { ptx::tmem_alloc(smem_dst, cols); }
#endif

// The arguments of a call, without workspace and row limits.
AttentionArgs attention_args(const eqat_cache_desc& d, const eqat_attention_desc& at, const eqat_bf16* Q, int64_t q_pitch,
                             const CacheView& view, eqat_bf16* O, int64_t o_pitch, float* lse);

// Sequences with at least this many rows (new tokens x query heads of a key/value head) are the prompt kernel's, in calls
// that it takes part in; all of them are where that is estimated to be no worse, which saves the launches for few rows.
constexpr int kPromptRows = 33;

// A call as unequal as its descriptors allow if every sequence has a row: as many as possible with max_new new tokens, or with
// all that the others leave, and these with what is left of the rows.
struct UnequalBatch {
  int64_t longest, with;       // the most new tokens, sequences that have them
  int64_t rest, each;          // other sequences, the tokens of one of these, rounded up
};
inline UnequalBatch unequal_batch(const eqat_cache_desc& d, const eqat_attention_desc& a) {
  const int64_t have = d.sequences < d.rows ? d.sequences : d.rows;
  const int64_t most = have * a.max_new, rows = d.rows < most ? d.rows : most;
  UnequalBatch u{};
  u.longest = a.max_new < rows - have + 1 ? a.max_new : rows - have + 1;
  u.with = u.longest > 1 ? (rows - have) / (u.longest - 1) : have;
  u.rest = have - u.with;
  u.each = u.rest > 0 ? (rows - u.with * u.longest + u.rest - 1) / u.rest : 0;
  return u;
}
int prompt_least_rows(const eqat_cache_desc& d, const eqat_attention_desc& a, int sms);
bool prompt_attention_applies(const eqat_cache_desc& d, const eqat_attention_desc& a, int sms);
int launch_prompt_attention(const eqat_cache_desc& d, AttentionArgs a, cudaStream_t st);

int launch_wait_expiry_prompt(cudaStream_t st);
int read_prompt_status(int* status, int* detail);

}  // namespace eqat
