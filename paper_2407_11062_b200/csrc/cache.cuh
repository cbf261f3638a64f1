// The 4-bit key/value cache: what its kernels share, and their host launchers (arguments already validated).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "eqat.h"
#include "ptx.cuh"

namespace eqat {

// Device-side view of a cache and of the rows of a call.
struct CacheView {
  uint8_t* kq;                 // codes of the keys  [pages, kv_heads, page_size, head_dim / 2]
  uint32_t* kp;                // (step, minimum) of the keys, one word per group
  uint8_t* vq;
  uint32_t* vp;
  const int32_t* row_offsets;  // [sequences + 1]
  const int32_t* lengths;      // [sequences]
  const int32_t* page_table;   // [sequences, max_pages]
  int sequences, max_pages, page_size, pages, kv_heads;
  int rows;
  int max_length;              // max_pages * page_size
};

inline CacheView cache_view(const eqat_cache_desc& d, const int32_t* row_offsets, const int32_t* lengths,
                            const int32_t* page_table, const eqat_cache& c) {
  CacheView v{};
  v.kq = c.k_codes;
  v.kp = reinterpret_cast<uint32_t*>(c.k_params);
  v.vq = c.v_codes;
  v.vp = reinterpret_cast<uint32_t*>(c.v_params);
  v.row_offsets = row_offsets;
  v.lengths = lengths;
  v.page_table = page_table;
  v.sequences = d.sequences;
  v.max_pages = d.max_pages;
  v.page_size = d.page_size;
  v.pages = d.pages;
  v.kv_heads = d.kv_heads;
  v.rows = (int)d.rows;
  v.max_length = d.max_pages * d.page_size;
  return v;
}

#ifdef __CUDACC__
// The rows of sequence b: first, how many, and the tokens it holds with them.  Whatever the arrays say, the rows lie in
// [0, rows) and the length in [0, max_length].
struct SequenceRows {
  int first, count, length;
};
__device__ __forceinline__ int ld_index(const int32_t* p) { return (int)ptx::ld_global(reinterpret_cast<const uint32_t*>(p)); }
__device__ __forceinline__ SequenceRows sequence_rows(const CacheView& v, int b) {
  const int at0 = ld_index(v.row_offsets + b), at1 = ld_index(v.row_offsets + b + 1), held = ld_index(v.lengths + b);
  SequenceRows s;
  s.first = min(max(at0, 0), v.rows);
  s.count = max(min(at1, v.rows) - s.first, 0);
  s.length = min(max(held, 0), v.max_length);
  return s;
}

// (step, minimum) of a group as two floats.
__device__ __forceinline__ float param_step(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float param_low(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
#endif

int launch_cache_append(const eqat_cache_desc& d, const eqat_bf16* K, int64_t k_pitch, const eqat_bf16* V, int64_t v_pitch,
                        const CacheView& view, eqat_bf16* K_hat, eqat_bf16* V_hat, cudaStream_t st);
int launch_cache_read(const eqat_cache_desc& d, const CacheView& view, eqat_bf16* K_hat, eqat_bf16* V_hat, cudaStream_t st);

void cache_attention_plan(const eqat_cache_desc& d, const eqat_attention_desc& a, int sms, int* plan);
size_t cache_attention_workspace(const eqat_cache_desc& d, const eqat_attention_desc& a);
int launch_cache_attention(const eqat_cache_desc& d, const eqat_attention_desc& a, const eqat_bf16* Q, int64_t q_pitch,
                           const CacheView& view, eqat_bf16* O, int64_t o_pitch, float* lse, void* workspace, cudaStream_t st);

int launch_wait_expiry_attention(cudaStream_t st);
int read_attention_status(int* status, int* detail);

}  // namespace eqat
