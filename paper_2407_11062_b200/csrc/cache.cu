// The 4-bit key/value cache: quantising rows as they are written, and reading them back.
//
// Both are streams: 2 bytes in and 1/2 + 4/group out per element (append; 2 more where the values are handed back), the
// other way round for reading.  A lane owns eight consecutive elements, one 16-byte vector of a row tensor and one word of
// codes, so a group is 4, 8 or 16 neighbouring lanes: minimum and maximum travel as one bf16 pair (maximum, -minimum)
// through two to four shuffles.  A warp takes one row's keys or values in pieces of 1024 elements and looks its sequence up
// by a search of 32 offsets at a time while its vectors are on their way.
#include "cache.cuh"

#include <cuda_bf16.h>

#include "common.cuh"

namespace eqat {
namespace {

constexpr int kWarps = 8;
constexpr int kVectors = 4;                          // 16-byte vectors of a lane per item
constexpr float kStepMin = 1.17549435e-38f;          // 2^-126
constexpr float kMagic = 12582912.0f;                // 1.5 * 2^23: x + kMagic holds round(x) in its low bits

struct RowPlace {
  int64_t token;                                     // (page * kv_heads) * page_size + place in the page, of head 0
  bool stands;                                       // the row has a place in the cache
  bool owned;                                        // the row belongs to a sequence
};

// Whole warp: the place of a row.  The sequence is the number of offsets [1 ..] that are not beyond the row.
__device__ __forceinline__ RowPlace place_of(const CacheView& v, int row, int lane) {
  int low = 0, high = v.sequences;
  while (low < high) {
    const int step = (high - low + 31) >> 5;
    const int probe = low + (lane + 1) * step;
    const bool before = probe <= high && ld_index(v.row_offsets + probe) <= row;
    const int n = __popc(__ballot_sync(0xFFFFFFFFu, before));
    low += n * step;
    high = min(high, low + step - 1);
  }
  RowPlace p{0, false, low < v.sequences};
  if (p.owned) {
    const SequenceRows s = sequence_rows(v, low);
    const int pos = s.length - s.count + (row - s.first);
    if (pos >= 0 && pos < s.length) {
      const int page = ld_index(v.page_table + (int64_t)low * v.max_pages + pos / v.page_size);
      p.stands = page >= 0 && page < v.pages;
      p.token = (int64_t)page * v.kv_heads * v.page_size + pos % v.page_size;
    }
  }
  return p;
}

__device__ __forceinline__ __nv_bfloat162 as_pair(uint32_t x) { return *reinterpret_cast<__nv_bfloat162*>(&x); }
__device__ __forceinline__ uint32_t as_word(__nv_bfloat162 x) { return *reinterpret_cast<uint32_t*>(&x); }

struct Rows {
  const eqat_bf16 *K, *V;                            // append
  int64_t k_pitch, v_pitch;
  eqat_bf16 *K_hat, *V_hat;                          // append: may be NULL
};

// GL: lanes of a group (group / 8).
template <int GL, bool APPEND>
__global__ void __launch_bounds__(kWarps * 32) cache_rows_kernel(const CacheView v, const Rows rows, int head_shift, int pieces) {
  ptx::grid_dependency_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t items = (int64_t)v.rows * 2 * pieces, step = (int64_t)gridDim.x * kWarps;
  const int vectors = v.kv_heads << (head_shift - 3);                      // of a row
  const int head_groups = 1 << (head_shift - 3 - (GL == 4 ? 2 : GL == 8 ? 3 : 4));
  for (int64_t item = (int64_t)blockIdx.x * kWarps + warp; item < items; item += step) {
    if (item + step >= items) ptx::grid_dependents_launch();
    const int piece = (int)(item % pieces);
    const int which = (int)(item / pieces % 2);                            // keys or values
    const int row = (int)(item / pieces / 2);
    const int first = piece * (32 * kVectors) + lane;
    uint4 x[kVectors] = {};
    if (APPEND) {
      const uint4* from = reinterpret_cast<const uint4*>(which == 0 ? rows.K + row * rows.k_pitch : rows.V + row * rows.v_pitch);
#pragma unroll
      for (int u = 0; u < kVectors; ++u)
        if (first + 32 * u < vectors) x[u] = ptx::ld_global(from + first + 32 * u);
    }
    const RowPlace place = place_of(v, row, lane);
    uint8_t* codes = which == 0 ? v.kq : v.vq;
    uint32_t* params = which == 0 ? v.kp : v.vp;
    uint4* out = reinterpret_cast<uint4*>(which == 0 ? rows.K_hat : rows.V_hat);
    if (out != nullptr) out += (int64_t)row * vectors;
    auto slot = [&](int vec) { return place.token + (int64_t)(vec >> (head_shift - 3)) * v.page_size; };
    auto code_at = [&](int vec) {
      return reinterpret_cast<uint32_t*>(codes) + (slot(vec) << (head_shift - 3)) + (vec & ((1 << (head_shift - 3)) - 1));
    };
    auto param_at = [&](int vec) { return params + slot(vec) * head_groups + (vec & ((1 << (head_shift - 3)) - 1)) / GL; };

    if (APPEND) {
#pragma unroll
      for (int u = 0; u < kVectors; ++u) {
        const int vec = first + 32 * u;
        if (piece * (32 * kVectors) + 32 * u >= vectors) break;            // the whole warp
        const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
        // the NaN forms hand a NaN on
        const __nv_bfloat162 lo = __hmin2_nan(__hmin2_nan(as_pair(w[0]), as_pair(w[1])), __hmin2_nan(as_pair(w[2]), as_pair(w[3])));
        const __nv_bfloat162 hi = __hmax2_nan(__hmax2_nan(as_pair(w[0]), as_pair(w[1])), __hmax2_nan(as_pair(w[2]), as_pair(w[3])));
        __nv_bfloat162 range = __halves2bfloat162(__hmax_nan(__low2bfloat16(hi), __high2bfloat16(hi)),
                                                  __hneg(__hmin_nan(__low2bfloat16(lo), __high2bfloat16(lo))));
#pragma unroll
        for (int d = 1; d < GL; d <<= 1) range = __hmax2_nan(range, as_pair(__shfl_xor_sync(0xFFFFFFFFu, as_word(range), d)));
        const float most = __low2float(range), least = -__high2float(range);
        float s = __bfloat162float(__float2bfloat16_rn(__fmul_rn(__fsub_rn(most, least), 1.0f / 15.0f)));
        if (s < kStepMin) s = 0.0f;
        if (!(s < __int_as_float(0x7F800000))) s = __int_as_float(0x7FC00000);
        const float inverse = s > 0.0f ? __frcp_rn(s) : 0.0f;
        // With s rounded by at most 2^-8 of itself a quotient stays below 15.06: no code leaves 0 .. 15.
        uint32_t word = 0;
        uint32_t value[4];
#pragma unroll
        for (int i = 3; i >= 0; --i) {
          const float even = __fadd_rn(__fmul_rn(__fsub_rn(__uint_as_float(w[i] << 16), least), inverse), kMagic);
          const float odd = __fadd_rn(__fmul_rn(__fsub_rn(__uint_as_float(w[i] & 0xFFFF0000u), least), inverse), kMagic);
          word = (word << 8) | ((__float_as_uint(odd) & 15u) << 4) | (__float_as_uint(even) & 15u);
          value[i] = pack_bf16x2(fmaf(even - kMagic, s, least), fmaf(odd - kMagic, s, least));
        }
        if (vec < vectors && place.stands) {
          *code_at(vec) = word;
          if ((vec & (GL - 1)) == 0) *param_at(vec) = (__float_as_uint(s) >> 16) | (__float_as_uint(least) & 0xFFFF0000u);
          if (out != nullptr) out[vec] = make_uint4(value[0], value[1], value[2], value[3]);
        } else if (vec < vectors && place.owned && out != nullptr) {
          out[vec] = make_uint4(0u, 0u, 0u, 0u);
        }
      }
    } else if (place.owned) {
      uint32_t word[kVectors] = {}, param[kVectors] = {};
      if (place.stands) {
#pragma unroll
        for (int u = 0; u < kVectors; ++u)
          if (first + 32 * u < vectors) {
            word[u] = ptx::ld_global(static_cast<const uint32_t*>(code_at(first + 32 * u)));
            param[u] = ptx::ld_global(static_cast<const uint32_t*>(param_at(first + 32 * u)));
          }
      }
#pragma unroll
      for (int u = 0; u < kVectors; ++u) {
        const float s = param_step(param[u]), least = param_low(param[u]);
        uint32_t value[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
          value[i] = pack_bf16x2(fmaf((float)((word[u] >> (8 * i)) & 15u), s, least), fmaf((float)((word[u] >> (8 * i + 4)) & 15u), s, least));
        if (first + 32 * u < vectors) out[first + 32 * u] = make_uint4(value[0], value[1], value[2], value[3]);
      }
    }
  }
}

inline int log2_of(int v) {
  int s = 0;
  while ((1 << s) < v) ++s;
  return s;
}

template <bool APPEND>
int launch_rows(const eqat_cache_desc& d, const CacheView& view, const Rows& rows, cudaStream_t st) {
  const int vectors = d.kv_heads * d.head_dim / 8, pieces = (vectors + 32 * kVectors - 1) / (32 * kVectors);
  const int64_t blocks = (d.rows * 2 * pieces + kWarps - 1) / kWarps;
  const int sms = sm_count();
  if (sms <= 0) return EQAT_ERR_CUDA;
  const int64_t most = (int64_t)sms * 8;                                   // 64 warps an SM
  const dim3 grid((unsigned)(blocks < most ? blocks : most));
  const int shift = log2_of(d.head_dim);
  switch (d.group) {
    case 32: return launch_overlapped(cache_rows_kernel<4, APPEND>, grid, dim3(kWarps * 32), 0, st, view, rows, shift, pieces);
    case 64: return launch_overlapped(cache_rows_kernel<8, APPEND>, grid, dim3(kWarps * 32), 0, st, view, rows, shift, pieces);
    default: return launch_overlapped(cache_rows_kernel<16, APPEND>, grid, dim3(kWarps * 32), 0, st, view, rows, shift, pieces);
  }
}

}  // namespace

int launch_cache_append(const eqat_cache_desc& d, const eqat_bf16* K, int64_t k_pitch, const eqat_bf16* V, int64_t v_pitch,
                        const CacheView& view, eqat_bf16* K_hat, eqat_bf16* V_hat, cudaStream_t st) {
  return launch_rows<true>(d, view, Rows{K, V, k_pitch, v_pitch, K_hat, V_hat}, st);
}

int launch_cache_read(const eqat_cache_desc& d, const CacheView& view, eqat_bf16* K_hat, eqat_bf16* V_hat, cudaStream_t st) {
  return launch_rows<false>(d, view, Rows{nullptr, nullptr, 0, 0, K_hat, V_hat}, st);
}

}  // namespace eqat
