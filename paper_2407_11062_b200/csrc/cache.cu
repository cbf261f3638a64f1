// The 4-bit key/value cache: quantising rows as they are written, and reading them back.
//
// Both are streams: 2 bytes in and 1/2 + 4/group out per element (append; 2 more where the values are handed back), the
// other way round for reading.  A lane owns eight consecutive elements, one 16-byte vector of a row tensor and one word of
// codes, so a group is 4, 8 or 16 neighbouring lanes: minimum and maximum travel as one bf16 pair (maximum, -minimum)
// through two to four shuffles.  A warp takes one row's keys or values in pieces of 1024 elements and looks its sequence up
// by a search of 32 offsets at a time while its vectors are on their way.
//
// HBM bounds long calls: reading 16 x 4096 tokens of 32 heads, groups of 64, takes 159 us, 0.82 of a copy's bandwidth; appending
// prompts of 32 heads in groups of 32 with the values handed back 60 to 61.5 us, 0.83 to 0.85.  (One piece of a row at a time took 195 and 69.5 us.)
// A call of one token takes 3 us, a launch.
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

// bf16 128 + q with a code in the last mantissa bits of each half, to q s + m, rounded once.
__device__ __forceinline__ uint32_t value_pair(uint32_t codes, __nv_bfloat162 s, __nv_bfloat162 m) {
  return as_word(__hfma2(__hsub2(as_pair(codes | 0x43004300u), as_pair(0x43004300u)), s, m));
}

// Keys (even blockIdx.y) or values of the rows, blockIdx.y / 2 says which `per` pieces of a row.
template <int D, int GROUP, bool APPEND>
__global__ void __launch_bounds__(kWarps * 32) cache_rows_kernel(const CacheView v, const Rows rows, int per) {
  constexpr int kHead = D / 8, kLanes = GROUP / 8, kGroups = D / GROUP;    // vectors of a head, of a group
  ptx::grid_dependency_wait();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int vectors = v.kv_heads * kHead;                                  // of a row
  const bool keys = (blockIdx.y & 1) == 0;
  const int from = (int)(blockIdx.y >> 1) * per * (32 * kVectors), upto = min(from + per * (32 * kVectors), vectors);
  uint32_t* const codes = reinterpret_cast<uint32_t*>(keys ? v.kq : v.vq);
  uint32_t* const params = keys ? v.kp : v.vp;
  const eqat_bf16* const in = keys ? rows.K : rows.V;
  const int64_t pitch = keys ? rows.k_pitch : rows.v_pitch;
  uint4* const hat = reinterpret_cast<uint4*>(keys ? rows.K_hat : rows.V_hat);
  const int step = (int)gridDim.x * kWarps;
  for (int row = (int)blockIdx.x * kWarps + warp; row < v.rows; row += step) {
    if (row >= v.rows - step) ptx::grid_dependents_launch();
    const uint4* x_at = reinterpret_cast<const uint4*>(in + row * pitch) + lane;
    uint4 x[kVectors] = {};
    auto load = [&](int at) {
#pragma unroll
      for (int u = 0; u < kVectors; ++u)
        if (at + 32 * u + lane < upto) x[u] = ptx::ld_global(x_at + at + 32 * u);
    };
    if (APPEND) load(from);
    const RowPlace place = place_of(v, row, lane);
    if (!place.owned) continue;
    uint4* const out = hat == nullptr ? nullptr : hat + (int64_t)row * vectors + lane;
    for (int at = from; at < upto; at += 32 * kVectors) {
      // vector at + 32 u + lane: a head further in the pool every kHead vectors
      const int64_t slot = place.token + (int64_t)((at + lane) / kHead) * v.page_size;
      const int64_t next = (int64_t)(32 / kHead) * v.page_size;
      uint32_t* const code_at = codes + slot * kHead + lane % kHead;
      uint32_t* const param_at = params + slot * kGroups + lane % kHead / kLanes;
      if (APPEND) {
#pragma unroll
        for (int u = 0; u < kVectors; ++u) {
          const uint32_t w[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
          // the NaN forms hand a NaN on
          const __nv_bfloat162 lo = __hmin2_nan(__hmin2_nan(as_pair(w[0]), as_pair(w[1])), __hmin2_nan(as_pair(w[2]), as_pair(w[3])));
          const __nv_bfloat162 hi = __hmax2_nan(__hmax2_nan(as_pair(w[0]), as_pair(w[1])), __hmax2_nan(as_pair(w[2]), as_pair(w[3])));
          // (maximum, -minimum)
          __nv_bfloat162 range = __hmax2_nan(as_pair(__byte_perm(as_word(hi), as_word(lo) ^ 0x80008000u, 0x5410)),
                                             as_pair(__byte_perm(as_word(hi), as_word(lo) ^ 0x80008000u, 0x7632)));
#pragma unroll
          for (int d = 1; d < kLanes; d <<= 1) range = __hmax2_nan(range, as_pair(__shfl_xor_sync(0xFFFFFFFFu, as_word(range), d)));
          const float most = __low2float(range), least = -__high2float(range);
          float s = __bfloat162float(__float2bfloat16_rn(__fmul_rn(__fsub_rn(most, least), 1.0f / 15.0f)));
          if (s < kStepMin) s = 0.0f;
          if (!(s < __int_as_float(0x7F800000))) s = __int_as_float(0x7FC00000);
          const float inverse = s > 0.0f ? __frcp_rn(s) : 0.0f;
          // A code is the low bits of (x - m) / s + 1.5 * 2^23.  With s rounded by at most 2^-8 of itself a quotient stays below
          // 15.06, so no code leaves 0 .. 15 (unless something is NaN).  The word is the sum of the shifted bit patterns,
          // less those of the constant.
          float t[8];
          uint32_t word = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            t[2 * i] = __fadd_rn(__fmul_rn(__fsub_rn(__uint_as_float(w[i] << 16), least), inverse), kMagic);
            t[2 * i + 1] = __fadd_rn(__fmul_rn(__fsub_rn(__uint_as_float(w[i] & 0xFFFF0000u), least), inverse), kMagic);
          }
#pragma unroll
          for (int i = 7; i >= 0; --i) word = word * 16 + __float_as_uint(t[i]);
          word -= 0x3F400000u;                                             // 0x4B400000 (1 + 16 + ... + 16^7) mod 2^32
          if (at + 32 * u + lane < upto) {
            if (place.stands) {
              code_at[u * next * kHead] = word;
              if (lane % kLanes == 0) param_at[u * next * kGroups] = (__float_as_uint(s) >> 16) | (__float_as_uint(least) & 0xFFFF0000u);
            }
            if (out != nullptr) {
              const __nv_bfloat162 s2 = __float2bfloat162_rn(s), m2 = __float2bfloat162_rn(least);
              uint32_t y[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint32_t pair = __byte_perm(__float_as_uint(t[2 * i]), __float_as_uint(t[2 * i + 1]), 0x5410);
                y[i] = place.stands ? value_pair(pair, s2, m2) : 0u;
              }
              out[at + 32 * u] = make_uint4(y[0], y[1], y[2], y[3]);
            }
          }
        }
        if (at + 32 * kVectors < upto) load(at + 32 * kVectors);
      } else {
        uint32_t word[kVectors] = {}, param[kVectors] = {};
        if (place.stands) {
#pragma unroll
          for (int u = 0; u < kVectors; ++u)
            if (at + 32 * u + lane < upto) {
              word[u] = ptx::ld_global(static_cast<const uint32_t*>(code_at + u * next * kHead));
              param[u] = ptx::ld_global(static_cast<const uint32_t*>(param_at + u * next * kGroups));
            }
        }
#pragma unroll
        for (int u = 0; u < kVectors; ++u) {
          const __nv_bfloat162 s2 = as_pair(__byte_perm(param[u], 0, 0x1010)), m2 = as_pair(__byte_perm(param[u], 0, 0x3232));
          uint32_t y[4];                                                   // codes i and i + 4
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = value_pair((word[u] >> (4 * i)) & 0x000F000Fu, s2, m2);
          if (at + 32 * u + lane < upto)
            out[at + 32 * u] = make_uint4(__byte_perm(y[0], y[1], 0x5410), __byte_perm(y[2], y[3], 0x5410), __byte_perm(y[0], y[1], 0x7632),
                                          __byte_perm(y[2], y[3], 0x7632));
        }
      }
    }
  }
}

template <bool APPEND>
int launch_rows(const eqat_cache_desc& d, const CacheView& view, const Rows& rows, cudaStream_t st) {
  const int sms = sm_count();
  if (sms <= 0) return EQAT_ERR_CUDA;
  // A warp takes a whole row where there are enough of them, a piece of one otherwise.
  const int pieces = (d.kv_heads * d.head_dim / 8 + 32 * kVectors - 1) / (32 * kVectors);
  const int64_t warps = (int64_t)sms * 64;
  int per = (int)(d.rows * 2 * pieces / warps);
  per = per < 1 ? 1 : per > pieces ? pieces : per;
  const int groups = (pieces + per - 1) / per;
  if (groups > 32767) return EQAT_ERR_SHAPE;
  const int64_t blocks = (d.rows + kWarps - 1) / kWarps, most = (warps / kWarps + 2 * groups - 1) / (2 * groups);
  const dim3 grid((unsigned)(blocks < most ? blocks : most), (unsigned)(2 * groups));
#define EQAT_ROWS(DD, GG) \
  if (d.head_dim == DD && d.group == GG) return launch_overlapped(cache_rows_kernel<DD, GG, APPEND>, grid, dim3(kWarps * 32), 0, st, view, rows, per);
  EQAT_ROWS(64, 32)
  EQAT_ROWS(64, 64)
  EQAT_ROWS(128, 32)
  EQAT_ROWS(128, 64)
  EQAT_ROWS(128, 128)
  EQAT_ROWS(256, 32)
  EQAT_ROWS(256, 64)
  EQAT_ROWS(256, 128)
#undef EQAT_ROWS
  return EQAT_ERR_UNSUPPORTED;
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
