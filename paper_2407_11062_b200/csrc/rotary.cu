// Rotary positions of queries and keys, forward and backward.
//
// A pair (a, b) at position p turns by p f:  (a cos - b sin, b cos + a sin).  2 pi is kept out of the product: f is given in
// units of 2^-64 of a turn, so the product of integers, mod 2^64, is the angle of any position without an error that grows
// with it (in binary32 a position of 100000 would leave 2^-8 of a radian).
//
// 4 bytes an element cross HBM, which bounds long calls.  A block takes up to eight rows: its warps look the rows' positions
// up, its threads compute the rows' sines and cosines into shared memory, once for all heads, and then every thread turns
// 2 x 8 elements at a time (HALVES: a vector of each half; PAIRS: one vector).
#include "between.cuh"
#include "common.cuh"
#include "ptx.cuh"

namespace eqat {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxRows = kThreads / 32;              // rows of a block: one a warp

struct RotaryParams : RotaryRows {
  int rows, sequences, q_heads, heads, head_dim, rotary_dim;
  int block_rows, block_heads;
  float amplitude, sine;                             // sine: amplitude, or its negative (backward)
};

__device__ __forceinline__ int ld_int(const int32_t* p) { return (int)ptx::ld_global(reinterpret_cast<const uint32_t*>(p)); }

// Whole warp: the position of a row; false if it belongs to no sequence.
__device__ __forceinline__ bool position_of(const RotaryParams& p, int row, int lane, int& pos) {
  if (p.positions != nullptr) {
    pos = ld_int(p.positions + row);
    return true;
  }
  int low = 0, high = p.sequences;
  while (low < high) {
    const int step = (high - low + 31) >> 5;
    const int probe = low + (lane + 1) * step;
    const bool before = probe <= high && ld_int(p.row_offsets + probe) <= row;
    const int n = __popc(__ballot_sync(0xFFFFFFFFu, before));
    low += n * step;
    high = min(high, low + step - 1);
  }
  if (low >= p.sequences) return false;
  pos = ld_int(p.lengths + low) - (min(ld_int(p.row_offsets + low + 1), p.rows) - row);
  return true;
}

__device__ __forceinline__ void halves_of(uint32_t w, float& lo, float& hi) {
  lo = __uint_as_float(w << 16);
  hi = __uint_as_float(w & 0xFFFF0000u);
}

// VECTORS: 16 bytes at a time (a half of the turned part, or all of it, is whole vectors), else element by element.
template <int LAYOUT, bool VECTORS>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const RotaryParams p) {
  __shared__ int s_pos[kMaxRows];
  __shared__ bool s_live[kMaxRows];
  extern __shared__ __align__(16) float2 s_turn[];   // [block_rows][rotary_dim / 2]: cosine, sine, times the amplitude
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int pairs = p.rotary_dim >> 1;
  const int row0 = (int)blockIdx.x * p.block_rows, nrows = min(p.block_rows, p.rows - row0);
  const int head0 = (int)blockIdx.y * p.block_heads, nheads = min(p.block_heads, p.heads - head0);
  ptx::grid_dependency_wait();
  if (warp < nrows) {
    int pos = 0;
    const bool live = position_of(p, row0 + warp, lane, pos);
    if (lane == 0) {
      s_pos[warp] = pos;
      s_live[warp] = live;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < nrows * pairs; i += kThreads) {
    const int r = i / pairs, k = i - r * pairs;
    const uint2 f = ptx::ld_global(reinterpret_cast<const uint2*>(p.turns) + k);
    const uint64_t angle = (uint64_t)(int64_t)s_pos[r] * (((uint64_t)f.y << 32) | f.x) + 0x80000000ull;
    float sn, cs;
    sincospif((float)(int32_t)(angle >> 32) * 0x1p-31f, &sn, &cs);
    s_turn[i] = make_float2(cs * p.amplitude, sn * p.sine);
  }
  __syncthreads();
  ptx::grid_dependents_launch();

  // items of a head: turned first, then handed on
  constexpr int kWide = VECTORS ? 8 : 1;
  const int turned = LAYOUT == EQAT_ROTARY_HALVES ? pairs / kWide : p.rotary_dim / (VECTORS ? 8 : 2);
  const int rest = (p.head_dim - p.rotary_dim) / kWide, items = turned + rest;
  const int per_row = nheads * items;
  for (int i = threadIdx.x; i < nrows * per_row; i += kThreads) {
    const int r = i / per_row, j = i - r * per_row;
    const int h = j / items, c = j - h * items, head = head0 + h, row = row0 + r;
    if (!s_live[r]) continue;
    const bool query = head < p.q_heads;
    const int64_t at = (int64_t)(query ? head : head - p.q_heads) * p.head_dim;
    const eqat_bf16* src = query ? p.q + row * p.q_pitch + at : p.k + row * p.k_pitch + at;
    eqat_bf16* dst = query ? p.q_out + row * p.q_out_pitch + at : p.k_out + row * p.k_out_pitch + at;
    if (c >= turned) {
      if (src != dst) {
        const int e = p.rotary_dim + (c - turned) * kWide;
        if constexpr (VECTORS) *reinterpret_cast<uint4*>(dst + e) = ptx::ld_global_once(reinterpret_cast<const uint4*>(src + e));
        else dst[e] = ptx::ld_global(src + e);
      }
      continue;
    }
    const float2* turn = s_turn + r * pairs;
    if constexpr (!VECTORS) {
      const int ia = LAYOUT == EQAT_ROTARY_HALVES ? c : 2 * c, ib = LAYOUT == EQAT_ROTARY_HALVES ? c + pairs : 2 * c + 1;
      const float a = __uint_as_float((uint32_t)ptx::ld_global(src + ia) << 16), b = __uint_as_float((uint32_t)ptx::ld_global(src + ib) << 16);
      const float2 t = turn[c];
      const uint32_t o = pack_bf16x2(a * t.x - b * t.y, b * t.x + a * t.y);
      dst[ia] = (eqat_bf16)(o & 0xFFFFu);
      dst[ib] = (eqat_bf16)(o >> 16);
    } else if constexpr (LAYOUT == EQAT_ROTARY_HALVES) {
      const uint4 va = ptx::ld_global_once(reinterpret_cast<const uint4*>(src) + c);
      const uint4 vb = ptx::ld_global_once(reinterpret_cast<const uint4*>(src + pairs) + c);
      const uint32_t wa[4] = {va.x, va.y, va.z, va.w}, wb[4] = {vb.x, vb.y, vb.z, vb.w};
      uint32_t oa[4], ob[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float4 t = reinterpret_cast<const float4*>(turn + 8 * c)[e];
        float a0, a1, b0, b1;
        halves_of(wa[e], a0, a1);
        halves_of(wb[e], b0, b1);
        oa[e] = pack_bf16x2(a0 * t.x - b0 * t.y, a1 * t.z - b1 * t.w);
        ob[e] = pack_bf16x2(b0 * t.x + a0 * t.y, b1 * t.z + a1 * t.w);
      }
      reinterpret_cast<uint4*>(dst)[c] = make_uint4(oa[0], oa[1], oa[2], oa[3]);
      reinterpret_cast<uint4*>(dst + pairs)[c] = make_uint4(ob[0], ob[1], ob[2], ob[3]);
    } else {
      const uint4 v = ptx::ld_global_once(reinterpret_cast<const uint4*>(src) + c);
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
      uint32_t o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 t = turn[4 * c + e];
        float a, b;
        halves_of(w[e], a, b);
        o[e] = pack_bf16x2(a * t.x - b * t.y, b * t.x + a * t.y);
      }
      reinterpret_cast<uint4*>(dst)[c] = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
}

}  // namespace

int launch_rotary(const eqat_rotary_desc& d, const RotaryRows& rows, bool backward, cudaStream_t st) {
  const int sms = sm_count();
  if (sms <= 0) return EQAT_ERR_CUDA;
  RotaryParams p;
  static_cast<RotaryRows&>(p) = rows;
  p.rows = (int)d.rows;
  p.sequences = d.sequences;
  p.q_heads = d.q_heads;
  p.heads = d.q_heads + d.kv_heads;
  p.head_dim = d.head_dim;
  p.rotary_dim = d.rotary_dim;
  p.amplitude = d.amplitude;
  p.sine = backward ? -d.amplitude : d.amplitude;
  // Several rows a block where there are enough of them, several blocks a row where there are few.
  const int64_t wave = (int64_t)sms * 4;
  int64_t per = d.rows / wave;
  p.block_rows = (int)(per < 1 ? 1 : per > kMaxRows ? kMaxRows : per);
  const int64_t bx = (d.rows + p.block_rows - 1) / p.block_rows;
  const int row_items = p.heads * (d.head_dim / 16);
  int64_t by = (wave + bx - 1) / bx;
  const int64_t most = (row_items + kThreads - 1) / kThreads;
  by = by > most ? most : by;
  by = by > p.heads ? p.heads : by;
  by = by < 1 ? 1 : by;
  p.block_heads = (int)((p.heads + by - 1) / by);
  const dim3 grid((unsigned)bx, (unsigned)((p.heads + p.block_heads - 1) / p.block_heads));
  const size_t smem = (size_t)p.block_rows * (d.rotary_dim / 2) * sizeof(float2);
  const bool halves = d.layout == EQAT_ROTARY_HALVES;
  const bool vectors = d.rotary_dim % (halves ? 16 : 8) == 0;
  if (halves)
    return vectors ? launch_overlapped(rotary_kernel<EQAT_ROTARY_HALVES, true>, grid, dim3(kThreads), smem, st, p)
                   : launch_overlapped(rotary_kernel<EQAT_ROTARY_HALVES, false>, grid, dim3(kThreads), smem, st, p);
  return vectors ? launch_overlapped(rotary_kernel<EQAT_ROTARY_PAIRS, true>, grid, dim3(kThreads), smem, st, p)
                 : launch_overlapped(rotary_kernel<EQAT_ROTARY_PAIRS, false>, grid, dim3(kThreads), smem, st, p);
}

}  // namespace eqat
