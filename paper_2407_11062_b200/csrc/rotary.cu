// Rotary positions of queries and keys, forward and backward.
//
// A pair (a, b) at position p turns by p f:  (a cos - b sin, b cos + a sin).  2 pi is kept out of the product: f is given in
// units of 2^-64 of a turn, so the product of integers, mod 2^64, is the angle of any position without an error that grows
// with it (in binary32 a position of 100000 would leave 2^-8 of a radian).
//
// 4 bytes an element cross HBM, which bounds long calls.  A thread owns one item of a row, the same in each of the block's rows:
// 2 x 16 elements of a head (HALVES: a piece of each half; PAIRS: one piece; 8 each where alignment says so), whose places it works out
// once.  It asks for the pieces of all its rows first; while they are on their way the block's warps look the rows' positions up, and
// its threads compute the rows' sines and cosines into shared memory.  4094 rows of 80 heads of 128, a quarter of each turned: 28.3 us,
// 0.90 of a copy's bandwidth (a thread on every 256th item of eight rows, one load at a time: 62.3; items kept, positions first: 43.6;
// 16 bytes at a time, four rows of 256 threads: 29.3; 32 bytes and up to 64, 192, 280 threads: 28.8, 28.7, 30.2; one row of 192:
// 32.4); 64 rows of 72 heads 3.0 us, a launch and two waits for memory.  4096 rows of 40 heads of 128, 34 elements of each turned: 25.3 us as
// halves, 14.4 as pairs (element by element 55.7 and 51.5).
#include "between.cuh"
#include "common.cuh"
#include "pieces.cuh"
#include "ptx.cuh"

namespace eqat {
namespace {

// Elements of a piece: 16 or 8, and of halves that are not whole pieces of 8 also 4, 2 or 1.  Rows of a block, all of whose pieces a
// thread has on their way, and its threads at most (128 against 256 for pieces of 8 and less: -15 % to +3 %; singles +10 %).
__host__ __device__ constexpr int max_rows(int wide) { return wide == 16 ? 2 : 4; }
__host__ __device__ constexpr int max_threads(int wide) { return wide > 1 ? 128 : 256; }

// Place of a pair's cosine and sine among a row's: 16 bytes stay free behind those of each piece (of 16 or 8 elements), or the threads of a
// head, which read at the same place of pieces of their own, would meet in one bank (4096 rows of 64 heads of 128, all of it turned: 20.5 us,
// without those bytes 26.8; of 32 heads of 256 20.9 and 40.9).
__host__ __device__ constexpr int piece_pairs(int layout, int wide) { return wide < 8 ? 1 << 20 : layout == EQAT_ROTARY_HALVES ? wide : wide / 2; }
__host__ __device__ constexpr int turn_place(int piece, int pair) { return pair + pair / piece * 2; }

struct RotaryParams : RotaryRows {
  int rows, sequences, q_heads, heads, head_dim, rotary_dim;
  int block_rows, turned, rest;                      // rows of a block; items of a head that turn, and that are handed on
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

// WIDE elements at a time: a half of the turned part (HALVES) is whole pieces; of neighbouring pairs the last piece may be turned in
// part (PART: asking costs 5 %).  Behind halves that are not whole pieces of 8 the rest is handed on two by two up to the next 16 bytes, from there 16 bytes
// at a time.
template <int LAYOUT, int WIDE, bool PART>
__global__ void __launch_bounds__(max_threads(WIDE)) rotary_kernel(const RotaryParams p) {
  constexpr int kRows = max_rows(WIDE);
  __shared__ int s_pos[kRows];
  __shared__ bool s_live[kRows];
  extern __shared__ __align__(16) float2 s_turn[];   // [block_rows][turn_place(rotary_dim / 2)]: cosine, sine, times the amplitude
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int kPiece = piece_pairs(LAYOUT, WIDE);
  const int pairs = p.rotary_dim >> 1, turn_pitch = turn_place(kPiece, pairs);
  const int row0 = (int)blockIdx.x * p.block_rows, nrows = min(p.block_rows, p.rows - row0);
  // this thread's item: the c-th of a head, turned ones first, then those handed on
  const int item = (int)(blockIdx.y * blockDim.x + threadIdx.x), items = p.turned + p.rest;
  int head = item / items;
  const int c = item - head * items;
  if (head >= p.heads) head = -1;
  const bool query = head < p.q_heads;
  const int64_t at = (int64_t)(query ? max(head, 0) : head - p.q_heads) * p.head_dim;
  const int64_t src_pitch = query ? p.q_pitch : p.k_pitch, dst_pitch = query ? p.q_out_pitch : p.k_out_pitch;
  const eqat_bf16* const src = (query ? p.q : p.k) + row0 * src_pitch + at;
  eqat_bf16* const dst = (query ? p.q_out : p.k_out) + row0 * dst_pitch + at;
  const bool turns = head >= 0 && c < p.turned, rests = head >= 0 && c >= p.turned && src != dst;
  constexpr bool kTwo = LAYOUT == EQAT_ROTARY_HALVES, kNarrow = WIDE < 8;  // an item that turns has two parts
  // first and (kTwo) second part of an item that turns; place of one that is handed on
  const int up = (p.rotary_dim + 7) & ~7, words = (up - p.rotary_dim) >> 1, r = c - p.turned;
  const int ea = turns || !kNarrow ? c * WIDE + (kTwo && !turns ? pairs : 0) : r < words ? p.rotary_dim + 2 * r : up + 8 * (r - words);
  const int eb = ea + pairs;
  ptx::grid_dependency_wait();
  Piece<WIDE> va[kRows], vb[kTwo ? kRows : 1];
  Piece<8> vr[kNarrow ? kRows : 1];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const eqat_bf16* const in = src + i * src_pitch;
    if (i < nrows && (turns || (rests && !kNarrow))) va[i] = load_piece<WIDE>(in + ea);
    if constexpr (kTwo)
      if (i < nrows && turns) vb[i] = load_piece<WIDE>(in + eb);
    if constexpr (kNarrow)
      if (i < nrows && rests) {
        if (r < words) vr[i].w[0] = load_piece<2>(in + ea).w[0];
        else vr[i] = load_piece<8>(in + ea);
      }
  }
  if (warp < nrows) {
    int pos = 0;
    const bool live = position_of(p, row0 + warp, lane, pos);
    if (lane == 0) {
      s_pos[warp] = pos;
      s_live[warp] = live;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < nrows * pairs; i += (int)blockDim.x) {
    const int r = i / pairs, k = i - r * pairs;
    const uint2 f = ptx::ld_global(reinterpret_cast<const uint2*>(p.turns) + k);
    const uint64_t angle = (uint64_t)(int64_t)s_pos[r] * (((uint64_t)f.y << 32) | f.x) + 0x80000000ull;
    float sn, cs;
    sincospif((float)(int32_t)(angle >> 32) * 0x1p-31f, &sn, &cs);
    s_turn[r * turn_pitch + turn_place(kPiece, k)] = make_float2(cs * p.amplitude, sn * p.sine);
  }
  __syncthreads();
  ptx::grid_dependents_launch();
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (i >= nrows || !s_live[i]) continue;
    eqat_bf16* const out = dst + i * dst_pitch;
    if (rests) {
      if constexpr (!kNarrow) store_piece(out + ea, va[i]);
      else if (r < words) store_piece(out + ea, Piece<2>{{vr[i].w[0]}});
      else store_piece(out + ea, vr[i]);
    }
    if (!turns) continue;
    if constexpr (WIDE == 1) {
      const float a = __uint_as_float((uint32_t)va[i].w << 16), b = __uint_as_float((uint32_t)vb[i].w << 16);
      const float2 t = s_turn[i * turn_pitch + c];
      const uint32_t o = pack_bf16x2(a * t.x - b * t.y, b * t.x + a * t.y);
      out[ea] = (eqat_bf16)(o & 0xFFFFu);
      out[eb] = (eqat_bf16)(o >> 16);
    } else {
      const float2* const turn = s_turn + i * turn_pitch + turn_place(kPiece, kTwo ? ea : ea / 2);
      Piece<WIDE> oa;
      if constexpr (kTwo) {
        Piece<WIDE> ob;
#pragma unroll
        for (int e = 0; e < WIDE / 2; ++e) {
          const float4 t = reinterpret_cast<const float4*>(turn)[e];
          float a0, a1, b0, b1;
          halves_of(va[i].w[e], a0, a1);
          halves_of(vb[i].w[e], b0, b1);
          oa.w[e] = pack_bf16x2(a0 * t.x - b0 * t.y, a1 * t.z - b1 * t.w);
          ob.w[e] = pack_bf16x2(b0 * t.x + a0 * t.y, b1 * t.z + a1 * t.w);
        }
        store_piece(out + eb, ob);
      } else {
#pragma unroll
        for (int e = 0; e < WIDE / 2; ++e) {
          if (PART && ea / 2 + e >= pairs) {
            oa.w[e] = va[i].w[e];
            continue;
          }
          const float2 t = turn[e];
          float a, b;
          halves_of(va[i].w[e], a, b);
          oa.w[e] = pack_bf16x2(a * t.x - b * t.y, b * t.x + a * t.y);
        }
      }
      store_piece(out + ea, oa);
    }
  }
}

// Items of a head that turn, and that are handed on where a result is not in place.
constexpr int turned_items(int layout, int wide, int rotary_dim) {
  return layout == EQAT_ROTARY_HALVES ? rotary_dim / 2 / wide : (rotary_dim + wide - 1) / wide;
}
constexpr int rest_items(int layout, int wide, int head_dim, int rotary_dim) {
  const int up = (rotary_dim + 7) & ~7;
  return wide < 8 ? (up - rotary_dim) / 2 + (head_dim - up) / 8
                  : head_dim / wide - (layout == EQAT_ROTARY_HALVES ? 2 : 1) * turned_items(layout, wide, rotary_dim);
}
// The largest piece that a half of `part` elements consists of (0: no halves), where 32 bytes at a time cannot be had.
constexpr int piece_of(int part) { return part % 8 == 0 ? 8 : part % 4 == 0 ? 4 : part % 2 == 0 ? 2 : 1; }

// A row's items go over the grid's second dimension, at most 65535 blocks: 256 items a head over 256 threads (510 elements as halves) and
// 129 over 128 (508) are the most there are.
constexpr bool rows_fit_the_grid() {
  for (int layout : {EQAT_ROTARY_HALVES, EQAT_ROTARY_PAIRS})
    for (int dim = 2; dim <= kMaxRotaryHeadDim; dim += 2) {
      const int part = layout == EQAT_ROTARY_HALVES ? dim / 2 : 0;
      for (int wide : {piece_of(part), 16}) {
        if (part % wide != 0) continue;
        const int64_t items = 2ll * kMaxRotaryHeads * (turned_items(layout, wide, dim) + rest_items(layout, wide, kMaxRotaryHeadDim, dim));
        if ((items + max_threads(wide) - 1) / max_threads(wide) > 65535) return false;
      }
    }
  return true;
}
static_assert(rows_fit_the_grid(), "blocks of a row");

template <int WIDE>
int launch_pieces(const eqat_rotary_desc& d, const RotaryRows& rows, RotaryParams& p, int sms, cudaStream_t st) {
  const bool halves = d.layout == EQAT_ROTARY_HALVES;
  const bool in_place = rows.q == rows.q_out && (d.kv_heads == 0 || rows.k == rows.k_out);
  p.turned = turned_items(d.layout, WIDE, d.rotary_dim);
  p.rest = in_place ? 0 : rest_items(d.layout, WIDE, d.head_dim, d.rotary_dim);
  constexpr int kMost = max_threads(WIDE);
  const int64_t items = (int64_t)p.heads * (p.turned + p.rest), chunks = (items + kMost - 1) / kMost;
  // threads enough for a row in as many blocks, and a warp for each row's position
  const int even = (int)((items + chunks - 1) / chunks + 31) / 32 * 32, least = 32 * max_rows(WIDE);
  const dim3 threads(even > least ? even : least);
  // several rows a block where there are enough blocks all the same
  const int64_t per = d.rows * chunks / ((int64_t)sms * 8);
  p.block_rows = (int)(per < 1 ? 1 : per > max_rows(WIDE) ? max_rows(WIDE) : per);
  const dim3 grid((unsigned)((d.rows + p.block_rows - 1) / p.block_rows), (unsigned)chunks);
  const size_t smem = (size_t)p.block_rows * turn_place(piece_pairs(d.layout, WIDE), d.rotary_dim / 2) * sizeof(float2);
  if constexpr (WIDE >= 8)
    if (!halves)
      return d.rotary_dim % WIDE == 0 ? launch_overlapped(rotary_kernel<EQAT_ROTARY_PAIRS, WIDE, false>, grid, threads, smem, st, p)
                                      : launch_overlapped(rotary_kernel<EQAT_ROTARY_PAIRS, WIDE, true>, grid, threads, smem, st, p);
  return launch_overlapped(rotary_kernel<EQAT_ROTARY_HALVES, WIDE, false>, grid, threads, smem, st, p);
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
  const int part = d.layout == EQAT_ROTARY_HALVES ? d.rotary_dim / 2 : 0;          // what has to be whole pieces
  const bool keys = d.kv_heads > 0;
  if (part % 16 == 0 && d.head_dim % 16 == 0 && (rows.q_pitch | rows.q_out_pitch) % 16 == 0 && aligned32(rows.q, rows.q_out) &&
      (!keys || ((rows.k_pitch | rows.k_out_pitch) % 16 == 0 && aligned32(rows.k, rows.k_out))))
    return launch_pieces<16>(d, rows, p, sms, st);
  switch (piece_of(part)) {
    case 8: return launch_pieces<8>(d, rows, p, sms, st);
    case 4: return launch_pieces<4>(d, rows, p, sms, st);
    case 2: return launch_pieces<2>(d, rows, p, sms, st);
    default: return launch_pieces<1>(d, rows, p, sms, st);
  }
}

}  // namespace eqat
