// Root-mean-square norm of the residual stream, with the addition to it and an output in bf16 or 8 bits; its gradient.
//
//     h = bf16(x + r),  c = (mean(h^2) + eps)^(-1/2),  y = h w c
//     dx = dr + c (v - h c^2 mean(v h)),  v = dy w;     dw = sum over the rows of dy h c
//
// One pass: each tensor crosses HBM once, 8 bytes an element forward with a residual (7 + 4/group with codes in place of y), 8
// backward.
//
// Forward: a row a block (a warp for short ones), 32 bytes of each tensor at a time where everything is aligned to them.  What hides
// the way to HBM are many blocks an SM, so registers count: rows one after the other in blocks that stay, the next ones copied ahead
// or not, took 54.8 and 60.5 us where this takes 50.1 (8191 x 5120 with a residual, 1.02 of a copy's bandwidth), 16 bytes at a time
// 55.4.  With codes (2001 x 8192 in e4m3: 24.7 us, 0.92: conversions and the groups' maxima) blocks have 256 threads at most, so that
// some load while others convert: 27.0 with 512, 26.5 with a row copied ahead.  One row of 4096: 2.6 us, a launch.
//
// Backward: a thread owns the same columns of every row that its block meets, so w is read once a block and dw is added up in registers.
// What it will read of the next rows it copies into shared memory itself (cp.async, up to two rows ahead): nobody else reads its
// places, so a row costs no barrier but that of the sum, and the copies run on through it.  4096 x 4096: 26.4 us (0.78; 22.4 us
// without dw, whose partial sums are a launch of 3 us).  Before the ring and with the row unpacked twice it took 38.2 us, 9 of them the
// sum of the partial sums by eight warps of a block.
#include <cuda_fp8.h>

#include "between.cuh"
#include "common.cuh"
#include "expand.cuh"
#include "pieces.cuh"
#include "ptx.cuh"

namespace eqat {
namespace {

constexpr int kBlock = 256;                          // threads of a block that gives each row to a warp
constexpr int kMaxThreads = 512;                     // of a block that shares a row
constexpr int kLoopThreads = 128;                    // forward: of a block that takes one row after the other
constexpr int kRingBytes = 200 * 1024;               // shared memory of an SM for the blocks' rings
constexpr float kSmallGroup = 0x1p-110f;             // 127 / a and 448 / a are finite above

__device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
// The sum rounded to bf16 once; rounding to binary32 on the way would not change it (operands of 8 bits whose exponents differ by
// more than 16 are nowhere near half a step).
__device__ __forceinline__ uint32_t add_pair(uint32_t a, uint32_t b) {
  const __nv_bfloat162 s = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&s);
}
__device__ __forceinline__ uint4 pack(const float (&f)[8]) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

__device__ __forceinline__ void two_vectors(const Piece<16>& v, uint4& a, uint4& b) {
  a = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
  b = make_uint4(v.w[4], v.w[5], v.w[6], v.w[7]);
}
__device__ __forceinline__ Piece<16> one_piece(const uint4& a, const uint4& b) { return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}}; }

// The sum of a pair and the maximum of a third over the threads of a row: a warp, or the block.  `red` is used in turns: a
// thread that writes the same half again has passed the barrier of the turn between, and so have all the readers.
struct Reduced {
  float a, b, most;
};
template <bool WARP>
__device__ __forceinline__ Reduced reduce_row(Reduced x, Reduced (*red)[32], int turn) {
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    x.a += __shfl_xor_sync(0xFFFFFFFFu, x.a, d);
    x.b += __shfl_xor_sync(0xFFFFFFFFu, x.b, d);
    x.most = fmaxf(x.most, __shfl_xor_sync(0xFFFFFFFFu, x.most, d));
  }
  if (WARP) return x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  if (lane == 0) red[turn & 1][warp] = x;
  __syncthreads();
  x = lane < warps ? red[turn & 1][lane] : Reduced{0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    x.a += __shfl_xor_sync(0xFFFFFFFFu, x.a, d);
    x.b += __shfl_xor_sync(0xFFFFFFFFu, x.b, d);
    x.most = fmaxf(x.most, __shfl_xor_sync(0xFFFFFFFFu, x.most, d));
  }
  return x;
}

__device__ __forceinline__ void copy_16(uint32_t dst, const uint4* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// All copies but those of the last stages - 1 groups have arrived.
__device__ __forceinline__ void copies_arrived(int stages) {
  if (stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else if (stages == 2) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

struct NormFwd {
  const eqat_bf16 *X, *R, *W;
  eqat_bf16 *H, *Y;
  uint8_t* codes;
  float* scales;
  int rows, vecs;                                    // vecs: 16-byte vectors of a row
  float eps, inverse_n;
  int lanes, lanes_log2;                             // codes: vectors of a group (4 .. 32 neighbouring lanes), or 0: the row
  int groups;                                        // of a row
};

// VPT vectors of a row per thread; a row belongs to a warp (WARP) or to the block.  Wide blocks have one row: a loop over rows costs
// registers, and with them threads of an SM (LOOP: short rows, where starting a block costs more).  A thread's vectors are
// neighbours by two where a row has an even number of them (NEXT); WIDE: and they are moved as one piece.  So the order of a sum
// hangs on the shape alone, not on alignment.
template <int VPT, bool WARP, bool LOOP, int CODES, bool NEXT, bool WIDE>
__global__ void __launch_bounds__(WARP ? kBlock : LOOP ? kLoopThreads : kMaxThreads, WARP ? (LOOP ? 8 : 4) : LOOP ? 8 : VPT == 2 ? 3 : VPT == 4 ? 2 : 1)
norm_fwd_kernel(const NormFwd p) {
  static_assert(!NEXT || VPT % 2 == 0, "two neighbours");
  __shared__ Reduced red[2][32];
  const int lane = threadIdx.x & 31;
  const int at = WARP ? lane : (int)threadIdx.x, span = WARP ? 32 : (int)blockDim.x;
  auto place = [&](int i) { return NEXT ? ((i >> 1) * span + at) * 2 + (i & 1) : at + i * span; };      // of vector i of this thread
  const int step = (int)gridDim.x * (WARP ? kBlock / 32 : 1);
  const int first = WARP ? (int)blockIdx.x * (kBlock / 32) + (int)(threadIdx.x >> 5) : (int)blockIdx.x;
  constexpr float kTop = CODES == EQAT_CODES_INT8 ? 127.0f : 448.0f;
  const bool residual = p.R != nullptr;
  ptx::grid_dependency_wait();
  uint4 w[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i)
    w[i] = place(i) < p.vecs ? ptx::ld_global(reinterpret_cast<const uint4*>(p.W) + place(i)) : make_uint4(0u, 0u, 0u, 0u);
  int turn = 0;
  for (int row = first; row < p.rows; row = LOOP ? row + step : p.rows, ++turn) {
    const size_t base = (size_t)row * p.vecs;
    uint4 x[VPT] = {}, r[VPT] = {};
    // vectors of this thread in a row, stored or loaded
    auto load = [&](const eqat_bf16* from, uint4 (&v)[VPT]) {
#pragma unroll
      for (int i = 0; i < VPT; ++i) {
        if constexpr (WIDE) {
          if (i % 2 == 0 && place(i) < p.vecs) two_vectors(load_piece<16>(from + (base + place(i)) * 8), v[i], v[i + 1]);
        } else {
          if (place(i) < p.vecs) v[i] = ptx::ld_global_once(reinterpret_cast<const uint4*>(from) + base + place(i));
        }
      }
    };
    auto store = [&](eqat_bf16* to, int i) {           // vector i of x, or with it the one before
      if constexpr (WIDE) {
        if (i % 2 == 1 && place(i) < p.vecs) store_piece(to + (base + place(i - 1)) * 8, one_piece(x[i - 1], x[i]));
      } else {
        if (place(i) < p.vecs) reinterpret_cast<uint4*>(to)[base + place(i)] = x[i];
      }
    };
    load(p.X, x);
    if (residual) load(p.R, r);
    if (!LOOP || row >= p.rows - step) ptx::grid_dependents_launch();
    // With codes, the products of up to two vectors a thread are held through the sum, more are formed again.
    constexpr int kHeld = VPT < 2 ? 1 : 2;
    float t[kHeld][8], most[VPT];
    Reduced s{0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      if (residual) x[i] = make_uint4(add_pair(x[i].x, r[i].x), add_pair(x[i].y, r[i].y), add_pair(x[i].z, r[i].z), add_pair(x[i].w, r[i].w));
      float h[8], g[8];
      unpack(x[i], h);
      if (p.H != nullptr && (residual || p.H != p.X)) store(p.H, i);
#pragma unroll
      for (int e = 0; e < 8; ++e) s.a = fmaf(h[e], h[e], s.a);
      if constexpr (CODES != EQAT_CODES_NONE) {
        unpack(w[i], g);
        most[i] = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          t[i % kHeld][e] = h[e] * g[e];
          most[i] = fmaxf(most[i], fabsf(t[i % kHeld][e]));
        }
        if (p.lanes == 0) {
          s.most = fmaxf(s.most, most[i]);
        } else if (!NEXT) {
          for (int d = 1; d < p.lanes; d <<= 1) most[i] = fmaxf(most[i], __shfl_xor_sync(0xFFFFFFFFu, most[i], d));
        } else if (i % 2 == 1) {                       // both are of one group, which is half as many lanes
          most[i] = fmaxf(most[i - 1], most[i]);
          for (int d = 1; d < p.lanes / 2; d <<= 1) most[i] = fmaxf(most[i], __shfl_xor_sync(0xFFFFFFFFu, most[i], d));
          most[i - 1] = most[i];
        }
      }
    }
    s = reduce_row<WARP>(s, red, turn);
    const float c = rsqrtf(fmaf(s.a, p.inverse_n, p.eps));
    uint2 even, odd = make_uint2(0u, 0u);              // codes of two vectors
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float (&h)[8] = t[i % kHeld];
      if (CODES == EQAT_CODES_NONE || VPT > kHeld) {
        float g[8];
        unpack(x[i], h);
        unpack(w[i], g);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] *= g[e];
      }
      if constexpr (CODES == EQAT_CODES_NONE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] *= c;
        x[i] = pack(h);
        store(p.Y, i);
      } else {
        float a = p.lanes == 0 ? s.most : most[i];
        if (a < kSmallGroup) a = 0.0f;
        const float up = a > 0.0f ? __fdiv_rn(kTop, a) : 0.0f;
        const float scale = a * c * (1.0f / kTop);
        even = odd;
        if constexpr (CODES == EQAT_CODES_INT8) {
          // |t| is at most 127 (1 + 2^-23), so the low byte of t + 1.5 2^23 is the code
          uint32_t k[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float v = __fadd_rn(__fmul_rn(h[e], up), 12582912.0f);
            k[e] = __float_as_uint(v);
            h[e] = (v - 12582912.0f) * scale;
          }
          odd = make_uint2(__byte_perm(__byte_perm(k[0], k[1], 0x0040), __byte_perm(k[2], k[3], 0x0040), 0x5410),
                           __byte_perm(__byte_perm(k[4], k[5], 0x0040), __byte_perm(k[6], k[7], 0x0040), 0x5410));
        } else {
          uint32_t k[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            k[e] = __nv_cvt_float2_to_fp8x2(make_float2(__fmul_rn(h[2 * e], up), __fmul_rn(h[2 * e + 1], up)), __NV_SATFINITE, __NV_E4M3);
            const __half2_raw v = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)k[e], __NV_E4M3);
            const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&v));
            h[2 * e] = y.x * scale;
            h[2 * e + 1] = y.y * scale;
          }
          odd = make_uint2(k[0] | (k[1] << 16), k[2] | (k[3] << 16));
        }
        x[i] = pack(h);
        if (p.Y != nullptr) store(p.Y, i);
        if (place(i) < p.vecs) {
          if constexpr (!NEXT) reinterpret_cast<uint2*>(p.codes)[base + place(i)] = odd;
          else if (i % 2 == 1) reinterpret_cast<uint4*>(p.codes)[(base + place(i - 1)) / 2] = make_uint4(even.x, even.y, odd.x, odd.y);
          if (p.lanes == 0) {
            if (at == 0 && i == 0) p.scales[row] = scale;
          } else if (NEXT ? i % 2 == 0 && (lane & (p.lanes / 2 - 1)) == 0 : (lane & (p.lanes - 1)) == 0) {
            p.scales[(size_t)row * p.groups + (place(i) >> p.lanes_log2)] = scale;
          }
        }
      }
    }
  }
}

struct NormBwd {
  const eqat_bf16 *dY, *H, *W, *dR;
  eqat_bf16* dX;
  float* partial;                                    // [blocks, features]; NULL: no dW
  int rows, vecs;
  float eps, inverse_n;
};

// `stages` of the ring, then (WARP) the warps' sums, [warps][features], in the same places.
template <int VPT, bool WARP>
__global__ void __launch_bounds__(WARP ? kBlock : kMaxThreads) norm_bwd_kernel(const NormBwd p, int stages) {
  __shared__ Reduced red[2][32];
  extern __shared__ __align__(16) uint8_t ring[];
  float* const share = reinterpret_cast<float*>(ring);
  constexpr int kHeld = VPT < 2 ? 1 : 2;
  const int lane = threadIdx.x & 31;
  const int at = WARP ? lane : (int)threadIdx.x, span = WARP ? 32 : (int)blockDim.x;
  const int step = (int)gridDim.x * (WARP ? kBlock / 32 : 1);
  const int first = WARP ? (int)blockIdx.x * (kBlock / 32) + (int)(threadIdx.x >> 5) : (int)blockIdx.x;
  const bool residual = p.dR != nullptr;
  const uint32_t mine = ptx::smem_addr(ring) + threadIdx.x * 16, pitch = blockDim.x * 16;
  const uint32_t stage_bytes = pitch * VPT * (residual ? 3 : 2);
  ptx::grid_dependency_wait();
  auto ask = [&](int row, int stage) {
    if (row < p.rows) {
      const size_t base = (size_t)row * p.vecs + at;
      uint32_t dst = mine + stage * stage_bytes;
#pragma unroll
      for (int t = 0; t < 3; ++t) {
        const eqat_bf16* src = t == 0 ? p.H : t == 1 ? p.dY : p.dR;
        if (t < 2 || residual) {
#pragma unroll
          for (int i = 0; i < VPT; ++i, dst += pitch)
            if (at + i * span < p.vecs) copy_16(dst, reinterpret_cast<const uint4*>(src) + base + i * span);
        }
      }
    }
    copies_issued();
  };
  int ahead = first, fill = 0;
  for (int k = 0; k + 1 < stages; ++k, ahead += step) ask(ahead, fill++);
  uint4 w[VPT];
  float dw[VPT][8];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    w[i] = at + i * span < p.vecs ? ptx::ld_global(reinterpret_cast<const uint4*>(p.W) + at + i * span) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[i][e] = 0.0f;
  }
  int turn = 0, stage = 0;
  for (int row = first; row < p.rows; row += step, ++turn) {
    if (row >= p.rows - step) ptx::grid_dependents_launch();
    ask(ahead, fill);
    ahead += step;
    if (++fill == stages) fill = 0;
    copies_arrived(stages);
    const uint32_t slot = mine + stage * stage_bytes;
    if (++stage == stages) stage = 0;
    auto vector_of = [&](int tensor, int i) {
      return at + i * span < p.vecs ? ptx::lds_128(slot + (tensor * VPT + i) * pitch) : make_uint4(0u, 0u, 0u, 0u);
    };
    // Up to two vectors a thread are held through the sum as they are used after it; of more, the row is read once more.
    float h[kHeld][8], y[kHeld][8];
    Reduced s{0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float (&hh)[8] = h[i % kHeld], (&yy)[8] = y[i % kHeld];
      unpack(vector_of(0, i), hh);
      unpack(vector_of(1, i), yy);
      float g[8];
      unpack(w[i], g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s.a = fmaf(hh[e], hh[e], s.a);
        s.b = fmaf(yy[e] * g[e], hh[e], s.b);
      }
    }
    s = reduce_row<WARP>(s, red, turn);
    const float c = rsqrtf(fmaf(s.a, p.inverse_n, p.eps));
    const float k = c * (s.b * p.inverse_n);           // c^2 by itself would leave binary32 where c passes 2^64
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float (&hh)[8] = h[i % kHeld], (&yy)[8] = y[i % kHeld];
      if constexpr (VPT > kHeld) {
        unpack(vector_of(0, i), hh);
        unpack(vector_of(1, i), yy);
      }
      float g[8], r[8];
      unpack(w[i], g);
      unpack(residual ? vector_of(2, i) : make_uint4(0u, 0u, 0u, 0u), r);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float hc = hh[e] * c;
        dw[i][e] = fmaf(yy[e], hc, dw[i][e]);
        r[e] = fmaf(c, fmaf(-hc, k, yy[e] * g[e]), r[e]);
      }
      if (at + i * span < p.vecs) reinterpret_cast<uint4*>(p.dX)[(size_t)row * p.vecs + at + i * span] = pack(r);
    }
  }
  if (p.partial == nullptr) return;
  const int features = p.vecs * 8;
  float* out = p.partial + (size_t)blockIdx.x * features;
  if (WARP) __syncthreads();                         // the ring is done with
  if (WARP) out = share + (size_t)(threadIdx.x >> 5) * features;
#pragma unroll
  for (int i = 0; i < VPT; ++i)
    if (at + i * span < p.vecs) {
      float4* o = reinterpret_cast<float4*>(out) + (size_t)(at + i * span) * 2;
      o[0] = make_float4(dw[i][0], dw[i][1], dw[i][2], dw[i][3]);
      o[1] = make_float4(dw[i][4], dw[i][5], dw[i][6], dw[i][7]);
    }
  if (WARP) {                                        // the warps' sums, in their order
    __syncthreads();
    for (int f = threadIdx.x; f < features; f += kBlock) {
      float v = 0.0f;
#pragma unroll
      for (int j = 0; j < kBlock / 32; ++j) v += share[j * features + f];
      p.partial[(size_t)blockIdx.x * features + f] = v;
    }
  }
}

// dW[f] = sum of the blocks' partial sums: 32 warps take every 32nd block each, 32 features to a block, then the first warp adds
// the warps' sums up.
constexpr int kSumWarps = 32;
__global__ void __launch_bounds__(kSumWarps * 32) norm_dw_kernel(const float* partial, int blocks, int features, float* dW) {
  __shared__ float part[kSumWarps][33];
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  const int lane = threadIdx.x & 31, f = (int)blockIdx.x * 32 + lane, j = threadIdx.x >> 5;
  float v = 0.0f;
  if (f < features) {
#pragma unroll 8
    for (int b = j; b < blocks; b += kSumWarps) v += ptx::ld_global(partial + (size_t)b * features + f);
  }
  part[j][lane] = v;
  __syncthreads();
  v = part[lane][j];                                 // warp j: the sums of feature j of the block's
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
  if (lane == 0 && (int)blockIdx.x * 32 + j < features) dW[blockIdx.x * 32 + j] = v;
}

// Threads of a row and vectors of each.
struct RowShape {
  int vpt, threads;                                  // threads 32: a warp a row
};
// `pairs`: threads that a row of two vectors a thread may have.
RowShape row_shape(int vecs, int pairs) {
  const int vpt = vecs <= 32 ? 1 : vecs <= 2 * pairs ? 2 : vecs <= 4 * kMaxThreads ? 4 : 8;
  return {vpt, ((vecs + vpt - 1) / vpt + 31) / 32 * 32};
}

// How the backward pass goes out: blocks, and stages of the ring.
struct Launch {
  int blocks, stages;
  size_t smem;
};
Launch backward_shape(const eqat_norm_desc& d, int sms) {
  constexpr int kBusy = 512, kMostStages = 3;          // threads of an SM that the kernel's registers leave room for
  const RowShape s = row_shape(d.features / 8, kMaxThreads);
  const int threads = s.threads == 32 ? kBlock : s.threads, rows_of_block = s.threads == 32 ? kBlock / 32 : 1;
  const int stage = threads * s.vpt * 3 * 16;          // of H, dY and dR
  int per_sm = kBusy / threads < 1 ? 1 : kBusy / threads, stages = kMostStages;
  // all stages, if need be with fewer blocks; fewer stages where they do not fit an SM
  while (per_sm > 1 && per_sm * stages * stage > kRingBytes) --per_sm;
  while (stages > 1 && stages * stage > kRingBytes) --stages;
  const int64_t need = (d.rows + rows_of_block - 1) / rows_of_block, most = (int64_t)sms * per_sm;
  Launch l{(int)(need < most ? need : most), stages, (size_t)stages * stage};
  const size_t share = (size_t)(kBlock / 32) * d.features * sizeof(float);
  if (s.threads == 32 && l.smem < share) l.smem = share;
  return l;
}

template <int VPT, bool WARP, bool LOOP, int CODES>
int launch_codes(const eqat_norm_desc& d, const NormFwd& p, const RowShape& s, int sms, cudaStream_t st) {
  constexpr int kRows = WARP ? kBlock / 32 : 1;
  const int threads = WARP ? kBlock : s.threads;
  const int64_t need = (d.rows + kRows - 1) / kRows, twice = (int64_t)sms * (2048 / threads);
  const dim3 grid((unsigned)(LOOP && need > twice ? twice : need)), block(threads);
  if constexpr (VPT % 2 == 0)
    if (p.vecs % 2 == 0)
      return aligned32(p.X, p.R, p.H, p.Y) ? launch_overlapped(norm_fwd_kernel<VPT, WARP, LOOP, CODES, true, true>, grid, block, 0, st, p)
                                           : launch_overlapped(norm_fwd_kernel<VPT, WARP, LOOP, CODES, true, false>, grid, block, 0, st, p);
  return launch_overlapped(norm_fwd_kernel<VPT, WARP, LOOP, CODES, false, false>, grid, block, 0, st, p);
}
template <int VPT, bool WARP, bool LOOP>
int launch_fwd(const eqat_norm_desc& d, const NormFwd& p, const RowShape& s, int sms, cudaStream_t st) {
  switch (d.codes) {
    case EQAT_CODES_INT8: return launch_codes<VPT, WARP, LOOP && !WARP, EQAT_CODES_INT8>(d, p, s, sms, st);
    case EQAT_CODES_E4M3: return launch_codes<VPT, WARP, LOOP && !WARP, EQAT_CODES_E4M3>(d, p, s, sms, st);
    default: return launch_codes<VPT, WARP, LOOP, EQAT_CODES_NONE>(d, p, s, sms, st);
  }
}
template <int VPT, bool WARP>
int launch_bwd(const NormBwd& p, const RowShape& s, const Launch& l, cudaStream_t st) {
  static SmemOptIn opt_in;
  if (l.smem > 40000 && !opt_in.ensure(norm_bwd_kernel<VPT, WARP>, kRingBytes)) return EQAT_ERR_CUDA;
  return launch_overlapped(norm_bwd_kernel<VPT, WARP>, dim3(l.blocks), dim3(WARP ? kBlock : s.threads), l.smem, st, p, l.stages);
}

}  // namespace

int launch_norm_fwd(const eqat_norm_desc& d, const eqat_bf16* X, const eqat_bf16* R, const eqat_bf16* W, eqat_bf16* H, eqat_bf16* Y,
                    void* codes, float* scales, cudaStream_t st) {
  const int sms = sm_count();
  if (sms <= 0) return EQAT_ERR_CUDA;
  const int vecs = d.features / 8;
  const int lanes = d.group > 0 && d.group <= 256 && d.group != d.features ? d.group / 8 : 0;
  const NormFwd p{X, R, W, H, Y, static_cast<uint8_t*>(codes), scales, (int)d.rows, vecs, d.eps, 1.0f / (float)d.features,
                  lanes, lanes > 0 ? log2_exact(lanes) : 0, lanes > 0 ? vecs / lanes : 1};
  // With codes blocks of up to 256 threads, several an SM, so that some load while others convert.
  const RowShape s = row_shape(vecs, d.codes == EQAT_CODES_NONE ? kMaxThreads : kMaxThreads / 2);
  if (s.threads == 32) return s.vpt == 1 ? launch_fwd<1, true, true>(d, p, s, sms, st) : launch_fwd<2, true, false>(d, p, s, sms, st);
  return s.threads <= kLoopThreads ? launch_fwd<2, false, true>(d, p, s, sms, st)          // (two vectors a thread)
         : s.vpt == 2              ? launch_fwd<2, false, false>(d, p, s, sms, st)
         : s.vpt == 4              ? launch_fwd<4, false, false>(d, p, s, sms, st)
                                   : launch_fwd<8, false, false>(d, p, s, sms, st);
}

size_t norm_workspace(const eqat_norm_desc& d, int sms) { return (size_t)backward_shape(d, sms).blocks * d.features * sizeof(float); }

int launch_norm_bwd(const eqat_norm_desc& d, const eqat_bf16* dY, const eqat_bf16* H, const eqat_bf16* W, const eqat_bf16* dR,
                    eqat_bf16* dX, float* dW, void* workspace, cudaStream_t st) {
  const int sms = sm_count();
  if (sms <= 0) return EQAT_ERR_CUDA;
  const int vecs = d.features / 8;
  const Launch l = backward_shape(d, sms);
  const NormBwd p{dY, H, W, dR, dX, dW != nullptr ? static_cast<float*>(workspace) : nullptr, (int)d.rows, vecs, d.eps,
                  1.0f / (float)d.features};
  const RowShape s = row_shape(vecs, kMaxThreads);
  const int rc = s.threads == 32 ? (s.vpt == 1 ? launch_bwd<1, true>(p, s, l, st) : launch_bwd<2, true>(p, s, l, st))
                 : s.vpt == 2    ? launch_bwd<2, false>(p, s, l, st)
                 : s.vpt == 4    ? launch_bwd<4, false>(p, s, l, st)
                                 : launch_bwd<8, false>(p, s, l, st);
  if (rc != EQAT_OK || dW == nullptr) return rc;
  return launch_overlapped(norm_dw_kernel, dim3((d.features + 31) / 32), dim3(kSumWarps * 32), 0, st, p.partial, l.blocks, d.features, dW);
}

}  // namespace eqat
