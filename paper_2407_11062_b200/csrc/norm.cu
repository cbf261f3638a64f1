// Root-mean-square norm of the residual stream, with the addition to it and an output in bf16 or 8 bits; its gradient.
//
//     h = bf16(x + r),  c = (mean(h^2) + eps)^(-1/2),  y = h w c
//     dx = dr + c (v - h c^2 mean(v h)),  v = dy w;     dw = sum over the rows of dy h c
//
// One pass: a row's threads keep it in registers between the sum over it and the output, so each tensor crosses HBM once: 8
// bytes an element forward with a residual (7 + 4/group with codes in place of y), 8 backward.  A thread owns the same
// columns of every row it meets, so w is read once a block and dw is added up in registers.
#include <cuda_fp8.h>

#include "between.cuh"
#include "common.cuh"
#include "ptx.cuh"

namespace eqat {
namespace {

constexpr int kBlock = 256;                          // threads of a block that gives each row to a warp
constexpr int kMaxThreads = 512;                     // of a block that shares a row
constexpr float kSmallGroup = 0x1p-110f;             // 127 / a and 448 / a are finite above

__device__ __forceinline__ void unpack(const uint4& v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ uint4 pack(const float (&f)[8]) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7]));
}

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

struct NormFwd {
  const eqat_bf16 *X, *R, *W;
  eqat_bf16 *H, *Y;
  uint8_t* codes;
  float* scales;
  int rows, vecs;                                    // vecs: 16-byte vectors of a row
  float eps, inverse_n;
  int lanes;                                         // codes: vectors of a group (4 .. 32 neighbouring lanes), or 0: the row
};

// VPT vectors of a row per thread.  A row belongs to a warp (WARP) or to the block.
template <int VPT, bool WARP, int CODES>
__global__ void __launch_bounds__(WARP ? kBlock : kMaxThreads) norm_fwd_kernel(const NormFwd p) {
  __shared__ Reduced red[2][32];
  const int lane = threadIdx.x & 31;
  const int at = WARP ? lane : (int)threadIdx.x, span = WARP ? 32 : (int)blockDim.x;
  const int step = (int)gridDim.x * (WARP ? kBlock / 32 : 1);
  constexpr float kTop = CODES == EQAT_CODES_INT8 ? 127.0f : 448.0f;
  ptx::grid_dependency_wait();
  uint4 w[VPT];
#pragma unroll
  for (int i = 0; i < VPT; ++i)
    w[i] = at + i * span < p.vecs ? ptx::ld_global(reinterpret_cast<const uint4*>(p.W) + at + i * span) : make_uint4(0u, 0u, 0u, 0u);
  int turn = 0;
  for (int row = WARP ? (int)blockIdx.x * (kBlock / 32) + (int)(threadIdx.x >> 5) : (int)blockIdx.x; row < p.rows; row += step, ++turn) {
    if (row >= p.rows - step) ptx::grid_dependents_launch();
    const size_t base = (size_t)row * p.vecs + at;
    uint4 x[VPT], r[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      x[i] = r[i] = make_uint4(0u, 0u, 0u, 0u);
      if (at + i * span < p.vecs) {
        x[i] = ptx::ld_global_once(reinterpret_cast<const uint4*>(p.X) + base + i * span);
        if (p.R != nullptr) r[i] = ptx::ld_global_once(reinterpret_cast<const uint4*>(p.R) + base + i * span);
      }
    }
    Reduced s{0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float h[8], g[8];
      unpack(x[i], h);
      if (p.R != nullptr) {
        unpack(r[i], g);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] += g[e];
        x[i] = pack(h);
        if (p.H != nullptr && at + i * span < p.vecs) reinterpret_cast<uint4*>(p.H)[base + i * span] = x[i];
        unpack(x[i], h);
      } else if (p.H != nullptr && p.H != p.X && at + i * span < p.vecs) {
        reinterpret_cast<uint4*>(p.H)[base + i * span] = x[i];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) s.a = fmaf(h[e], h[e], s.a);
      if (CODES != EQAT_CODES_NONE && p.lanes == 0) {
        unpack(w[i], g);
#pragma unroll
        for (int e = 0; e < 8; ++e) s.most = fmaxf(s.most, fabsf(h[e] * g[e]));
      }
    }
    s = reduce_row<WARP>(s, red, turn);
    const float c = rsqrtf(fmaf(s.a, p.inverse_n, p.eps));
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const bool live = at + i * span < p.vecs;
      float h[8], g[8];
      unpack(x[i], h);
      unpack(w[i], g);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[e] *= g[e];
      if constexpr (CODES == EQAT_CODES_NONE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] *= c;
        if (live) reinterpret_cast<uint4*>(p.Y)[base + i * span] = pack(h);
      } else {
        float most = s.most;
        if (p.lanes != 0) {
          most = 0.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(h[e]));
          for (int d = 1; d < p.lanes; d <<= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, d));
        }
        if (most < kSmallGroup) most = 0.0f;
        const float up = most > 0.0f ? __fdiv_rn(kTop, most) : 0.0f;
        const float scale = most * c * (1.0f / kTop);
        uint32_t q[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float t = __fmul_rn(h[e], up);
          if constexpr (CODES == EQAT_CODES_INT8) {
            const int k = min(max(__float2int_rn(t), -127), 127);
            q[e] = (uint32_t)k & 0xFFu;
            h[e] = (float)k * scale;
          } else {
            q[e] = __nv_cvt_float_to_fp8(t, __NV_SATFINITE, __NV_E4M3);
            h[e] = __half2float(__nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)q[e], __NV_E4M3)) * scale;
          }
        }
        if (live) {
          reinterpret_cast<uint2*>(p.codes)[base + i * span] = make_uint2(q[0] | (q[1] << 8) | (q[2] << 16) | (q[3] << 24),
                                                                           q[4] | (q[5] << 8) | (q[6] << 16) | (q[7] << 24));
          if (p.Y != nullptr) reinterpret_cast<uint4*>(p.Y)[base + i * span] = pack(h);
          if (p.lanes == 0) {
            if (at == 0 && i == 0) p.scales[row] = scale;
          } else if ((lane & (p.lanes - 1)) == 0) {
            p.scales[(size_t)row * (p.vecs / p.lanes) + (at + i * span) / p.lanes] = scale;
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

template <int VPT, bool WARP>
__global__ void __launch_bounds__(WARP ? kBlock : kMaxThreads) norm_bwd_kernel(const NormBwd p) {
  __shared__ Reduced red[2][32];
  extern __shared__ float share[];                   // WARP: [warps][features]
  const int lane = threadIdx.x & 31;
  const int at = WARP ? lane : (int)threadIdx.x, span = WARP ? 32 : (int)blockDim.x;
  const int step = (int)gridDim.x * (WARP ? kBlock / 32 : 1);
  ptx::grid_dependency_wait();
  uint4 w[VPT];
  float dw[VPT][8];
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
    w[i] = at + i * span < p.vecs ? ptx::ld_global(reinterpret_cast<const uint4*>(p.W) + at + i * span) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[i][e] = 0.0f;
  }
  int turn = 0;
  for (int row = WARP ? (int)blockIdx.x * (kBlock / 32) + (int)(threadIdx.x >> 5) : (int)blockIdx.x; row < p.rows; row += step, ++turn) {
    if (row >= p.rows - step) ptx::grid_dependents_launch();
    const size_t base = (size_t)row * p.vecs + at;
    uint4 h4[VPT], y4[VPT], r4[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      h4[i] = y4[i] = r4[i] = make_uint4(0u, 0u, 0u, 0u);
      if (at + i * span < p.vecs) {
        h4[i] = ptx::ld_global_once(reinterpret_cast<const uint4*>(p.H) + base + i * span);
        y4[i] = ptx::ld_global_once(reinterpret_cast<const uint4*>(p.dY) + base + i * span);
        if (p.dR != nullptr) r4[i] = ptx::ld_global_once(reinterpret_cast<const uint4*>(p.dR) + base + i * span);
      }
    }
    Reduced s{0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float h[8], y[8], g[8];
      unpack(h4[i], h);
      unpack(y4[i], y);
      unpack(w[i], g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s.a = fmaf(h[e], h[e], s.a);
        s.b = fmaf(y[e] * g[e], h[e], s.b);
      }
    }
    s = reduce_row<WARP>(s, red, turn);
    const float c = rsqrtf(fmaf(s.a, p.inverse_n, p.eps));
    const float k = c * c * (s.b * p.inverse_n);
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      float h[8], y[8], g[8], r[8];
      unpack(h4[i], h);
      unpack(y4[i], y);
      unpack(w[i], g);
      unpack(r4[i], r);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        dw[i][e] = fmaf(y[e], h[e] * c, dw[i][e]);
        r[e] = fmaf(c, fmaf(-h[e], k, y[e] * g[e]), r[e]);
      }
      if (at + i * span < p.vecs) reinterpret_cast<uint4*>(p.dX)[base + i * span] = pack(r);
    }
  }
  if (p.partial == nullptr) return;
  const int features = p.vecs * 8;
  float* out = p.partial + (size_t)blockIdx.x * features;
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

// dW[f] = sum of the blocks' partial sums: eight threads take an eighth of the blocks each, 32 features to a block.
__global__ void __launch_bounds__(256) norm_dw_kernel(const float* partial, int blocks, int features, float* dW) {
  __shared__ float part[8][33];
  ptx::grid_dependency_wait();
  ptx::grid_dependents_launch();
  const int f = (int)blockIdx.x * 32 + (threadIdx.x & 31), j = threadIdx.x >> 5;
  float v = 0.0f;
  if (f < features)
    for (int b = j; b < blocks; b += 8) v += ptx::ld_global(partial + (size_t)b * features + f);
  part[j][threadIdx.x & 31] = v;
  __syncthreads();
  if (j == 0 && f < features) {
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) v += part[i][threadIdx.x];
    dW[f] = v;
  }
}

// Threads of a row and vectors of each.
struct RowShape {
  int vpt, threads;                                  // threads 32: a warp a row
};
RowShape row_shape(int vecs) {
  const int vpt = vecs <= 32 ? 1 : vecs <= 2 * kMaxThreads ? 2 : vecs <= 4 * kMaxThreads ? 4 : 8;
  return {vpt, ((vecs + vpt - 1) / vpt + 31) / 32 * 32};
}

int blocks_of(int64_t rows, int threads, int sms) {
  const int64_t need = threads == 32 ? (rows + kBlock / 32 - 1) / (kBlock / 32) : rows;
  const int64_t most = (int64_t)sms * (threads == 32 ? 2048 / kBlock : 2048 / threads);
  return (int)(need < most ? need : most);
}

// The backward pass holds w's sums and three tensors in registers.
int backward_blocks(const eqat_norm_desc& d, int sms) {
  const RowShape s = row_shape(d.features / 8);
  const int64_t need = s.threads == 32 ? (d.rows + kBlock / 32 - 1) / (kBlock / 32) : d.rows;
  const int64_t most = (int64_t)sms * (s.threads == 32 ? 4 : (s.threads <= 512 ? 1024 / s.threads : 1));
  return (int)(need < most ? need : most);
}

template <int VPT, bool WARP>
int launch_fwd(const eqat_norm_desc& d, const NormFwd& p, int threads, int sms, cudaStream_t st) {
  const dim3 grid(blocks_of(d.rows, threads, sms)), block(WARP ? kBlock : threads);
  switch (d.codes) {
    case EQAT_CODES_INT8: return launch_overlapped(norm_fwd_kernel<VPT, WARP, EQAT_CODES_INT8>, grid, block, 0, st, p);
    case EQAT_CODES_E4M3: return launch_overlapped(norm_fwd_kernel<VPT, WARP, EQAT_CODES_E4M3>, grid, block, 0, st, p);
    default: return launch_overlapped(norm_fwd_kernel<VPT, WARP, EQAT_CODES_NONE>, grid, block, 0, st, p);
  }
}

}  // namespace

int launch_norm_fwd(const eqat_norm_desc& d, const eqat_bf16* X, const eqat_bf16* R, const eqat_bf16* W, eqat_bf16* H, eqat_bf16* Y,
                    void* codes, float* scales, cudaStream_t st) {
  const int sms = sm_count();
  if (sms <= 0) return EQAT_ERR_CUDA;
  const int vecs = d.features / 8;
  const NormFwd p{X, R, W, H, Y, static_cast<uint8_t*>(codes), scales, (int)d.rows, vecs, d.eps, 1.0f / (float)d.features,
                  d.group > 0 && d.group <= 256 && d.group != d.features ? d.group / 8 : 0};
  const RowShape s = row_shape(vecs);
  if (s.threads == 32) return s.vpt == 1 ? launch_fwd<1, true>(d, p, 32, sms, st) : launch_fwd<2, true>(d, p, 32, sms, st);
  return s.vpt == 2   ? launch_fwd<2, false>(d, p, s.threads, sms, st)
         : s.vpt == 4 ? launch_fwd<4, false>(d, p, s.threads, sms, st)
                      : launch_fwd<8, false>(d, p, s.threads, sms, st);
}

size_t norm_workspace(const eqat_norm_desc& d, int sms) { return (size_t)backward_blocks(d, sms) * d.features * sizeof(float); }

int launch_norm_bwd(const eqat_norm_desc& d, const eqat_bf16* dY, const eqat_bf16* H, const eqat_bf16* W, const eqat_bf16* dR,
                    eqat_bf16* dX, float* dW, void* workspace, cudaStream_t st) {
  const int sms = sm_count();
  if (sms <= 0) return EQAT_ERR_CUDA;
  const int vecs = d.features / 8, blocks = backward_blocks(d, sms);
  const NormBwd p{dY, H, W, dR, dX, dW != nullptr ? static_cast<float*>(workspace) : nullptr, (int)d.rows, vecs, d.eps,
                  1.0f / (float)d.features};
  const RowShape s = row_shape(vecs);
  const dim3 grid(blocks);
  const size_t share = (size_t)(kBlock / 32) * d.features * sizeof(float);
  int rc;
  if (s.threads == 32) rc = s.vpt == 1 ? launch_overlapped(norm_bwd_kernel<1, true>, grid, dim3(kBlock), share, st, p)
                                       : launch_overlapped(norm_bwd_kernel<2, true>, grid, dim3(kBlock), share, st, p);
  else rc = s.vpt == 2   ? launch_overlapped(norm_bwd_kernel<2, false>, grid, dim3(s.threads), 0, st, p)
            : s.vpt == 4 ? launch_overlapped(norm_bwd_kernel<4, false>, grid, dim3(s.threads), 0, st, p)
                         : launch_overlapped(norm_bwd_kernel<8, false>, grid, dim3(s.threads), 0, st, p);
  if (rc != EQAT_OK || dW == nullptr) return rc;
  return launch_overlapped(norm_dw_kernel, dim3((d.features + 31) / 32), dim3(256), 0, st, p.partial, blocks, d.features, dW);
}

}  // namespace eqat
