// The gated product H = act(G) * U of two projections that stand in memory, and its gradient.  (With packed weights the
// projections and their product are one kernel: gemm.cu, gemv.cu.)
//
// Element-wise: 6 bytes an element forward and 10 backward, which HBM bounds: 4096 x 11008 forward 44.6 us (0.93 of a copy's
// bandwidth), 4095 x 13824 backward 98.9 us (0.87).  A thread takes 8 elements at a time; blocks stay (a block for every 2048
// elements: 49.4 and 99.6 us), and a thread follows row and column by addition, not by a division for each vector.
#include "activation.cuh"
#include "between.cuh"
#include "common.cuh"
#include "ptx.cuh"

namespace eqat {
namespace {

constexpr int kThreads = 256;

struct GatedParams {
  const eqat_bf16 *dH, *G, *U;
  eqat_bf16 *H, *dG, *dU;
  int64_t g_pitch, u_pitch, dg_pitch, du_pitch;      // in vectors of 8
  int64_t total;                                     // vectors in all
  int vecs;                                          // of a row
  int row_step, col_step;                            // what a step of the grid is
};

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

template <int ACT, bool BACKWARD>
__global__ void __launch_bounds__(kThreads) gated_kernel(const GatedParams p) {
  ptx::grid_dependency_wait();
  const int64_t step = (int64_t)gridDim.x * kThreads;
  int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  int64_t row = i / p.vecs;
  int col = (int)(i - row * p.vecs);
  for (; i < p.total; i += step, row += p.row_step, col += p.col_step) {
    if (col >= p.vecs) {
      col -= p.vecs;
      ++row;
    }
    float g[8], u[8];
    unpack(ptx::ld_global_once(reinterpret_cast<const uint4*>(p.G) + row * p.g_pitch + col), g);
    unpack(ptx::ld_global_once(reinterpret_cast<const uint4*>(p.U) + row * p.u_pitch + col), u);
    if constexpr (BACKWARD) {
      float h[8];
      unpack(ptx::ld_global_once(reinterpret_cast<const uint4*>(p.dH) + i), h);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float a, slope;
        activate_with_slope<ACT>(g[e], a, slope);
        g[e] = h[e] * u[e] * slope;
        u[e] = h[e] * a;
      }
      reinterpret_cast<uint4*>(p.dG)[row * p.dg_pitch + col] = pack(g);
      reinterpret_cast<uint4*>(p.dU)[row * p.du_pitch + col] = pack(u);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = activate<ACT>(g[e]) * u[e];
      reinterpret_cast<uint4*>(p.H)[i] = pack(g);
    }
  }
  ptx::grid_dependents_launch();
}

template <bool BACKWARD>
int launch_gated(const eqat_gated_desc& d, GatedParams p, cudaStream_t st) {
  const int sms = sm_count();
  if (sms <= 0) return EQAT_ERR_CUDA;
  p.vecs = d.features / 8;
  p.total = d.rows * p.vecs;
  const int64_t need = (p.total + kThreads - 1) / kThreads, most = (int64_t)sms * 8;
  const dim3 grid((unsigned)(need < most ? need : most));
  const int step = (int)grid.x * kThreads;
  p.row_step = step / p.vecs;
  p.col_step = step % p.vecs;
  EQAT_WITH_ACTIVATION(d.activation, return launch_overlapped(gated_kernel<kAct, BACKWARD>, grid, dim3(kThreads), 0, st, p));
  return EQAT_ERR_UNSUPPORTED;
}

}  // namespace

int launch_gated_fwd(const eqat_gated_desc& d, const eqat_bf16* G, int64_t g_pitch, const eqat_bf16* U, int64_t u_pitch,
                     eqat_bf16* H, cudaStream_t st) {
  GatedParams p{};
  p.G = G; p.U = U; p.H = H;
  p.g_pitch = g_pitch / 8; p.u_pitch = u_pitch / 8;
  return launch_gated<false>(d, p, st);
}

int launch_gated_bwd(const eqat_gated_desc& d, const eqat_bf16* dH, const eqat_bf16* G, int64_t g_pitch, const eqat_bf16* U,
                     int64_t u_pitch, eqat_bf16* dG, int64_t dg_pitch, eqat_bf16* dU, int64_t du_pitch, cudaStream_t st) {
  GatedParams p{};
  p.dH = dH; p.G = G; p.U = U; p.dG = dG; p.dU = dU;
  p.g_pitch = g_pitch / 8; p.u_pitch = u_pitch / 8; p.dg_pitch = dg_pitch / 8; p.du_pitch = du_pitch / 8;
  return launch_gated<true>(d, p, st);
}

}  // namespace eqat
