// The gated product H = act(G) * U of two projections that stand in memory, and its gradient.  (With packed weights the
// projections and their product are one kernel, in gemm.cu, gemv.cu or slim.cu, but for prompts on pairs of weight-row tiles, whose
// projections pass through memory and come here too.)
//
// Element-wise: 6 bytes an element forward and 10 backward, which HBM bounds: 4096 x 11008 forward 40.3 us (1.02 of a copy's
// bandwidth), 4095 x 13824 backward 82.0 to 86.8 us (1.00 to 1.05; one GPU and another).  A thread takes 16 elements, 32 bytes of
// each tensor, and is done: backward with a loop around it, which costs registers and so threads of an SM, 85.3 to 93.8 us where this
// took 82.0; blocks that stay, eight an SM, 42.7 and 93.8, sixteen 41.4 and 87.9.  Where rows or places are multiples of 16 bytes only, a
// thread takes 8 at a time and blocks stay (44.1 and 98.0; a block for every 2048 elements 49.4 and 99.6); it follows row and column by
// addition, not by a division for each piece.
#include "activation.cuh"
#include "between.cuh"
#include "common.cuh"
#include "pieces.cuh"
#include "ptx.cuh"

namespace eqat {
namespace {

constexpr int kThreads = 256;

struct GatedParams {
  const eqat_bf16 *dH, *G, *U;
  eqat_bf16 *H, *dG, *dU;
  int64_t g_pitch, u_pitch, dg_pitch, du_pitch;
  int64_t total;                                     // pieces in all
  int pieces;                                        // of a row
  int row_step, col_step;                            // what a step of the grid is
};

// N elements a thread and step; of 16 one step.
template <int ACT, bool BACKWARD, int N>
__global__ void __launch_bounds__(kThreads) gated_kernel(const GatedParams p) {
  ptx::grid_dependency_wait();
  const int64_t step = (int64_t)gridDim.x * kThreads;
  int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  int64_t row = i / p.pieces;
  int col = (int)(i - row * p.pieces);
  for (; i < p.total; i = N == 16 ? p.total : i + step, row += p.row_step, col += p.col_step) {
    if (col >= p.pieces) {
      col -= p.pieces;
      ++row;
    }
    const Piece<N> pg = load_piece<N>(p.G + row * p.g_pitch + (int64_t)col * N), pu = load_piece<N>(p.U + row * p.u_pitch + (int64_t)col * N);
    float g[N], u[N];
    if constexpr (BACKWARD) {
      const Piece<N> ph = load_piece<N>(p.dH + i * N);
      float h[N];
      unpack(pg, g);
      unpack(pu, u);
      unpack(ph, h);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        float a, slope;
        activate_with_slope<ACT>(g[e], a, slope);
        g[e] = h[e] * u[e] * slope;
        u[e] = h[e] * a;
      }
      store_piece(p.dG + row * p.dg_pitch + (int64_t)col * N, pack(g));
      store_piece(p.dU + row * p.du_pitch + (int64_t)col * N, pack(u));
    } else {
      unpack(pg, g);
      unpack(pu, u);
#pragma unroll
      for (int e = 0; e < N; ++e) g[e] = activate<ACT>(g[e]) * u[e];
      store_piece(p.H + i * N, pack(g));
    }
  }
  ptx::grid_dependents_launch();
}

template <bool BACKWARD, int N>
int launch_pieces(const eqat_gated_desc& d, GatedParams& p, int64_t most_blocks, cudaStream_t st) {
  p.pieces = d.features / N;
  p.total = d.rows * p.pieces;
  const int64_t need = (p.total + kThreads - 1) / kThreads;
  const dim3 grid((unsigned)(need < most_blocks ? need : most_blocks));
  const int64_t step = (int64_t)grid.x * kThreads;
  p.row_step = (int)(step / p.pieces);
  p.col_step = (int)(step % p.pieces);
  EQAT_WITH_ACTIVATION(d.activation, return launch_overlapped(gated_kernel<kAct, BACKWARD, N>, grid, dim3(kThreads), 0, st, p));
  return EQAT_ERR_UNSUPPORTED;
}

template <bool BACKWARD>
int launch_gated(const eqat_gated_desc& d, GatedParams p, cudaStream_t st) {
  const int sms = sm_count();
  if (sms <= 0) return EQAT_ERR_CUDA;
  const int64_t most = INT32_MAX;                    // blocks of a grid; of 4096 elements, more than any memory
  const bool wide = (d.features | p.g_pitch | p.u_pitch | p.dg_pitch | p.du_pitch) % 16 == 0 && aligned32(p.dH, p.G, p.U, p.H, p.dG, p.dU) &&
                    d.rows * (d.features / 16) <= most * kThreads;
  return wide ? launch_pieces<BACKWARD, 16>(d, p, most, st) : launch_pieces<BACKWARD, 8>(d, p, (int64_t)sms * 8, st);
}

}  // namespace

int launch_gated_fwd(const eqat_gated_desc& d, const eqat_bf16* G, int64_t g_pitch, const eqat_bf16* U, int64_t u_pitch,
                     eqat_bf16* H, cudaStream_t st) {
  GatedParams p{};
  p.G = G; p.U = U; p.H = H;
  p.g_pitch = g_pitch; p.u_pitch = u_pitch;
  return launch_gated<false>(d, p, st);
}

int launch_gated_bwd(const eqat_gated_desc& d, const eqat_bf16* dH, const eqat_bf16* G, int64_t g_pitch, const eqat_bf16* U,
                     int64_t u_pitch, eqat_bf16* dG, int64_t dg_pitch, eqat_bf16* dU, int64_t du_pitch, cudaStream_t st) {
  GatedParams p{};
  p.dH = dH; p.G = G; p.U = U; p.dG = dG; p.dU = dU;
  p.g_pitch = g_pitch; p.u_pitch = u_pitch; p.dg_pitch = dg_pitch; p.du_pitch = du_pitch;
  return launch_gated<true>(d, p, st);
}

}  // namespace eqat
