// Host launchers of what stands between a block's linears: norm, rotary positions, gated product (arguments already
// validated).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "eqat.h"

namespace eqat {

int launch_norm_fwd(const eqat_norm_desc& d, const eqat_bf16* X, const eqat_bf16* R, const eqat_bf16* W, eqat_bf16* H, eqat_bf16* Y,
                    void* codes, float* scales, cudaStream_t st);
// Scratch of the weight gradient's partial sums on a device of `sms` SMs.
size_t norm_workspace(const eqat_norm_desc& d, int sms);
int launch_norm_bwd(const eqat_norm_desc& d, const eqat_bf16* dY, const eqat_bf16* H, const eqat_bf16* W, const eqat_bf16* dR,
                    eqat_bf16* dX, float* dW, void* workspace, cudaStream_t st);

constexpr int kMaxRotaryHeads = 1 << 14, kMaxRotaryHeadDim = 512;       // of queries, and of keys
struct RotaryRows {
  const eqat_bf16 *q, *k;
  int64_t q_pitch, k_pitch;
  eqat_bf16 *q_out, *k_out;
  int64_t q_out_pitch, k_out_pitch;
  const uint64_t* turns;
  const int32_t *positions, *row_offsets, *lengths;
};
int launch_rotary(const eqat_rotary_desc& d, const RotaryRows& rows, bool backward, cudaStream_t st);

int launch_gated_fwd(const eqat_gated_desc& d, const eqat_bf16* G, int64_t g_pitch, const eqat_bf16* U, int64_t u_pitch,
                     eqat_bf16* H, cudaStream_t st);
int launch_gated_bwd(const eqat_gated_desc& d, const eqat_bf16* dH, const eqat_bf16* G, int64_t g_pitch, const eqat_bf16* U,
                     int64_t u_pitch, eqat_bf16* dG, int64_t dg_pitch, eqat_bf16* dU, int64_t du_pitch, cudaStream_t st);

}  // namespace eqat
