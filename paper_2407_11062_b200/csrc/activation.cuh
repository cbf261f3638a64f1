// Activations of the gated product and their derivatives, in binary32.
//
// The sigmoid s(x) = 1 / (1 + e^-x) carries two of the three: g s(g), and g s(2z), which is the form with tanh (0.5 (1 + tanh
// z) = s(2z), so nothing cancels for large negative g).  One exponential and one reciprocal, both to 2 ulp and with
// denormals as zeros: where e^-x leaves the range the value is below 2^-110 of anything that bf16 rounds.  A bf16 result
// needs no more; what it must not have is an error that grows where the value is small, which tanh.approx would bring.
#pragma once
#include "common.cuh"

namespace eqat {

__device__ __forceinline__ float sigmoid(float x) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-1.4426950408889634f * x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return r;
}

constexpr float kTwoZ = 1.5957691216057308f;           // 2 (2/pi)^(1/2)
constexpr float kCubic = 0.044715f;

// -inf has the limit 0; a NaN stays one through the other factor.
__device__ __forceinline__ float above_minus_inf(float g) { return fmaxf(g, -3.0e38f); }

template <int ACT>
__device__ __forceinline__ float activate(float g) {
  if constexpr (ACT == EQAT_ACT_SILU) return above_minus_inf(g) * sigmoid(g);
  else if constexpr (ACT == EQAT_ACT_GELU) return above_minus_inf(g) * (0.5f * erfcf(-0.7071067811865476f * g));
  else return above_minus_inf(g) * sigmoid(kTwoZ * fmaf(kCubic * g * g, g, g));
}

// act(g) and act'(g).  Beyond |g| = 128 the second terms of the derivatives are 0 (s(g) below 2^-126, or 1 - s(g) below 2^-24),
// and the limit keeps infinities out of them.
template <int ACT>
__device__ __forceinline__ void activate_with_slope(float g, float& a, float& slope) {
  const float c = fminf(fmaxf(g, -128.0f), 128.0f);
  if constexpr (ACT == EQAT_ACT_SILU) {
    const float s = sigmoid(g);
    a = above_minus_inf(g) * s;
    slope = s * fmaf(c, 1.0f - s, 1.0f);
  } else if constexpr (ACT == EQAT_ACT_GELU) {
    const float phi = 0.5f * erfcf(-0.7071067811865476f * g);
    a = above_minus_inf(g) * phi;
    float e;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(-0.7213475204444817f * c * c));       // e^(-g^2/2)
    slope = fmaf(0.3989422804014327f * c, e, phi);
  } else {
    const float s = sigmoid(kTwoZ * fmaf(kCubic * g * g, g, g));
    a = above_minus_inf(g) * s;
    slope = s * fmaf(c * (1.0f - s), kTwoZ * fmaf(3.0f * kCubic * c, c, 1.0f), 1.0f);
  }
}

// Runs the statements with kAct, a constant, as the activation that `act` says at run time.
#define EQAT_WITH_ACTIVATION(act, ...)                                                     \
  do {                                                                                     \
    if ((act) == EQAT_ACT_SILU) { constexpr int kAct = EQAT_ACT_SILU; __VA_ARGS__; }       \
    else if ((act) == EQAT_ACT_GELU) { constexpr int kAct = EQAT_ACT_GELU; __VA_ARGS__; }  \
    else { constexpr int kAct = EQAT_ACT_GELU_TANH; __VA_ARGS__; }                         \
  } while (0)

}  // namespace eqat
