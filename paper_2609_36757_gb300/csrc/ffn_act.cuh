// The gated feed-forward's activations.
#pragma once

#include "fastvr_internal.h"

namespace fastvr {

// act(g) and its derivative in float32.  Where g is far below 0 the activations are
// small and 1 + tanh y or 1 + erf y cancels, so they are written as
// (1 + tanh y) / 2 = 1 / (1 + exp(-2 y)) and with the normal distribution's own tail,
// which keep their relative accuracy: some 30 units of 2^-24 and, for the
// exponential of a large argument, 2.4 times that argument, 2e-5 at most before the
// results leave float32's range.  Rounding them to bfloat16 is off by 2^-8.
__device__ __forceinline__ float logistic(float y) {
  return __fdividef(1.f, 1.f + __expf(-y));
}
// Phi(g), and e = exp(-g^2 / 2).  Phi(-a) = e P(1 / (1 + 0.265 a)) for a >= 0, the
// form of Abramowitz and Stegun's 7.1.26; P, of degree 7, is a fit of its own to the
// least relative error, 6.3e-7 for a up to 13.3 (where e leaves float32's range).
// erfcf is as accurate, but the feed-forward of 16320 tokens of 1536 to 4096 takes
// 250 us with it.
__device__ __forceinline__ float normal_cdf(float g, float* e) {
  *e = __expf(-0.5f * g * g);
  const float t = __fdividef(1.f, fmaf(0.265f, fabsf(g), 1.f));
  float q = fmaf(-0.067786485f, t, 0.19527118f);
  q = fmaf(q, t, -0.06636022f);
  q = fmaf(q, t, 0.14249139f);
  q = fmaf(q, t, 0.08294734f);
  q = fmaf(q, t, 0.10783663f);
  q = fmaf(q, t, 0.10559984f);
  q *= t * *e;
  return g < 0.f ? q : 1.f - q;
}
template <int kAct>
__device__ __forceinline__ float activation(float g) {
  if (kAct == kActSilu) return g * logistic(g);
  if (kAct == kActGelu) {
    float e;
    return g * normal_cdf(g, &e);
  }
  // 2 sqrt(2 / pi) and its product with 0.044715
  return g * logistic(g * (1.5957691f + 0.071354816f * g * g));
}
template <int kAct>
__device__ __forceinline__ float activation(float g, float* slope) {
  if (kAct == kActSilu) {
    const float s = logistic(g);
    *slope = s * (1.f + g * (1.f - s));
    return g * s;
  }
  if (kAct == kActGelu) {
    float e;
    const float c = normal_cdf(g, &e);
    *slope = c + g * 0.39894228f * e;
    return g * c;
  }
  // s (1 - s) is 0 past +-30, where the other factor could overflow
  const float s = logistic(g * (1.5957691f + 0.071354816f * g * g));
  const float b = fminf(fmaxf(g, -30.f), 30.f);
  *slope = s + b * s * (1.f - s) * (1.5957691f + 0.21406445f * b * b);
  return g * s;
}

// The kernel for few tokens (gated_ffn_rows.cu): its time grows with the tokens,
// the tiles' does not.  32 tokens: 1536 to 4096 12.0 us against 13.6, 2048 to 5632
// 16.2 against 15.5, 400 to 1000 3.7 against 5.6.
constexpr int kFfnMaxRows = 32;
inline bool ffn_few_rows(int64_t tokens) { return tokens <= kFfnMaxRows; }
cudaError_t launch_ffn_rows(const FfnArgs& a, cudaStream_t stream);

}  // namespace fastvr
