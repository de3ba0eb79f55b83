// The gated feed-forward's activations.
#pragma once

#include "fastvr_internal.h"

namespace fastvr {

// act(g) and its derivative in float32.  tanh's form is written with the
// logistic function, (1 + tanh y) / 2 = 1 / (1 + exp(-2 y)), which keeps its
// relative accuracy where g is far below 0.  The approximate exponential and
// reciprocal are off by a few units of 2^-24 (more for an exponential's large
// argument, where the logistic function is 0 or 1), far below bfloat16's 2^-9.
__device__ __forceinline__ float logistic(float y) {
  return __fdividef(1.f, 1.f + __expf(-y));
}
template <int kAct>
__device__ __forceinline__ float activation(float g) {
  if (kAct == kActSilu) return g * logistic(g);
  if (kAct == kActGelu) return 0.5f * g * (1.f + erff(g * 0.70710678f));
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
    const float c = 0.5f * (1.f + erff(g * 0.70710678f));
    *slope = c + g * 0.39894228f * __expf(-0.5f * g * g);
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
