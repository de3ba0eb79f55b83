// Cross attention forward: one warp per query row, online softmax over the
// keys (lanes hold the head's elements).
#include <cuda_bf16.h>
#include <math.h>

#include "fastvr_internal.h"

namespace fastvr {
namespace {

template <int D>
__global__ void __launch_bounds__(256) cross_rows_kernel(CrossArgs p) {
  constexpr int E = D / 32;
  const int64_t i = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / 32;
  const int lane = threadIdx.x % 32;
  const int64_t rows = (int64_t)p.batch * p.heads * p.q_tokens;
  if (i >= rows) return;
  const int t = (int)(i % p.q_tokens);
  const int h = (int)(i / p.q_tokens % p.heads);
  const int b = (int)(i / p.q_tokens / p.heads);
  const int hk = h / (p.heads / p.kv_heads);
  const int n = p.kv_len ? min(max(p.kv_len[b], 0), p.kv_tokens) : p.kv_tokens;
  const uint16_t* q = p.q + b * p.q_str.batch + t * p.q_str.token + h * p.q_str.head;
  const uint16_t* k = p.k + b * p.k_str.batch + hk * p.k_str.head;
  const uint16_t* v = p.v + b * p.v_str.batch + hk * p.v_str.head;
  float qf[E], acc[E];
  for (int e = 0; e < E; ++e) {
    qf[e] = bf16_lo(q[lane * E + e]);
    acc[e] = 0.f;
  }
  float m = -INFINITY, l = 0.f;
  for (int j = 0; j < n; ++j) {
    float s = 0.f;
    for (int e = 0; e < E; ++e)
      s += qf[e] * bf16_lo(k[j * p.k_str.token + lane * E + e]);
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    s *= p.scale;
    const float mn = fmaxf(m, s), a = expf(m - mn), w = expf(s - mn);
    l = l * a + w;
    for (int e = 0; e < E; ++e)
      acc[e] = acc[e] * a + w * bf16_lo(v[j * p.v_str.token + lane * E + e]);
    m = mn;
  }
  uint16_t* o = p.o + b * p.o_str.batch + t * p.o_str.token + h * p.o_str.head;
  for (int e = 0; e < E; ++e)
    o[lane * E + e] =
        __bfloat16_as_ushort(__float2bfloat16_rn(n ? acc[e] / l : 0.f));
  if (p.lse && lane == 0)
    p.lse[((int64_t)b * p.heads + h) * p.q_tokens + t] =
        n ? m + logf(l) : -INFINITY;
}

}  // namespace

cudaError_t launch_cross_attn(const CrossArgs& a, cudaStream_t stream) {
  const int64_t rows = (int64_t)a.batch * a.heads * a.q_tokens;
  const unsigned grid = (unsigned)((rows + 7) / 8);
  if (a.head_dim == 64)
    cross_rows_kernel<64><<<grid, 256, 0, stream>>>(a);
  else
    cross_rows_kernel<128><<<grid, 256, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace fastvr
