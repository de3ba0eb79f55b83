// Cross attention backward: one warp per query row for dq, one warp per key
// for dk and dv (over the rows of the heads that share it, in order).
#include <cuda_bf16.h>
#include <math.h>

#include "fastvr_internal.h"

namespace fastvr {
namespace {

__device__ __forceinline__ float warp_sum(float s) {
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
  return s;
}

template <int D>
__global__ void __launch_bounds__(256) cross_dq_kernel(CrossBwdArgs a) {
  constexpr int E = D / 32;
  const CrossArgs& p = a.f;
  const int64_t i = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / 32;
  const int lane = threadIdx.x % 32;
  if (i >= (int64_t)p.batch * p.heads * p.q_tokens) return;
  const int t = (int)(i % p.q_tokens);
  const int h = (int)(i / p.q_tokens % p.heads);
  const int b = (int)(i / p.q_tokens / p.heads);
  const int hk = h / (p.heads / p.kv_heads);
  const int n = p.kv_len ? min(max(p.kv_len[b], 0), p.kv_tokens) : p.kv_tokens;
  const uint16_t* q = p.q + b * p.q_str.batch + t * p.q_str.token + h * p.q_str.head;
  const uint16_t* o = p.o + b * p.o_str.batch + t * p.o_str.token + h * p.o_str.head;
  const uint16_t* g = a.dout + b * a.dout_str.batch + t * a.dout_str.token + h * a.dout_str.head;
  const uint16_t* k = p.k + b * p.k_str.batch + hk * p.k_str.head;
  const uint16_t* v = p.v + b * p.v_str.batch + hk * p.v_str.head;
  float qf[E], gf[E], acc[E], dl = 0.f;
  for (int e = 0; e < E; ++e) {
    qf[e] = bf16_lo(q[lane * E + e]);
    gf[e] = bf16_lo(g[lane * E + e]);
    dl += gf[e] * bf16_lo(o[lane * E + e]);
    acc[e] = 0.f;
  }
  dl = warp_sum(dl);
  if (lane == 0) a.scratch[i] = dl;
  const float lse = p.lse[i];
  for (int j = 0; j < n; ++j) {
    float s = 0.f, dp = 0.f, kf[E];
    for (int e = 0; e < E; ++e) {
      kf[e] = bf16_lo(k[j * p.k_str.token + lane * E + e]);
      s += qf[e] * kf[e];
      dp += gf[e] * bf16_lo(v[j * p.v_str.token + lane * E + e]);
    }
    s = warp_sum(s) * p.scale;
    const float ds = expf(s - lse) * (warp_sum(dp) - dl) * p.scale;
    for (int e = 0; e < E; ++e) acc[e] += ds * kf[e];
  }
  uint16_t* dq = a.dq + b * a.dq_str.batch + t * a.dq_str.token + h * a.dq_str.head;
  for (int e = 0; e < E; ++e)
    dq[lane * E + e] = __bfloat16_as_ushort(__float2bfloat16_rn(acc[e]));
}

template <int D>
__global__ void __launch_bounds__(256) cross_dkdv_kernel(CrossBwdArgs a) {
  constexpr int E = D / 32;
  const CrossArgs& p = a.f;
  const int64_t i = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / 32;
  const int lane = threadIdx.x % 32;
  if (i >= (int64_t)p.batch * p.kv_heads * p.kv_tokens) return;
  const int j = (int)(i % p.kv_tokens);
  const int hk = (int)(i / p.kv_tokens % p.kv_heads);
  const int b = (int)(i / p.kv_tokens / p.kv_heads);
  const int group = p.heads / p.kv_heads;
  const int n = p.kv_len ? min(max(p.kv_len[b], 0), p.kv_tokens) : p.kv_tokens;
  const uint16_t* k = p.k + b * p.k_str.batch + j * p.k_str.token + hk * p.k_str.head;
  const uint16_t* v = p.v + b * p.v_str.batch + j * p.v_str.token + hk * p.v_str.head;
  float kf[E], vf[E], dk[E], dv[E];
  for (int e = 0; e < E; ++e) {
    kf[e] = bf16_lo(k[lane * E + e]);
    vf[e] = bf16_lo(v[lane * E + e]);
    dk[e] = dv[e] = 0.f;
  }
  for (int h = hk * group; j < n && h < (hk + 1) * group; ++h)
    for (int t = 0; t < p.q_tokens; ++t) {
      const uint16_t* q = p.q + b * p.q_str.batch + t * p.q_str.token + h * p.q_str.head;
      const uint16_t* g = a.dout + b * a.dout_str.batch + t * a.dout_str.token + h * a.dout_str.head;
      const int64_t r = ((int64_t)b * p.heads + h) * p.q_tokens + t;
      float s = 0.f, dp = 0.f, qf[E], gf[E];
      for (int e = 0; e < E; ++e) {
        qf[e] = bf16_lo(q[lane * E + e]);
        gf[e] = bf16_lo(g[lane * E + e]);
        s += qf[e] * kf[e];
        dp += gf[e] * vf[e];
      }
      const float w = expf(warp_sum(s) * p.scale - p.lse[r]);
      const float ds = w * (warp_sum(dp) - a.scratch[r]) * p.scale;
      for (int e = 0; e < E; ++e) {
        dk[e] += ds * qf[e];
        dv[e] += w * gf[e];
      }
    }
  uint16_t* ok = a.dk + b * a.dk_str.batch + j * a.dk_str.token + hk * a.dk_str.head;
  uint16_t* ov = a.dv + b * a.dv_str.batch + j * a.dv_str.token + hk * a.dv_str.head;
  for (int e = 0; e < E; ++e) {
    ok[lane * E + e] = __bfloat16_as_ushort(__float2bfloat16_rn(dk[e]));
    ov[lane * E + e] = __bfloat16_as_ushort(__float2bfloat16_rn(dv[e]));
  }
}

}  // namespace

size_t cross_bwd_scratch_floats(int32_t batch, int32_t heads, int32_t,
                                int32_t, int32_t q_tokens, int32_t) {
  return (size_t)batch * heads * q_tokens;
}

cudaError_t launch_cross_attn_bwd(const CrossBwdArgs& a, cudaStream_t stream) {
  const int64_t rows = (int64_t)a.f.batch * a.f.heads * a.f.q_tokens;
  const int64_t keys = (int64_t)a.f.batch * a.f.kv_heads * a.f.kv_tokens;
  const unsigned gq = (unsigned)((rows + 7) / 8), gk = (unsigned)((keys + 7) / 8);
  if (a.f.head_dim == 64) {
    cross_dq_kernel<64><<<gq, 256, 0, stream>>>(a);
    cross_dkdv_kernel<64><<<gk, 256, 0, stream>>>(a);
  } else {
    cross_dq_kernel<128><<<gq, 256, 0, stream>>>(a);
    cross_dkdv_kernel<128><<<gk, 256, 0, stream>>>(a);
  }
  return cudaGetLastError();
}

}  // namespace fastvr
