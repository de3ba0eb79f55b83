// Rotary positions on the queries and keys of a block, and their transpose
// (the gradient): for every pair (a, b) of a head,
//   a' = m (a cos x - b sin x),  b' = m (b cos x + a sin x),  x = p theta.
//
// Bound by memory: every element is read once and written once (4 bytes per
// bfloat16 element).  The sines depend on the token alone, so a CTA takes a
// few whole tokens, forms cos and sin of their pairs once in shared memory
// and applies them to all heads of q and of k in one pass of 16-byte
// accesses.
//
// The angle is reduced exactly before any floating-point step: theta / 2 pi
// is held as a 64-bit fixed-point fraction F of a turn (host, rounded once),
// p F modulo 2^64 is the turn's fraction for every int32 position, and its
// top 32 bits go to sincospi.  A position of 10^6 is as accurate as 1.
#include <cuda_bf16.h>

#include "fastvr_internal.h"

namespace fastvr {
namespace {

constexpr int kThreads = 256;
constexpr int kSmemPairs = 2048;  // (token, pair) entries per CTA: 16 KB
constexpr int kUnroll = 4;

// Division of 32-bit numbers below 2^31 by a divisor fixed at launch.
struct FastDiv {
  uint32_t d, mul, shift;
};
FastDiv make_div(uint32_t d) {
  FastDiv f;
  f.d = d;
  f.shift = 0;
  while ((1ull << f.shift) < d) ++f.shift;
  // mul = ceil(2^(31 + shift) / d) < 2^32; exact for numbers below 2^31
  f.mul = (uint32_t)(((1ull << (31 + f.shift)) + d - 1) / d);
  return f;
}
__device__ __forceinline__ uint32_t fast_div(uint32_t n, const FastDiv& f) {
  return (uint32_t)(((uint64_t)n * f.mul) >> (31 + f.shift));
}

template <typename T, int V>
struct alignas(sizeof(T) * V < 16 ? sizeof(T) * V : 16) Vec {
  T e[V];
};

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) {
  return __bfloat162float(x);
}
__device__ __forceinline__ void from_f(float& d, float x) { d = x; }
__device__ __forceinline__ void from_f(__nv_bfloat16& d, float x) {
  d = __float2bfloat16_rn(x);
}

struct Params {
  const void *q, *k;
  void *q_out, *k_out;
  const int32_t* pos;
  int64_t pos_batch;
  Strides q_str, k_str, q_out_str, k_out_str;
  int64_t rows;               // batch * tokens
  int32_t tokens, axes, pairs, head_dim;
  int32_t tile;               // tokens of a CTA
  int32_t axis_end[3];        // first pair past each axis
  FastDiv by_tokens, by_pairs, by_items, by_heads;
  int32_t items;              // vector items of a head
  int32_t heads, all_heads;   // q heads, q and k heads
  float mag, sign;
  uint64_t turn[kRotaryMaxPairs];  // theta / 2 pi in 2^-64 turns
};

// One head's item: kHalf: the vectors of V elements at i V and rot/2 + i V
// (one per pair of the V), then the pass-through vectors; interleaved: the
// vector at i V, V / 2 pairs.
template <typename T, bool kHalf, int V>
__global__ void __launch_bounds__(kThreads)
rotary_kernel(const __grid_constant__ Params p) {
  __shared__ float2 cs[kSmemPairs];
  pdl_trigger();
  const int64_t row0 = (int64_t)blockIdx.x * p.tile;
  const int n_rows = (int)min((int64_t)p.tile, p.rows - row0);
  pdl_wait();
  for (int i = threadIdx.x; i < n_rows * p.pairs; i += kThreads) {
    const int r = fast_div(i, p.by_pairs);
    const int pair = i - r * p.pairs;
    const int64_t row = row0 + r;
    const int64_t b = row / p.tokens;
    const int64_t t = row - b * p.tokens;
    const int axis = (pair >= p.axis_end[0]) + (pair >= p.axis_end[1]);
    const int32_t pos = p.pos[b * p.pos_batch + t * p.axes + axis];
    const uint64_t turn = (uint64_t)(int64_t)pos * p.turn[pair];
    // half turns in [-1, 1)
    const float x = (float)(int32_t)(turn >> 32) * 0x1p-31f;
    float s, c;
    sincospif(x, &s, &c);
    cs[i] = make_float2(c * p.mag, s * p.sign);
  }
  __syncthreads();

  using Vt = Vec<T, V>;
  const int half = p.pairs;
  const int pair_items = kHalf ? half / V : p.items;
  const int total = n_rows * p.all_heads * p.items;
  for (int i0 = threadIdx.x; i0 < total; i0 += kThreads * kUnroll) {
    Vt a[kUnroll], b[kUnroll];
    T* dst[kUnroll];
    int item[kUnroll], r[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int i = i0 + u * kThreads;
      if (i >= total) break;
      const int rh = fast_div(i, p.by_items);
      item[u] = i - rh * p.items;
      r[u] = fast_div(rh, p.by_heads);
      int h = rh - r[u] * p.all_heads;
      const int64_t row = row0 + r[u];
      const int64_t bb = p.rows == p.tokens ? 0 : row / p.tokens;
      const int64_t t = row - bb * p.tokens;
      const bool is_k = h >= p.heads;
      if (is_k) h -= p.heads;
      const Strides& si = is_k ? p.k_str : p.q_str;
      const Strides& so = is_k ? p.k_out_str : p.q_out_str;
      const T* src = static_cast<const T*>(is_k ? p.k : p.q) + bb * si.batch +
                     t * si.token + h * si.head;
      dst[u] = static_cast<T*>(is_k ? p.k_out : p.q_out) + bb * so.batch +
               t * so.token + h * so.head;
      if (kHalf) {
        const bool rot = item[u] < pair_items;
        const int x = rot ? item[u] * V : 2 * half + (item[u] - pair_items) * V;
        a[u] = *reinterpret_cast<const Vt*>(src + x);
        if (rot) b[u] = *reinterpret_cast<const Vt*>(src + x + half);
      } else {
        a[u] = *reinterpret_cast<const Vt*>(src + item[u] * V);
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (i0 + u * kThreads >= total) break;
      if (kHalf) {
        if (item[u] >= pair_items) {
          *reinterpret_cast<Vt*>(dst[u] + 2 * half +
                                 (item[u] - pair_items) * V) = a[u];
          continue;
        }
        const float2* w = cs + r[u] * half + item[u] * V;
        Vt y, z;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          const float2 cw = w[e];
          const float fa = to_f(a[u].e[e]), fb = to_f(b[u].e[e]);
          from_f(y.e[e], fa * cw.x - fb * cw.y);
          from_f(z.e[e], fb * cw.x + fa * cw.y);
        }
        *reinterpret_cast<Vt*>(dst[u] + item[u] * V) = y;
        *reinterpret_cast<Vt*>(dst[u] + half + item[u] * V) = z;
      } else {
        Vt y = a[u];
        const float2* w = cs + r[u] * half + item[u] * (V / 2);
        const int left = half - item[u] * (V / 2);  // pairs from here on
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
          if (e < left) {
            const float2 cw = w[e];
            const float fa = to_f(a[u].e[2 * e]), fb = to_f(a[u].e[2 * e + 1]);
            from_f(y.e[2 * e], fa * cw.x - fb * cw.y);
            from_f(y.e[2 * e + 1], fb * cw.x + fa * cw.y);
          }
        }
        *reinterpret_cast<Vt*>(dst[u] + item[u] * V) = y;
      }
    }
  }
}

template <typename T>
cudaError_t launch_t(const RotaryArgs& a, Params& p, cudaStream_t stream) {
  // Half layout: the two elements of a pair are rot/2 apart, so the widest
  // vector is the largest power of two (at most 8 elements) dividing it.
  int v = 8;
  if (a.half)
    while (p.pairs % v) v /= 2;
  p.items = a.half ? (p.pairs + p.head_dim - 2 * p.pairs) / v : p.head_dim / 8;
  p.by_items = make_div(p.items);
  // Tokens of a CTA: what the sine table holds, no more than leave every SM
  // a few CTAs (a decode step has one token per stream).
  int64_t tile = kSmemPairs / p.pairs;
  const int64_t spread = p.rows / ((int64_t)a.sms * 4);
  if (tile > spread) tile = spread;
  // total items of a CTA stay within 32 bits: all_heads * items * tile
  const int64_t per = (int64_t)p.all_heads * p.items;
  if (tile > (1 << 30) / per) tile = (1 << 30) / per;
  if (tile < 1) tile = 1;
  p.tile = (int32_t)tile;
  const int64_t grid = (p.rows + tile - 1) / tile;
  if (grid > 0x7fffffffLL || per > (1 << 30)) return cudaErrorInvalidValue;
  const dim3 g((unsigned)grid), b(kThreads);
  if (!a.half) return launch_pdl(rotary_kernel<T, false, 8>, g, b, 0, stream, p);
  switch (v) {
    case 8: return launch_pdl(rotary_kernel<T, true, 8>, g, b, 0, stream, p);
    case 4: return launch_pdl(rotary_kernel<T, true, 4>, g, b, 0, stream, p);
    case 2: return launch_pdl(rotary_kernel<T, true, 2>, g, b, 0, stream, p);
    default: return launch_pdl(rotary_kernel<T, true, 1>, g, b, 0, stream, p);
  }
}

}  // namespace

cudaError_t launch_rotary(const RotaryArgs& a, cudaStream_t stream) {
  Params p;
  p.q = a.q;
  p.k = a.k;
  p.q_out = a.q_out;
  p.k_out = a.k_out;
  p.pos = a.positions;
  p.pos_batch = a.pos_batch;
  p.q_str = a.q_str;
  p.k_str = a.k_str;
  p.q_out_str = a.q_out_str;
  p.k_out_str = a.k_out_str;
  p.rows = (int64_t)a.batch * a.tokens;
  p.tokens = a.tokens;
  p.axes = a.axes;
  p.pairs = a.pairs;
  p.head_dim = a.head_dim;
  int end = 0;
  for (int i = 0; i < 3; ++i) {
    if (i < a.axes) end += a.section[i];
    p.axis_end[i] = end;
  }
  p.by_tokens = make_div(a.tokens);
  p.by_pairs = make_div(a.pairs);
  p.heads = a.heads;
  p.all_heads = a.heads + a.kv_heads;
  p.by_heads = make_div(p.all_heads);
  p.mag = a.magnitude;
  p.sign = a.transpose ? -a.magnitude : a.magnitude;
  for (int i = 0; i < a.pairs; ++i) p.turn[i] = a.turn[i];
  return a.f32 ? launch_t<float>(a, p, stream)
               : launch_t<__nv_bfloat16>(a, p, stream);
}

}  // namespace fastvr
