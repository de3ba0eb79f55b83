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

#include <algorithm>

#include "fastvr_internal.h"

namespace fastvr {
namespace {

constexpr int kThreads = 256;
constexpr int kSmemPairs = 2048;  // (token, pair) entries per CTA: 16 KB

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
  int32_t rows;               // batch * tokens
  int32_t tokens, axes, pairs, head_dim;
  int32_t tile;               // tokens of a CTA
  int32_t axis_end[3];        // first pair past each axis
  FastDiv by_tokens, by_pairs, by_blocks;
  int32_t items;              // vector items of a head
  int32_t lanes;              // threads of a group, one per item
  int32_t head_blocks;
  int32_t heads, all_heads;   // q heads, q and k heads
  float mag, sign;
  uint64_t turn[kRotaryMaxPairs];  // theta / 2 pi in 2^-64 turns
};

// Heads that a thread takes at once: 64 bytes of loads in flight (64 registers
// keep 32 warps on an SM).
__host__ __device__ constexpr int head_block(int elem_bytes, bool half) {
  return 8 / elem_bytes / (half ? 2 : 1);
}

// One head's item: kHalf: the vectors of V elements at i V and rot/2 + i V
// (one per pair of the V), then the pass-through vectors; interleaved: the
// vector at i V, V / 2 pairs.  A group of threads, one per item, takes a block
// of HB heads of a token at a time: the sines of a thread's item are read once
// for the block, and the block's loads are in flight together.
template <typename T, bool kHalf, int V>
__global__ void __launch_bounds__(kThreads, 4)
rotary_kernel(const __grid_constant__ Params p) {
  constexpr int HB = head_block(sizeof(T), kHalf);
  constexpr int kPairs = kHalf ? V : V / 2;  // pairs of an item
  __shared__ __align__(16) float2 cs[kSmemPairs + 8];
  pdl_trigger();
  const int row0 = blockIdx.x * p.tile;
  const int n_rows = min(p.tile, p.rows - row0);
  pdl_wait();
  for (int i = threadIdx.x; i < n_rows * p.pairs; i += kThreads) {
    const int r = fast_div(i, p.by_pairs);
    const int pair = i - r * p.pairs;
    const int row = row0 + r;
    const int b = fast_div(row, p.by_tokens);
    const int t = row - b * p.tokens;
    const int axis = (pair >= p.axis_end[0]) + (pair >= p.axis_end[1]);
    const int32_t pos = p.pos[b * p.pos_batch + (int64_t)t * p.axes + axis];
    const uint64_t turn = (uint64_t)(int64_t)pos * p.turn[pair];
    // half turns in [-1, 1)
    const float x = (float)(int32_t)(turn >> 32) * 0x1p-31f;
    float s, c;
    sincospif(x, &s, &c);
    cs[i] = make_float2(c * p.mag, s * p.sign);
  }
  __syncthreads();

  using Vt = Vec<T, V>;
  const int pair_items = kHalf ? p.pairs / V : p.items;
  const int group = threadIdx.x / p.lanes;
  const int groups = kThreads / p.lanes;
  const int lane = threadIdx.x - group * p.lanes;
  if (group >= groups) return;
  const int tasks = n_rows * p.head_blocks;
  for (int task = group; task < tasks; task += groups) {
    const int r = fast_div(task, p.by_blocks);
    const int h0 = (task - r * p.head_blocks) * HB;
    const int row = row0 + r;
    const int b = fast_div(row, p.by_tokens);
    const int t = row - b * p.tokens;
    const T* q = static_cast<const T*>(p.q) + b * p.q_str.batch +
                 t * p.q_str.token;
    const T* k = static_cast<const T*>(p.k) + b * p.k_str.batch +
                 t * p.k_str.token;
    T* qo = static_cast<T*>(p.q_out) + b * p.q_out_str.batch +
            t * p.q_out_str.token;
    T* ko = static_cast<T*>(p.k_out) + b * p.k_out_str.batch +
            t * p.k_out_str.token;
    for (int item = lane; item < p.items; item += p.lanes) {
      const bool rot = !kHalf || item < pair_items;
      const int x =
          rot ? item * V : 2 * p.pairs + (item - pair_items) * V;
      Vt a[HB], z[HB];
#pragma unroll
      for (int u = 0; u < HB; ++u) {
        const int h = h0 + u;
        if (h >= p.all_heads) continue;
        const T* src = h < p.heads ? q + h * p.q_str.head
                                   : k + (h - p.heads) * p.k_str.head;
        a[u] = *reinterpret_cast<const Vt*>(src + x);
        if (kHalf && rot)
          z[u] = *reinterpret_cast<const Vt*>(src + x + p.pairs);
      }
      if (rot) {
        float2 w[kPairs];
        const int pair0 = item * kPairs;
#pragma unroll
        for (int e = 0; e < kPairs; ++e)
          w[e] = cs[r * p.pairs + pair0 + e];  // the table is padded
#pragma unroll
        for (int u = 0; u < HB; ++u) {
          if (h0 + u >= p.all_heads) continue;
#pragma unroll
          for (int e = 0; e < kPairs; ++e) {
            // the rotated part may end inside a piece; the rest is copied
            if (!kHalf && pair0 + e >= p.pairs) continue;
            T& ra = kHalf ? a[u].e[e] : a[u].e[(2 * e) % V];
            T& rb = kHalf ? z[u].e[e] : a[u].e[(2 * e + 1) % V];
            const float fa = to_f(ra), fb = to_f(rb);
            from_f(ra, fa * w[e].x - fb * w[e].y);
            from_f(rb, fb * w[e].x + fa * w[e].y);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < HB; ++u) {
        const int h = h0 + u;
        if (h >= p.all_heads) continue;
        T* dst = h < p.heads ? qo + h * p.q_out_str.head
                             : ko + (h - p.heads) * p.k_out_str.head;
        *reinterpret_cast<Vt*>(dst + x) = a[u];
        if (kHalf && rot) *reinterpret_cast<Vt*>(dst + x + p.pairs) = z[u];
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
  p.items = a.half ? (p.head_dim - p.pairs) / v : p.head_dim / 8;
  p.lanes = p.items < kThreads ? p.items : kThreads;
  const int hb = head_block(sizeof(T), a.half);
  p.head_blocks = (p.all_heads + hb - 1) / hb;
  p.by_blocks = make_div(p.head_blocks);
  // Tokens of a CTA: what the sine table holds, and few enough that every SM
  // has a dozen CTAs to even out its last ones.
  int64_t tile = kSmemPairs / p.pairs;
  tile = std::min<int64_t>(tile, p.rows / (a.sms * 12));
  tile = std::min<int64_t>(tile, (1 << 30) / p.head_blocks);
  if (tile < 1) tile = 1;
  p.tile = (int32_t)tile;
  const dim3 g((unsigned)((p.rows + tile - 1) / tile)), b(kThreads);
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
  p.rows = a.batch * a.tokens;
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
  p.mag = a.magnitude;
  p.sign = a.transpose ? -a.magnitude : a.magnitude;
  for (int i = 0; i < a.pairs; ++i) p.turn[i] = a.turn[i];
  return a.f32 ? launch_t<float>(a, p, stream)
               : launch_t<__nv_bfloat16>(a, p, stream);
}

}  // namespace fastvr
