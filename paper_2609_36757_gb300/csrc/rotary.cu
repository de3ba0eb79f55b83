// Rotary positions on the queries and keys of a block, and their transpose
// (the gradient): for every pair (a, b) of a head,
//   a' = m (a cos x - b sin x),  b' = m (b cos x + a sin x),  x = p theta.
//
// Bound by memory: every element is read once and written once (4 bytes per
// bfloat16 element).  The sines depend on the token alone, so a CTA takes a
// few whole tokens, forms cos and sin of their pairs once in shared memory
// and applies them to all heads of q and of k in one pass of 16-byte
// accesses, the first of which are asked for before the sines: 32.0 us (6.3
// TB/s) for q and k of 16320 tokens of 12 heads of 128, 50.0 us (6.0 TB/s) for
// the transpose on 12288 tokens of 24 heads, 64 of 128 elements rotated.
//
// The angle is reduced exactly before any floating-point step: theta / 2 pi
// is held as a 64-bit fixed-point fraction F of a turn (host, rounded once),
// p F modulo 2^64 is the turn's fraction for every int32 position, and its
// top 32 bits go to sincospi.  A position of 10^6 is as accurate as 1.
#include <cuda_bf16.h>

#include <algorithm>

#include "fastvr_internal.h"
#include "vec_math.cuh"

namespace fastvr {
namespace {

constexpr int kThreads = 256;
constexpr int kSmemPairs = 2048;  // (token, pair) entries per CTA: 16 KB

// V consecutive elements of T as they lie in memory.
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

// Elements (2 i, 2 i + 1) of a vector as a pair, and back.
template <int V>
__device__ __forceinline__ F2 get2(const Vec<__nv_bfloat16, V>& v, int i) {
  const uint32_t w = reinterpret_cast<const uint32_t*>(v.e)[i];
  return f2(bf16_lo(w), bf16_hi(w));
}
template <int V>
__device__ __forceinline__ F2 get2(const Vec<float, V>& v, int i) {
  return f2(v.e[2 * i], v.e[2 * i + 1]);
}
template <int V>
__device__ __forceinline__ void put2(Vec<__nv_bfloat16, V>& v, int i, F2 x) {
  reinterpret_cast<uint32_t*>(v.e)[i] = bf16_pack(x);
}
template <int V>
__device__ __forceinline__ void put2(Vec<float, V>& v, int i, F2 x) {
  split(x, v.e[2 * i], v.e[2 * i + 1]);
}
// Elements (4 i, 4 i + 2) and (4 i + 1, 4 i + 3): the first and the second
// ones of two neighbouring pairs.
template <int V>
__device__ __forceinline__ void get_pairs(const Vec<__nv_bfloat16, V>& v, int i,
                                          F2& a, F2& b) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(v.e) + 2 * i;
  a = f2(bf16_lo(w[0]), bf16_lo(w[1]));
  b = f2(bf16_hi(w[0]), bf16_hi(w[1]));
}
template <int V>
__device__ __forceinline__ void get_pairs(const Vec<float, V>& v, int i, F2& a,
                                          F2& b) {
  a = f2(v.e[4 * i], v.e[4 * i + 2]);
  b = f2(v.e[4 * i + 1], v.e[4 * i + 3]);
}
template <int V>
__device__ __forceinline__ void put_pairs(Vec<__nv_bfloat16, V>& v, int i, F2 a,
                                          F2 b) {
  float a0, a1, b0, b1;
  split(a, a0, a1);
  split(b, b0, b1);
  uint32_t* w = reinterpret_cast<uint32_t*>(v.e) + 2 * i;
  w[0] = bf16_pack(a0, b0);
  w[1] = bf16_pack(a1, b1);
}
template <int V>
__device__ __forceinline__ void put_pairs(Vec<float, V>& v, int i, F2 a, F2 b) {
  split(a, v.e[4 * i], v.e[4 * i + 2]);
  split(b, v.e[4 * i + 1], v.e[4 * i + 3]);
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
  int32_t items;              // vector items of a head
  int32_t pass_step;          // half layout: see rotary_kernel; or 0
  int32_t lanes;              // threads of a group, an item each
  int32_t heads, kv_heads;
  int32_t q_blocks, blocks;   // blocks of heads of q, of q and k
  int32_t item_blocks;        // of `lanes` items
  FastDiv by_tokens, by_pairs, by_blocks, by_item_blocks;
  float mag, sign;
  uint64_t turn[kRotaryMaxPairs];  // theta / 2 pi in 2^-64 turns
};

// Heads that a thread takes at once: 64 bytes of loads in flight (64 registers
// keep 32 warps on an SM).
__host__ __device__ constexpr int head_block(int elem_bytes, bool half) {
  return 8 / elem_bytes / (half ? 2 : 1);
}

// One head's item: kHalf: the vectors of V elements at i V and rot/2 + i V
// (one per pair of the V), then the pass-through vectors, two to an item as
// well (pass_step apart) when their number is even; interleaved: the vector at
// i V, V / 2 pairs.  A group of threads, one per item, takes a block
// of HB heads of a token at a time: the sines of a thread's item are read once
// for the block, and the block's loads are in flight together.  The first
// block's are on their way while the sines are formed.
template <typename T, bool kHalf, int V>
__global__ void __launch_bounds__(kThreads, 4)
rotary_kernel(const __grid_constant__ Params p) {
  constexpr int HB = head_block(sizeof(T), kHalf);
  constexpr int kPairs = kHalf ? V : V / 2;  // pairs of an item
  using Vt = Vec<T, V>;
  // (cos, cos, sin, sin) of two neighbouring pairs of a token
  __shared__ float4 cs[kSmemPairs / 2 + 4];
  pdl_trigger();
  const int row0 = blockIdx.x * p.tile;
  const int n_rows = min(p.tile, p.rows - row0);
  const int entries = (p.pairs + 1) / 2;  // of a token
  const int pair_items = kHalf ? p.pairs / V : p.items;
  const int group = threadIdx.x / p.lanes;
  const int groups = kThreads / p.lanes;
  const int lane = threadIdx.x - group * p.lanes;
  const int tasks = group < groups ? n_rows * p.blocks * p.item_blocks : 0;
  pdl_wait();

  Vt a[HB], z[HB];
  T* dst;
  int64_t dst_head;
  int n_heads, item, r, second;  // second: distance of the item's other vector
  bool rot;
  auto load = [&](int task) {
    const int rb = fast_div(task, p.by_item_blocks);
    item = (task - rb * p.item_blocks) * p.lanes + lane;
    r = fast_div(rb, p.by_blocks);
    const int block = rb - r * p.blocks;
    const bool is_k = block >= p.q_blocks;
    const int h0 = (is_k ? block - p.q_blocks : block) * HB;
    n_heads = item < p.items
                  ? min(HB, (is_k ? p.kv_heads : p.heads) - h0)
                  : 0;
    rot = !kHalf || item < pair_items;
    const int x = rot ? item * V : 2 * p.pairs + (item - pair_items) * V;
    second = rot ? p.pairs : p.pass_step;
    const int row = row0 + r;
    const int b = fast_div(row, p.by_tokens);
    const int t = row - b * p.tokens;
    const Strides& si = is_k ? p.k_str : p.q_str;
    const Strides& so = is_k ? p.k_out_str : p.q_out_str;
    const T* src = static_cast<const T*>(is_k ? p.k : p.q) + b * si.batch +
                   t * si.token + h0 * si.head + x;
    dst = static_cast<T*>(is_k ? p.k_out : p.q_out) + b * so.batch +
          t * so.token + h0 * so.head + x;
    dst_head = so.head;
#pragma unroll
    for (int u = 0; u < HB; ++u)
      if (u < n_heads) {
        a[u] = *reinterpret_cast<const Vt*>(src + u * si.head);
        if (kHalf && second)
          z[u] = *reinterpret_cast<const Vt*>(src + u * si.head + second);
      }
  };
  int task = group;
  if (task < tasks) load(task);

  for (int i = threadIdx.x; i < n_rows * p.pairs; i += kThreads) {
    const int row_i = fast_div(i, p.by_pairs);
    const int pair = i - row_i * p.pairs;
    const int row = row0 + row_i;
    const int b = fast_div(row, p.by_tokens);
    const int t = row - b * p.tokens;
    const int axis = (pair >= p.axis_end[0]) + (pair >= p.axis_end[1]);
    const int32_t pos = p.pos[b * p.pos_batch + (int64_t)t * p.axes + axis];
    const uint64_t turn = (uint64_t)(int64_t)pos * p.turn[pair];
    // half turns in [-1, 1)
    const float x = (float)(int32_t)(turn >> 32) * 0x1p-31f;
    float s, c;
    sincospif(x, &s, &c);
    float* e = reinterpret_cast<float*>(cs + row_i * entries + pair / 2) +
               pair % 2;
    e[0] = c * p.mag;
    e[2] = s * p.sign;
  }
  __syncthreads();

  for (; task < tasks; task += groups, task < tasks ? load(task) : void()) {
    const int pair0 = item * kPairs;
    const float4* w = cs + r * entries + pair0 / 2;
    if (V == 1 || (!kHalf && pair0 + kPairs > p.pairs)) {
      // one pair, or a piece inside which the rotated part ends (the rest of
      // it is copied)
      if (rot) {
#pragma unroll
        for (int e = 0; e < kPairs; ++e) {
          if (pair0 + e >= p.pairs) continue;
          const float* f = reinterpret_cast<const float*>(
                               cs + r * entries + (pair0 + e) / 2) +
                           (pair0 + e) % 2;
          const float c = f[0], s = f[2];
#pragma unroll
          for (int u = 0; u < HB; ++u) {
            T& ra = kHalf ? a[u].e[e] : a[u].e[(2 * e) % V];
            T& rb = kHalf ? z[u].e[e] : a[u].e[(2 * e + 1) % V];
            const float fa = to_f(ra), fb = to_f(rb);
            from_f(ra, fa * c - fb * s);
            from_f(rb, fb * c + fa * s);
          }
        }
      }
    } else if (rot) {
#pragma unroll
      for (int e = 0; e < kPairs / 2; ++e) {
        const float4 f = w[e];
        const F2 c = f2(f.x, f.y), s = f2(f.z, f.w), ns = f2(-f.z, -f.w);
#pragma unroll
        for (int u = 0; u < HB; ++u) {
          F2 fa, fb;
          if constexpr (kHalf) {
            fa = get2(a[u], e);
            fb = get2(z[u], e);
          } else {
            get_pairs(a[u], e, fa, fb);
          }
          const F2 ya = fma(fb, ns, mul(fa, c));
          const F2 yb = fma(fa, s, mul(fb, c));
          if constexpr (kHalf) {
            put2(a[u], e, ya);
            put2(z[u], e, yb);
          } else {
            put_pairs(a[u], e, ya, yb);
          }
        }
      }
    }
#pragma unroll
    for (int u = 0; u < HB; ++u)
      if (u < n_heads) {
        *reinterpret_cast<Vt*>(dst + u * dst_head) = a[u];
        if (kHalf && second)
          *reinterpret_cast<Vt*>(dst + u * dst_head + second) = z[u];
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
  p.items = p.head_dim / 8;
  p.pass_step = 0;
  if (a.half) {
    const int pass = (p.head_dim - 2 * p.pairs) / v;  // vectors
    p.pass_step = pass % 2 == 0 ? pass / 2 * v : 0;
    p.items = p.pairs / v + (pass % 2 == 0 ? pass / 2 : pass);
  }
  p.lanes = std::min(p.items, kThreads);
  p.item_blocks = (p.items + p.lanes - 1) / p.lanes;
  const int hb = head_block(sizeof(T), a.half);
  p.q_blocks = (p.heads + hb - 1) / hb;
  p.blocks = p.q_blocks + (p.kv_heads + hb - 1) / hb;
  p.by_blocks = make_div(p.blocks);
  p.by_item_blocks = make_div(p.item_blocks);
  // Tokens of a CTA: what the sine table holds, at most 8, and few enough
  // that every SM has eight CTAs to even out its last ones.
  const int entries = (p.pairs + 1) / 2;
  int64_t tile = std::min(8, kSmemPairs / 2 / entries);
  tile = std::min<int64_t>(tile, p.rows / (a.sms * 8));
  tile = std::min<int64_t>(tile, (1 << 30) / ((int64_t)p.blocks * p.item_blocks));
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
  p.kv_heads = a.kv_heads;
  p.mag = a.magnitude;
  p.sign = a.transpose ? -a.magnitude : a.magnitude;
  for (int i = 0; i < a.pairs; ++i) p.turn[i] = a.turn[i];
  return a.f32 ? launch_t<float>(a, p, stream)
               : launch_t<__nv_bfloat16>(a, p, stream);
}

}  // namespace fastvr
