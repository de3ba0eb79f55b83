// Shared by the forward and the backward of the gated residual and norms.
#pragma once

#include <cuda_bf16.h>

#include "fastvr_internal.h"
#include "vec_math.cuh"

namespace fastvr {
namespace norm {

// 8 float32 values, two to a register pair.
struct F8 {
  F2 v[4];
};
__device__ __forceinline__ F8 splat(float x) {
  F8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.v[i] = f2(x);
  return r;
}
__device__ __forceinline__ F8 add(const F8& a, const F8& b) {
  F8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.v[i] = add(a.v[i], b.v[i]);
  return r;
}
__device__ __forceinline__ F8 mul(const F8& a, const F8& b) {
  F8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.v[i] = mul(a.v[i], b.v[i]);
  return r;
}
__device__ __forceinline__ F8 fma(const F8& a, const F8& b, const F8& c) {
  F8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.v[i] = fma(a.v[i], b.v[i], c.v[i]);
  return r;
}
// The same with one factor, or a factor and a summand, for all.
__device__ __forceinline__ F8 mul(const F8& a, float b) {
  return mul(a, splat(b));
}
__device__ __forceinline__ F8 fma(const F8& a, float b, const F8& c) {
  return fma(a, splat(b), c);
}
__device__ __forceinline__ F8 fma(const F8& a, float b, float c) {
  return fma(a, splat(b), splat(c));
}
__device__ __forceinline__ float sum(const F8& a) {
  return sum(add(add(a.v[0], a.v[1]), add(a.v[2], a.v[3])));
}

// 8 consecutive elements in memory: 16 bytes of bfloat16 or 32 of float32.
template <typename T>
struct Raw8;
template <>
struct Raw8<__nv_bfloat16> {
  uint4 u;
  __device__ __forceinline__ void load(const void* base, int64_t i) {
    u = *reinterpret_cast<const uint4*>(
        static_cast<const __nv_bfloat16*>(base) + i);
  }
  __device__ __forceinline__ F8 widen() const {
    F8 r;
    r.v[0] = f2(bf16_lo(u.x), bf16_hi(u.x));
    r.v[1] = f2(bf16_lo(u.y), bf16_hi(u.y));
    r.v[2] = f2(bf16_lo(u.z), bf16_hi(u.z));
    r.v[3] = f2(bf16_lo(u.w), bf16_hi(u.w));
    return r;
  }
};
template <>
struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const void* base, int64_t i) {
    const float4* p =
        reinterpret_cast<const float4*>(static_cast<const float*>(base) + i);
    a = p[0];
    b = p[1];
  }
  __device__ __forceinline__ F8 widen() const {
    F8 r;
    r.v[0] = f2(a.x, a.y);
    r.v[1] = f2(a.z, a.w);
    r.v[2] = f2(b.x, b.y);
    r.v[3] = f2(b.z, b.w);
    return r;
  }
};

__device__ __forceinline__ void store8(__nv_bfloat16* base, int64_t i,
                                       const F8& f) {
  *reinterpret_cast<uint4*>(base + i) =
      make_uint4(bf16_pack(f.v[0]), bf16_pack(f.v[1]), bf16_pack(f.v[2]),
                 bf16_pack(f.v[3]));
}
__device__ __forceinline__ void store8(float* base, int64_t i, const F8& f) {
  float x[8];
#pragma unroll
  for (int e = 0; e < 4; ++e) split(f.v[e], x[2 * e], x[2 * e + 1]);
  float4* p = reinterpret_cast<float4*>(base + i);
  p[0] = make_float4(x[0], x[1], x[2], x[3]);
  p[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// Rows on their way: 16-byte pieces of each thread's columns, copied
// asynchronously by the threads of its own warp, so that they need not meet the
// others.  kDeep rows of kPieces pieces; a row is asked for kDeep - 1 rows
// ahead, in the place of the one last worked on.
template <int kDeep, int kPieces>
struct Ring {
  float4* base;  // [row][piece][thread]
  int at = 0;    // the row that is worked on
  // Piece i, half h of a vector of a thread: neighbours swap their second
  // halves' places, so that neither the copies nor the reads meet in a bank.
  __device__ __forceinline__ float4* piece(int row, int i, int h,
                                           int thread) const {
    return base + (row * kPieces + i + h) * blockDim.x + (thread ^ 4 * h);
  }
  // 8 elements per thread into the row `ahead` of the one that is worked on;
  // index(thread): where a thread's elements are, negative if it has none.
  // Float32: the 64 pieces of a warp in the order of memory.
  template <typename T, typename F>
  __device__ __forceinline__ void ask(int ahead, int i, const void* from,
                                      F index) const {
    int row = at + ahead;
    if (row >= kDeep) row -= kDeep;
    if constexpr (sizeof(T) == 2) {
      const int64_t e = index(threadIdx.x);
      if (e >= 0)
        copy_async<16>(smem_u32(piece(row, i, 0, threadIdx.x)),
                       static_cast<const T*>(from) + e, true);
    } else {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int of =
            (threadIdx.x & ~31) + (threadIdx.x & 31) / 2 + 16 * n;
        const int64_t e = index(of);
        const int h = threadIdx.x & 1;
        if (e >= 0)
          copy_async<16>(smem_u32(piece(row, i, h, of)),
                         static_cast<const T*>(from) + e + 4 * h, true);
      }
    }
  }
  // until the row that is worked on is there
  __device__ __forceinline__ void wait() const {
    copy_wait<kDeep - 1>();
    __syncwarp();
  }
  template <typename T>
  __device__ __forceinline__ F8 get(int i) const {
    if constexpr (sizeof(T) == 2) {
      const Raw8<T> r = {*reinterpret_cast<const uint4*>(
          piece(at, i, 0, threadIdx.x))};
      return r.widen();
    } else {
      const Raw8<T> r = {*piece(at, i, 0, threadIdx.x),
                         *piece(at, i, 1, threadIdx.x)};
      return r.widen();
    }
  }
  // done with it on every lane
  __device__ __forceinline__ void next() {
    __syncwarp();
    at = at + 1 == kDeep ? 0 : at + 1;
  }
};

// Its depth: what a CTA's share of an SM's 227 KB leaves beside `fixed` bytes
// of each of its vectors (2 KB for the system and the static part); 0 where two
// rows do not fit.
constexpr int kSmBytes = 232448;
constexpr int ring_depth(int ctas, int vectors, int fixed, int bytes,
                         int most) {
  const int fit = ((kSmBytes / ctas - 2048) / vectors - fixed) / bytes;
  return fit < 2 ? 0 : fit > most ? most : fit;
}

// 8 floats of an optional vector, `absent` where there is none.
__device__ __forceinline__ F8 load8_or(const float* base, int64_t i,
                                       float absent) {
  if (base == nullptr) return splat(absent);
  Raw8<float> r;
  r.load(base, i);
  return r.widen();
}

// Vectors of 8 floats that belong to a thread, in shared memory: what is used
// once per row leaves its registers to the rows in flight (a spilled register
// costs more than such a read).  The halves lie apart, so that the lanes of a
// warp touch consecutive 16 bytes.
struct Private {
  float4* base;  // [vector][half][thread]
  __device__ __forceinline__ F8 get(int i) const {
    const float4 a = base[2 * i * blockDim.x + threadIdx.x];
    const float4 b = base[(2 * i + 1) * blockDim.x + threadIdx.x];
    F8 r;
    r.v[0] = f2(a.x, a.y);
    r.v[1] = f2(a.z, a.w);
    r.v[2] = f2(b.x, b.y);
    r.v[3] = f2(b.z, b.w);
    return r;
  }
  __device__ __forceinline__ void set(int i, const F8& f) const {
    float x[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) split(f.v[e], x[2 * e], x[2 * e + 1]);
    base[2 * i * blockDim.x + threadIdx.x] =
        make_float4(x[0], x[1], x[2], x[3]);
    base[(2 * i + 1) * blockDim.x + threadIdx.x] =
        make_float4(x[4], x[5], x[6], x[7]);
  }
};

// N such vectors, the first kRegs in registers.
template <int kRegs, int N>
struct Kept {
  F8 r[kRegs ? kRegs : 1];
  Private m;
  __device__ __forceinline__ F8 get(int i) const {
    return i < kRegs ? r[i < kRegs ? i : 0] : m.get(i - kRegs);
  }
  __device__ __forceinline__ void set(int i, const F8& f) {
    if (i < kRegs)
      r[i < kRegs ? i : 0] = f;
    else
      m.set(i - kRegs, f);
  }
};

// Sums of a and of b over the L lanes of a row within a warp, at the price of
// about one: the halves of the lanes first trade what they do not keep.
// `keep_sums` leaves a's sum on the lanes of the lower half and b's on those
// of the upper one; `both_sums` leaves both on every lane.
template <int L>
__device__ __forceinline__ float keep_sums(float a, float b) {
  const bool hi = threadIdx.x & (L / 2);
  float v = hi ? b : a;
  v += __shfl_xor_sync(0xffffffffu, hi ? a : b, L / 2);
#pragma unroll
  for (int m = L / 4; m > 0; m >>= 1) v += __shfl_xor_sync(0xffffffffu, v, m);
  return v;
}
template <int L>
__device__ __forceinline__ void both_sums(float& a, float& b) {
  const bool hi = threadIdx.x & (L / 2);
  const float v = keep_sums<L>(a, b);
  const float o = __shfl_xor_sync(0xffffffffu, v, L / 2);
  a = hi ? o : v;
  b = hi ? v : o;
}

// Groups of fewer tokens than this: what happens once per group counts.
constexpr int kFewTokens = 16;

// A row's threads: TPR of them with NV vectors of 8 columns each, vector i at
// column (i TPR + thread) 8.  Up to 32: 128 / TPR rows side by side in a CTA of
// 128 threads, their sums within a warp.  Above: a row to a CTA, its sums
// across the warps.
template <int TPR>
struct Shape {
  static constexpr int kThreads = TPR <= 32 ? 128 : TPR;
  static constexpr int kLanes = TPR < 32 ? TPR : 32;
  static constexpr int kRows = TPR <= 32 ? 128 / TPR : 1;
  static constexpr bool kMany = TPR > 32;
  static constexpr int kWarps = kMany ? TPR / 32 : 1;
  // (all of many warps' parts at once take too many registers)
  static constexpr int kUnroll = kWarps <= 8 ? kWarps : 4;
};

// What a thread knows of its row's columns.
template <int TPR, int NV>
struct Cols {
  using S = Shape<TPR>;
  int dim, c;  // c: its first column
  float inv_dim, inv_warp;  // 1 / columns of the row, of this warp
  const float* counts;      // columns of each warp of the row
  // `n`: kWarps floats of shared memory, filled before the first exchange
  __device__ __forceinline__ Cols(int d, float* n) : dim(d), counts(n) {
    c = (S::kRows > 1 ? threadIdx.x % TPR : threadIdx.x) * 8;
    inv_dim = 1.f / (float)d;
    int mine = d;
    if (S::kMany) {
      mine = 0;
      for (int i = 0; i < NV; ++i)
        mine += min(256, max(0, d - (i * TPR + (int)threadIdx.x / 32 * 32) * 8));
    }
    inv_warp = 1.f / (float)max(mine, 1);
    if (threadIdx.x % 32 == 0 && (S::kMany || threadIdx.x == 0))
      n[S::kMany ? threadIdx.x / 32 : 0] = (float)mine;
  }
  __device__ __forceinline__ int at(int i) const { return c + i * TPR * 8; }
  // the same for another thread
  __device__ __forceinline__ int at(int i, int thread) const {
    return ((S::kRows > 1 ? thread % TPR : thread) + i * TPR) * 8;
  }
  __device__ __forceinline__ bool on(int i) const { return at(i) < dim; }
};

// Sums of the N (4 or 8) values over the L lanes of a row within a warp: the
// lanes trade halves, quarters and so on of what they hold, so lane i ends with
// the sum of value i / (L / N).
template <int L, int N>
__device__ __forceinline__ float keep_sum(float (&v)[N]) {
#pragma unroll
  for (int n = N / 2, m = L / 2; n > 0; n /= 2, m /= 2) {
    const bool hi = threadIdx.x & m;
#pragma unroll
    for (int i = 0; i < n; ++i) {
      const float give = hi ? v[i] : v[n + i];
      v[i] = (hi ? v[n + i] : v[i]) + __shfl_xor_sync(0xffffffffu, give, m);
    }
  }
  float s = v[0];
#pragma unroll
  for (int m = L / N / 2; m > 0; m >>= 1)
    s += __shfl_xor_sync(0xffffffffu, s, m);
  return s;
}

// Sums over a row of many warps of a and of b, on every thread; `part` (kWarps
// entries) is this exchange's own: two exchanges with another part between them
// need one barrier each.
template <int TPR>
__device__ __forceinline__ void row_sums(float& a, float& b, float2* part) {
  using S = Shape<TPR>;
  const float v = keep_sums<32>(a, b);
  if (threadIdx.x % 16 == 0)
    reinterpret_cast<float*>(part)[threadIdx.x / 16] = v;
  __syncthreads();
  F2 all = f2(0.f);
#pragma unroll(S::kUnroll)
  for (int w = 0; w < S::kWarps; ++w)
    all = add(all, f2(part[w].x, part[w].y));
  split(all, a, b);
}

// Mean (0 where it is not wanted) and sum of squared deviations of two rows,
// 8 columns per thread (zeros where !k.on), on every thread.  Two passes over
// the warp's registers; the warps' parts are then put together: their own
// squares, and what their means differ from the row's.
struct Stats {
  float mu_a, mu_b, sq_a, sq_b;
};
template <int TPR, int NV>
__device__ __forceinline__ Stats row_stats(const F8 (&a)[NV], const F8 (&b)[NV],
                                           bool mean, const Cols<TPR, NV>& k,
                                           float4* part) {
  using S = Shape<TPR>;
  Stats st;
  st.mu_a = st.mu_b = 0.f;
  if (S::kMany && !mean) {  // squares alone
    F8 qa = mul(a[0], a[0]), qb = mul(b[0], b[0]);
#pragma unroll
    for (int i = 1; i < NV; ++i) {
      qa = fma(a[i], a[i], qa);
      qb = fma(b[i], b[i], qb);
    }
    st.sq_a = sum(qa);
    st.sq_b = sum(qb);
    row_sums<TPR>(st.sq_a, st.sq_b, reinterpret_cast<float2*>(part));
    return st;
  }
  if (mean) {
    F8 x = a[0], y = b[0];
#pragma unroll
    for (int i = 1; i < NV; ++i) {
      x = add(x, a[i]);
      y = add(y, b[i]);
    }
    st.mu_a = sum(x);
    st.mu_b = sum(y);
    both_sums<S::kLanes>(st.mu_a, st.mu_b);
    st.mu_a *= k.inv_warp;
    st.mu_b *= k.inv_warp;
  }
  F8 qa = splat(0.f), qb = qa;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (k.on(i)) {
      const F8 x = add(a[i], splat(-st.mu_a)), y = add(b[i], splat(-st.mu_b));
      qa = fma(x, x, qa);
      qb = fma(y, y, qb);
    }
  st.sq_a = sum(qa);
  st.sq_b = sum(qb);
  if constexpr (!S::kMany) {
    both_sums<S::kLanes>(st.sq_a, st.sq_b);
  } else {
    // part[w] = (mean of a, of b, squares of a, of b) in warp w
    const float v = keep_sums<32>(st.sq_a, st.sq_b);
    if (threadIdx.x % 16 == 0) {  // lane 0: of a, lane 16: of b
      float* to = reinterpret_cast<float*>(part + threadIdx.x / 32) +
                  (threadIdx.x & 16 ? 1 : 0);
      to[0] = threadIdx.x & 16 ? st.mu_b : st.mu_a;
      to[2] = v;
    }
    __syncthreads();
    F2 mu = f2(0.f), sq = f2(0.f);
#pragma unroll(S::kUnroll)
    for (int w = 0; w < S::kWarps; ++w) {
      const float4 x = part[w];
      mu = fma(f2(x.x, x.y), f2(k.counts[w]), mu);
      sq = add(sq, f2(x.z, x.w));
    }
    if (mean) {
      mu = mul(mu, f2(k.inv_dim));
      const F2 back = mul(mu, f2(-1.f));
#pragma unroll(S::kUnroll)
      for (int w = 0; w < S::kWarps; ++w) {
        const float4 x = part[w];
        const F2 d = add(f2(x.x, x.y), back);
        sq = fma(mul(d, f2(k.counts[w])), d, sq);
      }
    }
    split(mu, st.mu_a, st.mu_b);
    split(sq, st.sq_a, st.sq_b);
  }
  return st;
}

}  // namespace norm
}  // namespace fastvr
