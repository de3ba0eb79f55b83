// Pieces of the attention's gradient that the tile kernels share: probabilities
// and their gradients of a score tile's rows in registers.
#pragma once

#include <cuda_bf16.h>
#include <math.h>
#include <stdint.h>

namespace fastvr {
namespace grad {

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}

__device__ __forceinline__ uint64_t f2(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void f2_split(uint64_t v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ uint64_t f2_fma(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

// 2^x of both halves of a packed pair on the FMA pipe: x = n + f with n the
// nearest integer (x + 1.5 * 2^23 rounds it into the low mantissa bits) and
// f in [-0.5, 0.5]; 2^f by a degree-3 polynomial (a relative-error minimax
// fit on [-0.5, 0.5], at most 7.5e-5 relative error in fp32: far below the
// 2^-9 of the bf16 P it feeds), then times 2^n, whose exponent field is n's
// low bits.  x is first clamped to >= -126 so that the exponent cannot wrap
// (2^x there is below 1.2e-38, against 0 from ex2.approx.ftz); a NaN stays
// NaN in the clamp and, 2^n being a factor instead of an integer added to the
// result's bits, in what follows.  Some of the pairs take this path instead of
// MUFU ex2: the exponential step is bounded by the MUFU throughput, while the
// FMA pipe has room.
constexpr float kExpC0 = 0.9999281168f, kExpC1 = 0.6932609677f,
                kExpC2 = 0.2426105440f, kExpC3 = 0.0551713221f;
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void exp2_poly(float& x0, float& x1) {
  const uint64_t x = f2(max_nan(x0, -126.f), max_nan(x1, -126.f));
  const uint64_t t = f2_add(x, f2(12582912.f, 12582912.f));
  const uint64_t fr = f2_fma(f2_add(t, f2(-12582912.f, -12582912.f)),
                             f2(-1.f, -1.f), x);
  uint64_t q = f2_fma(f2(kExpC3, kExpC3), fr, f2(kExpC2, kExpC2));
  q = f2_fma(q, fr, f2(kExpC1, kExpC1));
  q = f2_fma(q, fr, f2(kExpC0, kExpC0));
  float t0, t1;
  f2_split(t, t0, t1);
  const uint32_t one = 0x3f800000u;  // 1.f, whose exponent n is added to
  f2_split(f2_mul(q, f2(__uint_as_float((__float_as_uint(t0) << 23) + one),
                        __uint_as_float((__float_as_uint(t1) << 23) + one))),
           x0, x1);
}
// Groups of four columns (of eight per 32) whose exponentials take the
// polynomial path in the unmasked step: one (training clip backward +0.5 %;
// two were slower, the FMA work then outweighing the MUFU it saves).
__device__ __forceinline__ constexpr bool poly_group(int q) { return q == 7; }

// P = 2^(s c2 - lse2) for 32 columns [c0, c0 + 32) of a half row, packed to
// bf16 pairs; with kMask, columns outside [lo, hi) are masked (p = 0).  nl
// holds -lse2 for the 32 columns, in registers: the dK/dV kernel reads its
// per-column values from shared memory ahead of use, because the SMEM x SMEM
// MMAs that run meanwhile take all of the shared-memory bandwidth and each
// read waits behind them.  The mask is a template argument, and the callers
// branch on a warp vote: a mask tested at run time inside the loop costs two
// compares and a select per element on every tile (measured: twice the time
// of the unmasked form), while only tiles that cross a chunk edge need it.
template <bool kMask>
__device__ __forceinline__ void p32(const uint32_t (&s)[32],
                                    const float4 (&nl)[8], int c0, int lo,
                                    int hi, uint64_t c2x2,
                                    uint32_t (&pp)[16]) {
#pragma unroll
  for (int q = 0; q < 8; ++q) {  // four columns at a time
    const float4 a = nl[q];
    float x[4];
    f2_split(f2_fma(f2(__uint_as_float(s[4 * q]), __uint_as_float(s[4 * q + 1])),
                    c2x2, f2(a.x, a.y)), x[0], x[1]);
    f2_split(f2_fma(f2(__uint_as_float(s[4 * q + 2]), __uint_as_float(s[4 * q + 3])),
                    c2x2, f2(a.z, a.w)), x[2], x[3]);
    if (kMask) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int col = c0 + 4 * q + u;
        if (col < lo || col >= hi) x[u] = -INFINITY;
      }
    }
    if (!kMask && poly_group(q)) {
      exp2_poly(x[0], x[1]);
      exp2_poly(x[2], x[3]);
      pp[2 * q] = pack_bf16(x[0], x[1]);
      pp[2 * q + 1] = pack_bf16(x[2], x[3]);
    } else {
      pp[2 * q] = pack_bf16(ex2(x[0]), ex2(x[1]));
      pp[2 * q + 1] = pack_bf16(ex2(x[2]), ex2(x[3]));
    }
  }
}

// dS = P (dP - D) for 32 columns: P as 16 bf16 pairs, dP fp32, nd holds -D
// for the 32 columns in registers.
__device__ __forceinline__ void ds32(const uint32_t (&pb)[16],
                                     const uint32_t (&dp)[32],
                                     const float4 (&nd)[8], uint32_t (&pd)[16]) {
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const float4 g = nd[q];
    float r[4];
    f2_split(f2_mul(f2(bf16_lo(pb[2 * q]), bf16_hi(pb[2 * q])),
                    f2_add(f2(__uint_as_float(dp[4 * q]),
                              __uint_as_float(dp[4 * q + 1])), f2(g.x, g.y))),
             r[0], r[1]);
    f2_split(f2_mul(f2(bf16_lo(pb[2 * q + 1]), bf16_hi(pb[2 * q + 1])),
                    f2_add(f2(__uint_as_float(dp[4 * q + 2]),
                              __uint_as_float(dp[4 * q + 3])), f2(g.z, g.w))),
             r[2], r[3]);
    pd[2 * q] = pack_bf16(r[0], r[1]);
    pd[2 * q + 1] = pack_bf16(r[2], r[3]);
  }
}

}  // namespace grad
}  // namespace fastvr
