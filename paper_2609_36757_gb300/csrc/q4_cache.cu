// The 4-bit KV cache: quantising append and read-back.
//
// A group of 32 values along d stores a scale s = max |v| / 7 rounded to 5
// significant bits, and codes c = 8 + n with n the whole number nearest to
// v / s (ties toward zero), |n| <= 7.  With 5 bits of scale and 3 of
// magnitude every n s is an exact bfloat16.  Both kernels are bound by
// memory: the append reads 2 bytes and writes 0.5625 per value, the read-back
// the reverse.
#include <cuda_bf16.h>

#include "fastvr_internal.h"

namespace fastvr {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;

// max |v| of a group -> its scale (the stored bfloat16 as a float); a group
// below 2^-100 becomes zeros, one that is not finite or reaches 2^120 NaN.
__device__ __forceinline__ float group_scale(float top) {
  if (!(top < 0x1p120f)) return __int_as_float(0x7fc00000);
  if (top < 0x1p-100f) return 0.f;
  // Correctly rounded division: with 8 significant bits in top, top / 7 is
  // either exact or further from a 5-bit tie than its rounding error.
  const uint32_t u = __float_as_uint(__fdiv_rn(top, 7.f));
  const uint32_t odd = (u >> 19) & 1;
  return __uint_as_float((u + 0x3ffffu + odd) & 0xfff80000u);
}

// The code of v for scale s, r being 1 / s slightly reduced.  v has 8
// significant bits and s 5, so v / s is either exactly halfway between two
// whole numbers or at least 2^-14 of itself away from it; r = (1 - 2^-18) / s
// (and its rounding) moves an exact half below the half and nothing else
// across one, which rounds ties toward zero.
__device__ __forceinline__ uint32_t code(float v, float r) {
  // 1.5 * 2^23 + 8: adding it leaves 8 + round(v r) in the low bits
  return __float_as_uint(__fmaf_rn(v, r, 12582920.f)) & 15u;
}

template <int VPR>  // words (8 values) of a row: d / 8
__global__ void __launch_bounds__(kThreads) q4_append_kernel(Q4AppendParams p) {
  pdl_trigger();
  pdl_wait();
  const bool is_v = blockIdx.y != 0;
  const uint16_t* src = is_v ? p.v : p.k;
  const Strides& st = is_v ? p.v_str : p.k_str;
  uint32_t* codes = is_v ? p.v_codes : p.k_codes;
  uint16_t* scales = is_v ? p.v_scales : p.k_scales;
  const int64_t rows = (int64_t)p.batch * p.tokens * p.heads;
  const int64_t n = rows * VPR;
  const int64_t stride = (int64_t)gridDim.x * kThreads;
  // n and stride are multiples of 4 (VPR and kThreads are), so the four
  // lanes of a group are in range, or out of it, together.
  for (int64_t i0 = (int64_t)blockIdx.x * kThreads + threadIdx.x;;
       i0 += kUnroll * stride) {
    // warp-uniform: whole warps leave together (shuffles below)
    if (i0 - (threadIdx.x & 31) >= n) break;
    uint4 raw[kUnroll];
    int64_t row_out[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t i = i0 + u * stride;
      raw[u] = make_uint4(0, 0, 0, 0);
      row_out[u] = -1;
      if (i < n) {
        const int64_t row = i / VPR;
        const int32_t h = (int32_t)(row % p.heads);
        const int64_t bt = row / p.heads;
        const int64_t b = bt / p.tokens;
        const int64_t t = bt - b * p.tokens;
        raw[u] = __ldcs(reinterpret_cast<const uint4*>(
            src + b * st.batch + t * st.token + h * st.head + (i % VPR) * 8));
        int64_t at = p.first_row + t;
        if (at >= p.cache_tokens) at -= p.cache_tokens;
        row_out[u] = (b * p.heads + h) * p.cache_tokens + at;
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      float v[8];
      const uint32_t w[4] = {raw[u].x, raw[u].y, raw[u].z, raw[u].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        v[2 * e] = __uint_as_float(w[e] << 16);
        v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
      }
      // |v| as integers: their order is that of the magnitudes, and a NaN
      // compares above everything, so it reaches the scale
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float s = group_scale(__uint_as_float(top));
      const float r = s > 0.f ? (1.f - 0x1p-18f) / s : 0.f;
      uint32_t word = 0;
      if (s > 0.f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) word |= code(v[e], r) << (4 * e);
      } else {
        word = 0x88888888u;  // zeros, or NaN through the scale
      }
      if (row_out[u] >= 0) {
        const int word_i = (int)((i0 + u * stride) % VPR);
        constexpr int kGroups = VPR / 4;
        const int at = is_v ? word_i : (word_i % 4) * kGroups + word_i / 4;
        if (in_bounds(row_out[u] * VPR + at, p.code_words, p.status))
          codes[row_out[u] * VPR + at] = word;
        if (word_i % 4 == 0 &&
            in_bounds(row_out[u] * kGroups + word_i / 4,
                      p.code_words / 4, p.status))
          scales[row_out[u] * kGroups + word_i / 4] =
              (uint16_t)(__float_as_uint(s) >> 16);
      }
    }
  }
}

// 8 codes -> 8 bfloat16 values: a nibble y in bits 3..6 of a bfloat16 with
// the exponent of 16 is 16 + y, and (16 + y) s - 24 s = (y - 8) s, exact in
// one fused step (24 s has 7 significant bits).
__device__ __forceinline__ uint4 expand(uint32_t w, __nv_bfloat162 s) {
  const __nv_bfloat162 c =
      __hmul2(s, __floats2bfloat162_rn(-24.f, -24.f));
  uint32_t pr[4];  // (e, e + 4)
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t x = j == 0 ? w << 3 : w >> (4 * j - 3);
    const uint32_t m = (x & 0x00780078u) | 0x41804180u;
    const __nv_bfloat162 v =
        __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&m), s, c);
    pr[j] = *reinterpret_cast<const uint32_t*>(&v);
  }
  uint4 o;
  o.x = __byte_perm(pr[0], pr[1], 0x5410);
  o.y = __byte_perm(pr[2], pr[3], 0x5410);
  o.z = __byte_perm(pr[0], pr[1], 0x7632);
  o.w = __byte_perm(pr[2], pr[3], 0x7632);
  return o;
}

// kHeadMajor: rows in the order (b, h, t) of a head-major output, else
// (b, t, h); the output itself is given by its strides.
template <int VPR, bool kHeadMajor>
__global__ void __launch_bounds__(kThreads) q4_read_kernel(Q4ReadParams p) {
  pdl_trigger();
  pdl_wait();
  const bool is_v = blockIdx.y != 0;
  const uint32_t* codes = is_v ? p.v_codes : p.k_codes;
  const uint16_t* scales = is_v ? p.v_scales : p.k_scales;
  uint16_t* out = is_v ? p.v_out : p.k_out;
  constexpr int kGroups = VPR / 4;
  const int64_t n = (int64_t)p.batch * p.tokens * p.heads * VPR;
  const int64_t stride = (int64_t)gridDim.x * kThreads;
  for (int64_t i0 = (int64_t)blockIdx.x * kThreads + threadIdx.x; i0 < n;
       i0 += kUnroll * stride) {
    uint32_t w[kUnroll];
    uint16_t sc[kUnroll];
    int64_t dst[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t i = i0 + u * stride;
      dst[u] = -1;
      w[u] = 0x88888888u;
      sc[u] = 0;
      if (i >= n) continue;
      const int word = (int)(i % VPR);
      const int64_t row = i / VPR;
      int64_t b, t;
      int32_t h;
      if (kHeadMajor) {
        t = row % p.tokens;
        h = (int32_t)(row / p.tokens % p.heads);
        b = row / p.tokens / p.heads;
      } else {
        h = (int32_t)(row % p.heads);
        t = row / p.heads % p.tokens;
        b = row / p.heads / p.tokens;
      }
      dst[u] = b * p.out_str.batch + t * p.out_str.token +
               h * p.out_str.head + word * 8;
      if (p.first_chunk != nullptr) {
        // Tokens before the first visible one: those that share a key tile
        // with it are read back as zeros (they meet a weight of zero, which
        // a stored NaN or infinity would survive), earlier ones are skipped.
        const int64_t start = first_visible_token(p.first_chunk[b], p.lo_chunk,
                                                  p.chunk_tokens, p.tokens);
        if (t < start) {
          if (t < start / 128 * 128) dst[u] = -1;
          continue;
        }
      }
      int64_t at = p.first_row + t;
      if (at >= p.cache_tokens) at -= p.cache_tokens;
      const int64_t r = (b * p.heads + h) * p.cache_tokens + at;
      const int pos = is_v ? word : (word % 4) * kGroups + word / 4;
      if (in_bounds(r * VPR + pos, p.code_words, p.status)) {
        w[u] = codes[r * VPR + pos];
        sc[u] = scales[r * kGroups + word / 4];
      }
    }
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      if (dst[u] < 0) continue;
      const uint32_t s2 = sc[u] * 0x10001u;
      *reinterpret_cast<uint4*>(out + dst[u]) =
          expand(w[u], *reinterpret_cast<const __nv_bfloat162*>(&s2));
    }
  }
}

int grid_for(int64_t n, int sms) {
  int64_t blocks = (int64_t)sms * 4;
  const int64_t need = (n + kThreads - 1) / kThreads;
  if (blocks > need) blocks = need;
  return (int)blocks;
}

}  // namespace

cudaError_t launch_q4_append(const Q4AppendParams& p, int sms,
                             cudaStream_t stream) {
  const int vpr = p.head_dim / 8;
  const int64_t n = (int64_t)p.batch * p.tokens * p.heads * vpr;
  const dim3 grid(grid_for(n, sms), 2);
  if (vpr == 16)
    return launch_pdl(q4_append_kernel<16>, grid, dim3(kThreads), 0, stream, p);
  if (vpr == 8)
    return launch_pdl(q4_append_kernel<8>, grid, dim3(kThreads), 0, stream, p);
  return cudaErrorInvalidValue;
}

cudaError_t launch_q4_read(const Q4ReadParams& p, bool head_major, int sms,
                           cudaStream_t stream) {
  const int vpr = p.head_dim / 8;
  const int64_t n = (int64_t)p.batch * p.tokens * p.heads * vpr;
  const dim3 grid(grid_for(n, sms), 2);
  const dim3 block(kThreads);
  if (vpr == 16)
    return head_major
               ? launch_pdl(q4_read_kernel<16, true>, grid, block, 0, stream, p)
               : launch_pdl(q4_read_kernel<16, false>, grid, block, 0, stream, p);
  if (vpr == 8)
    return head_major
               ? launch_pdl(q4_read_kernel<8, true>, grid, block, 0, stream, p)
               : launch_pdl(q4_read_kernel<8, false>, grid, block, 0, stream, p);
  return cudaErrorInvalidValue;
}

}  // namespace fastvr
