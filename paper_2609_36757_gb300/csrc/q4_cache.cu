// The 4-bit KV cache: quantising append and read-back.
//
// A group of 32 values along d stores a scale s = max |v| / 7 rounded to 5
// significant bits, and codes c = 8 + n with n the whole number nearest to
// v / s (ties toward zero), |n| <= 7.  With 5 bits of scale and 3 of
// magnitude every n s is an exact bfloat16.  Both kernels are bound by
// memory: the append reads 2 bytes and writes 0.5625 per value, the read-back
// the reverse.  For 3 x 8160 tokens of 24 heads of 128: 71 us (5.4 TB/s) and
// 65 us (5.9 TB/s).  The append issues in 73 % of the cycles, for the scale's
// exact rounding and the codes; the read-back waits for memory.
#include <cuda_bf16.h>

#include <algorithm>

#include "fastvr_internal.h"

namespace fastvr {
namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 4;      // tokens of a thread at once: append
constexpr int kReadUnroll = 8;  // and read-back, which loads 6 bytes for each

// A thread keeps one 16-byte piece of one head and walks over tokens, 4 or 8
// consecutive ones at a time: in the cache these are neighbouring rows, 256
// bytes of codes and a whole sector of scales (tokens far apart left every
// 64-byte row and 8-byte scale on a DRAM page of its own: 97 us for that
// read-back).  The groups of d / 8 threads that make
// up a row are numbered over the grid with the head fastest (token-major
// tensors: neighbouring groups touch neighbouring memory), or they all belong
// to one head (head-major ones).
struct Walk {
  int32_t slots;  // groups of threads along the tokens
  int32_t ctas;   // grid.x
};
Walk make_walk(int64_t tokens, int64_t lanes, int groups_per_cta,
               int64_t others, int unroll, int sms) {
  // Eight CTAs of 256 threads per SM in all.
  const int64_t target =
      std::max<int64_t>(1, (int64_t)sms * 8 * groups_per_cta / others);
  const int64_t units = (tokens + unroll - 1) / unroll;
  const int64_t passes = (units * lanes + target - 1) / target;
  Walk w;
  w.slots = (int32_t)((units + passes - 1) / passes);
  w.ctas = (int32_t)((w.slots * lanes + groups_per_cta - 1) / groups_per_cta);
  return w;
}

__device__ __forceinline__ float approx_rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// max |v| of a group -> its scale (the stored bfloat16 as a float); a group
// below 2^-100 becomes zeros, one that is not finite or reaches 2^120 NaN.
__device__ __forceinline__ float group_scale(float top) {
  // top / 7 correctly rounded by one residual step (division by a known
  // divisor, Brisebarre, Muller and Raina, 2004).  With 8 significant bits in
  // top, top / 7 is either exact or further from a 5-bit tie than the
  // rounding error.
  constexpr float kSeventh = 1.f / 7.f;
  const float q0 = top * kSeventh;
  const float q = __fmaf_rn(__fmaf_rn(-7.f, q0, top), kSeventh, q0);
  const uint32_t u = __float_as_uint(q);
  const uint32_t odd = (u >> 19) & 1;
  const float s = __uint_as_float((u + 0x3ffffu + odd) & 0xfff80000u);
  if (!(top < 0x1p120f)) return __int_as_float(0x7fc00000);
  return top < 0x1p-100f ? 0.f : s;
}

// The codes of 8 values for scale s, r being 1 / s slightly reduced.  v has 8
// significant bits and s 5, so v / s is either exactly halfway between two
// whole numbers or at least 2^-14 of itself away from it; r = (1 - 2^-18) / s
// (with the 2^-22 of an approximate reciprocal) moves an exact half below the
// half and nothing else across one, which rounds ties toward zero.
__device__ __forceinline__ uint32_t encode8(const uint32_t (&v)[4], float r) {
  // Adding 1.5 * 2^23 + 8 leaves 8 + round(v r) in the low bits of the float
  // 0x4b400000; the words are summed up shifted, and what the upper parts add
  // modulo 2^32 is taken off: 0x4b400000 * (1 + 16 + 256).  Two values to an
  // instruction: the low and the high halves of two words.
  uint64_t r2, big2;
  asm("mov.b64 %0, {%1, %1};" : "=l"(r2) : "f"(r));
  asm("mov.b64 %0, {%1, %1};" : "=l"(big2) : "f"(12582920.f));
  uint32_t n[8];
#pragma unroll
  for (int e = 0; e < 4; e += 2) {
    uint64_t lo, hi;
    asm("mov.b64 %0, {%1, %2};" : "=l"(lo) : "r"(v[e] << 16), "r"(v[e + 1] << 16));
    asm("mov.b64 %0, {%1, %2};"
        : "=l"(hi)
        : "r"(v[e] & 0xffff0000u), "r"(v[e + 1] & 0xffff0000u));
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(lo) : "l"(lo), "l"(r2), "l"(big2));
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(hi) : "l"(hi), "l"(r2), "l"(big2));
    asm("mov.b64 {%0, %1}, %2;" : "=r"(n[2 * e]), "=r"(n[2 * e + 2]) : "l"(lo));
    asm("mov.b64 {%0, %1}, %2;" : "=r"(n[2 * e + 1]), "=r"(n[2 * e + 3]) : "l"(hi));
  }
  uint32_t w = 0;
#pragma unroll
  for (int e = 7; e >= 0; --e) w = w * 16u + n[e];
  return w - (0x4b400000u + 0xb4000000u + 0x40000000u);
}

// blockIdx.y: V or K of batch entries y / 2, + gridDim.y / 2, ...
template <int VPR>  // words (8 values) of a row: d / 8
__global__ void __launch_bounds__(kThreads)
q4_append_kernel(const __grid_constant__ Q4AppendParams p, Walk walk) {
  constexpr int kGroups = VPR / 4;
  pdl_trigger();
  pdl_wait();
  const bool is_v = blockIdx.y & 1;
  const Strides st = is_v ? p.v_str : p.k_str;
  uint32_t* codes = is_v ? p.v_codes : p.k_codes;
  uint16_t* scales = is_v ? p.v_scales : p.k_scales;
  const int word = threadIdx.x % VPR;
  const int group = blockIdx.x * (kThreads / VPR) + threadIdx.x / VPR;
  const int slot = group / p.heads;
  const int h = group - slot * p.heads;
  const int at_word = is_v ? word : (word % 4) * kGroups + word / 4;
  const uint32_t cache_tokens = (uint32_t)p.cache_tokens;
  const uint32_t stride = (uint32_t)walk.slots * kUnroll;
  for (int b = blockIdx.y / 2; b < p.batch; b += gridDim.y / 2) {
    const uint16_t* base =
        (is_v ? p.v : p.k) + b * st.batch + h * st.head + word * 8;
    const int64_t head_row = ((int64_t)b * p.heads + h) * p.cache_tokens;
    // Every group of threads makes the same number of passes (shuffles
    // inside); a surplus group (slot >= slots) copies nothing.
    for (uint32_t t0 = 0; t0 < (uint32_t)p.tokens; t0 += stride) {
      const uint32_t t = t0 + slot * kUnroll;
      const uint16_t* src = base + (int64_t)t * st.token;
      const uint32_t left =
          slot < walk.slots && t < (uint32_t)p.tokens ? p.tokens - t : 0;
      uint4 raw[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        raw[u] = make_uint4(0, 0, 0, 0);
        if (u < left)
          raw[u] = __ldcs(reinterpret_cast<const uint4*>(src + u * st.token));
      }
      uint32_t at = (uint32_t)p.first_row + t;  // both below 2^30
      if (at >= cache_tokens) at -= cache_tokens;
      // rows of the pass from `wrap` on lie at the start of the head
      const uint32_t wrap = cache_tokens - at;
      const int64_t row0 = head_row + at;
      uint32_t* code_to = codes + row0 * VPR + at_word;
      uint16_t* scale_to = scales + row0 * kGroups + word / 4;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const uint32_t w[4] = {raw[u].x, raw[u].y, raw[u].z, raw[u].w};
        // |v| as 15-bit integers, two to a word: their order is that of the
        // magnitudes, and a NaN is above everything, so it reaches the scale
        uint32_t top = __vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu),
                                __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
        top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 2));
        top = max(top << 16, top & 0xffff0000u);
        const float s = group_scale(__uint_as_float(top));
        const float r = s > 0.f ? approx_rcp(s) * (1.f - 0x1p-18f) : 0.f;
        // zeros, also under a NaN scale
        const uint32_t code = s > 0.f ? encode8(w, r) : 0x88888888u;
        if (u < left) {
          const int64_t back = u < wrap ? 0 : p.cache_tokens;
          if (in_bounds((row0 + u - back) * VPR + at_word, p.code_words,
                        p.status)) {
            code_to[u * VPR - back * VPR] = code;
            if (word % 4 == 0)
              scale_to[u * kGroups - back * kGroups] =
                  (uint16_t)(__float_as_uint(s) >> 16);
          }
        }
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

// kHeadMajor: blockIdx.y walks over V or K of (batch entry, head) pairs and
// the groups of threads over tokens; else as the append.
template <int VPR, bool kHeadMajor>
__global__ void __launch_bounds__(kThreads)
q4_read_kernel(const __grid_constant__ Q4ReadParams p, Walk walk) {
  constexpr int kGroups = VPR / 4;
  pdl_trigger();
  pdl_wait();
  const bool is_v = blockIdx.y & 1;
  const uint32_t* codes = is_v ? p.v_codes : p.k_codes;
  const uint16_t* scales = is_v ? p.v_scales : p.k_scales;
  const int word = threadIdx.x % VPR;
  const int group = blockIdx.x * (kThreads / VPR) + threadIdx.x / VPR;
  const int slot = kHeadMajor ? group : group / p.heads;
  if (slot >= walk.slots) return;
  const int at_word = is_v ? word : (word % 4) * kGroups + word / 4;
  const int outer = kHeadMajor ? p.batch * p.heads : p.batch;
  for (int y = blockIdx.y / 2; y < outer; y += gridDim.y / 2) {
    const int b = kHeadMajor ? y / p.heads : y;
    const int h = kHeadMajor ? y - b * p.heads : group - slot * p.heads;
    uint16_t* out = (is_v ? p.v_out : p.k_out) + b * p.out_str.batch +
                    h * p.out_str.head + word * 8;
    const int64_t head_row = ((int64_t)b * p.heads + h) * p.cache_tokens;
    // Tokens before the first visible one: those that share a key tile with
    // it are read back as zeros (they meet a weight of zero, which a stored
    // NaN or infinity would survive), earlier ones are skipped.
    const int64_t start =
        p.first_chunk == nullptr
            ? 0
            : first_visible_token(p.first_chunk[b], p.lo_chunk, p.chunk_tokens,
                                  p.tokens);
    const uint32_t skip = (uint32_t)start / 128 * 128;
    const uint32_t cache_tokens = (uint32_t)p.cache_tokens;
    constexpr int U = kReadUnroll;
    const uint32_t stride = (uint32_t)walk.slots * U;
    for (uint32_t t0 = slot * U; t0 < (uint32_t)p.tokens; t0 += stride) {
      if (t0 + U <= skip) continue;
      uint32_t at = (uint32_t)p.first_row + t0;  // both below 2^30
      if (at >= cache_tokens) at -= cache_tokens;
      const uint32_t wrap = cache_tokens - at;
      const int64_t row0 = head_row + at;
      const uint32_t* code_at = codes + row0 * VPR + at_word;
      const uint16_t* scale_at = scales + row0 * kGroups + word / 4;
      uint32_t w[U], sc[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t t = t0 + u;
        w[u] = sc[u] = 0;
        const int64_t back = u < wrap ? 0 : p.cache_tokens;
        if (t >= (uint32_t)start && t < (uint32_t)p.tokens &&
            in_bounds((row0 + u - back) * VPR + at_word, p.code_words,
                      p.status)) {
          w[u] = __ldcs(code_at + u * VPR - back * VPR);
          sc[u] = scale_at[u * kGroups - back * kGroups];
        }
      }
      uint16_t* dst = out + (int64_t)t0 * p.out_str.token;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t t = t0 + u;
        if (t < skip || t >= (uint32_t)p.tokens) continue;
        const uint32_t s2 = sc[u] * 0x10001u;
        *reinterpret_cast<uint4*>(dst + u * p.out_str.token) =
            expand(w[u], *reinterpret_cast<const __nv_bfloat162*>(&s2));
      }
    }
  }
}

}  // namespace

cudaError_t launch_q4_append(const Q4AppendParams& p, int sms,
                             cudaStream_t stream) {
  const int vpr = p.head_dim / 8;
  if (vpr != 16 && vpr != 8) return cudaErrorInvalidValue;
  const int ys = std::min(p.batch, 32767);
  const Walk w = make_walk(p.tokens, p.heads, kThreads / vpr, 2 * ys,
                           kUnroll, sms);
  const dim3 grid(w.ctas, 2 * ys), block(kThreads);
  return vpr == 16 ? launch_pdl(q4_append_kernel<16>, grid, block, 0, stream, p,
                                w)
                   : launch_pdl(q4_append_kernel<8>, grid, block, 0, stream, p,
                                w);
}

cudaError_t launch_q4_read(const Q4ReadParams& p, bool head_major, int sms,
                           cudaStream_t stream) {
  const int vpr = p.head_dim / 8;
  if (vpr != 16 && vpr != 8) return cudaErrorInvalidValue;
  const int ys = std::min(head_major ? p.batch * p.heads : p.batch, 32767);
  const Walk w = make_walk(p.tokens, head_major ? 1 : p.heads, kThreads / vpr,
                           2 * ys, kReadUnroll, sms);
  const dim3 grid(w.ctas, 2 * ys), block(kThreads);
  if (vpr == 16)
    return head_major ? launch_pdl(q4_read_kernel<16, true>, grid, block, 0,
                                   stream, p, w)
                      : launch_pdl(q4_read_kernel<16, false>, grid, block, 0,
                                   stream, p, w);
  return head_major ? launch_pdl(q4_read_kernel<8, true>, grid, block, 0,
                                 stream, p, w)
                    : launch_pdl(q4_read_kernel<8, false>, grid, block, 0,
                                 stream, p, w);
}

}  // namespace fastvr
