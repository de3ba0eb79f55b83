// Warp-level products for the kernels of few rows, which are bound by memory and
// feed the tensor cores from registers.
#pragma once

#include <stdint.h>

namespace fastvr {

// c (16 x 8, float32) += a (16 x 16, bfloat16 rows) b (16 x 8, bfloat16
// columns).  With g = lane / 4 and t = lane % 4 a lane holds, as pairs,
//   a: (g, 2t), (g + 8, 2t), (g, 2t + 8), (g + 8, 2t + 8)
//   b: (2t, g), (2t + 8, g)   c: (g, 2t), (g, 2t + 1), (g + 8, 2t), (g + 8, 2t + 1)
// The summed axis may be in any order that a and b share: the callers give a
// lane 8 neighbouring elements (16 bytes) of it for two products, so both
// operands come straight from rows in memory.
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0,
                                            uint32_t a1, uint32_t a2,
                                            uint32_t a3, uint32_t b0,
                                            uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 "
      "{%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// 16 bytes that are read once.
__device__ __forceinline__ uint4 load_once(const void* p) {
  return __ldcs(reinterpret_cast<const uint4*>(p));
}

}  // namespace fastvr
