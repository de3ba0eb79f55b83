// What the cross attention kernels share.
#pragma once

#include <cuda.h>
#include <stdint.h>

#include "fastvr_internal.h"

namespace fastvr {

bool cross_map(CUtensorMap* m, const void* base, int d, int tokens, int heads,
               int batch, const Strides& str, int32_t* batch_step);

// The kernel for few query rows (cross_attn_rows.cu).  32 rows: 12 heads over 2048
// keys 15.1 us against the tiles' 21.4, 16 streams of 8 key heads over 512 keys 18.9
// against 28.8, but 12 heads over 512 keys 11.1 against 8.1.  The rule goes by rows
// alone, so a few units of some rows over few keys take longer here than they had to,
// and a token of more than 32 query heads to a key head fills one row of a tile with
// each.
constexpr int kCrossRows = 16;  // rows of a block: tokens times shared heads
inline bool cross_few_rows(int64_t rows) { return rows <= 2 * kCrossRows; }
cudaError_t launch_cross_rows(const CrossArgs& a, cudaStream_t stream);

#ifdef __CUDACC__
// Keys that batch entry b sees.
__device__ __forceinline__ int cross_keys(const int32_t* kv_len, int b,
                                          int kv_tokens) {
  return kv_len == nullptr ? kv_tokens : min(max(kv_len[b], 0), kv_tokens);
}
#endif

}  // namespace fastvr
