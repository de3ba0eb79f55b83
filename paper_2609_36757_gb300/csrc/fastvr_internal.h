// Internal interfaces between the host library (fastvr_host.cpp) and the
// CUDA kernels.  Not part of the public ABI.
#pragma once

#include <cuda.h>  // CUtensorMap types (the driver itself is reached
                   // through the runtime's entry-point query)
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "vec_math.cuh"

namespace fastvr {

// At most two contiguous token ranges of one head's cache make up the keys a
// chunk sees: the visible chunk slots are consecutive modulo the ring size
// and only the newest chunk can be partly filled (Eq. 1 at chunk granularity,
// Sec. 3.1 KV caching).
constexpr int kMaxSegments = 2;

// Split-KV workspace of the attention kernel: at most kMaxParts partial
// results of 256 query rows, each d fp32 outputs plus one log-sum-exp.
constexpr int kMaxParts = 256;
constexpr int kUnitRows = 256;
inline size_t workspace_bytes(int head_dim) {
  return (size_t)kMaxParts * kUnitRows * (head_dim + 1) * sizeof(float);
}

// cuTensorMapEncodeTiled, looked up through the CUDA runtime's driver entry
// point (the library links the runtime statically and not libcuda); null
// when the driver does not provide it.
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType,
                                  cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled_fn();

// Error codes a kernel writes into the cache's control block.
constexpr int kDevOk = 0;
constexpr int kDevTimeout = 1;
constexpr int kDevBounds = 2;  // an index check (debug builds) or a layout
                               // check failed

#ifdef __CUDACC__
// Debug builds (-DFASTVR_BOUNDS_CHECK, libfastvr_attn_debug.so) check every
// computed global-memory index of the streaming path before the access: an
// index outside [0, n) records kDevBounds in the status word (the first
// error wins) and the access is skipped.  Release builds compile the check
// away.  compute-sanitizer is not available, and a trap or failed assert
// would take the GPU down with it.
#ifdef FASTVR_BOUNDS_CHECK
__device__ __forceinline__ bool in_bounds(int64_t i, int64_t n, int* status) {
  if (i >= 0 && i < n) return true;
  if (status != nullptr) atomicCAS(status, kDevOk, kDevBounds);
  return false;
}
#else
__device__ __forceinline__ bool in_bounds(int64_t, int64_t, int*) {
  return true;
}
#endif
#endif

#ifdef __CUDACC__
// Programmatic dependent launch.  The streaming kernels (append, attention,
// split merge) and the one-step update are launched with programmatic stream
// serialization, so a kernel may become resident and do its set-up (barrier
// and TMEM initialisation) while the previous kernel on the stream drains.
// Each of them executes pdl_wait() before its first global-memory access
// that a preceding kernel may produce or still read (the wait returns once
// that kernel has completed and its writes are visible), and pdl_trigger()
// early, so that the next kernel's launch can begin.
__device__ __forceinline__ void pdl_wait() {
  asm volatile("griddepcontrol.wait;" ::: "memory");
}
__device__ __forceinline__ void pdl_trigger() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

template <typename... KArgs, typename... Args>
inline cudaError_t launch_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block,
                              size_t smem, cudaStream_t stream,
                              Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, static_cast<Args&&>(args)...);
}
#endif

// Strided view of a bfloat16 [B, L, H, d] token-major tensor or of a head-major
// cache [B, H, L, d]: element (b, t, h, x) lives at
// base + b*batch + t*token + h*head + x (strides in elements).
struct Strides {
  int64_t batch, token, head;
};

struct AppendParams {
  const uint16_t* k_new;  // [B, L, H, d] token-major
  const uint16_t* v_new;
  uint16_t* k_cache;      // [B, H, cache_tokens, d] head-major
  uint16_t* v_cache;
  int32_t batch, tokens, heads, head_dim;
  int64_t cache_tokens;   // tokens per head in the cache (S * k * N)
  int64_t token_offset;   // first cache token of the destination slot
  int* status;            // control block word (bounds checks), or null
};

struct AttnParams {
  const uint16_t* q;      // bfloat16 [B, Lq, H, d] token-major
  uint16_t* o;            // bfloat16 [B, Lq, H, d] token-major
  float* lse;             // float32 [B, H, Lq] or null
  const uint16_t* k;      // keys: head-major cache view
  const uint16_t* v;      // values: same layout as k
  Strides q_str;          // strides of q and o
  Strides kv_str;         // strides of k and v
  int32_t batch, heads, head_dim, q_tokens;
  int64_t kv_tokens;      // tokens per head addressable through k/v
  int32_t num_segments;
  int64_t seg_start[kMaxSegments];
  int32_t seg_len[kMaxSegments];
  float scale_log2;       // softmax_scale * log2(e)
  int* status;            // control word (device)
  float* workspace;       // split-KV scratch (device): workspace_parts
                          // partial results of kUnitRows x (d + 1) floats
  int32_t workspace_parts;
  uint64_t wait_limit_ns; // bound of every in-kernel wait (0 = default)
  int32_t inject_stall;   // test hook: stall the MMA issuer until timeout
  int32_t kv_group;       // query heads that share a key head (0: 1)
  // Null, or the first chunk that each batch entry sees; the keys are then
  // one segment whose first token is that of chunk lo_chunk.
  const int32_t* first_chunk;
  int64_t lo_chunk;
  int32_t chunk_tokens;
};

cudaError_t launch_kv_append(const AppendParams& p, cudaStream_t stream);
// The one-step update z_hat = z - sigma * v over n elements; z and out are
// bf16 (dtype 0) or float32 (dtype 1), v is bf16.
cudaError_t launch_one_step(const void* z, const void* v, void* out, int64_t n,
                            float sigma, int dtype, cudaStream_t stream);

// One-shot (training-form) attention over a whole token-major sequence.
struct OneShotParams {
  const uint16_t* q;      // bfloat16 [B, L, H, d] token-major
  const uint16_t* k;
  const uint16_t* v;
  uint16_t* o;            // bfloat16 [B, L, H, d]
  float* lse;             // float32 [B, H, L] or null
  int32_t batch, heads, head_dim;
  int32_t seq_tokens;     // L = frames * tokens per frame
  int32_t chunk_tokens;   // k * N
  int32_t window;         // W, -1 = unbounded
  float scale_log2;
  int* status;            // device status word or null (not reported)
  int32_t inject_stall;   // failure-detection test hook
  uint64_t wait_limit_ns; // 0 = kernel default
};
cudaError_t launch_blockcausal_attn(const OneShotParams& p, cudaStream_t stream);

// Backward of the one-shot attention.
struct BwdArgs {
  const uint16_t *q, *k, *v, *out, *dout;  // bf16 [B, L, H, d] token-major
  const float* lse;                        // forward LSE [B, H, L]
  uint16_t *dq, *dk, *dv;                  // bf16 [B, L, H, d]
  float* scratch;  // 2 * B * H * round_up(L, 128) floats
  int32_t batch, heads, head_dim, seq_tokens, chunk_tokens, window;
  float scale;
  int* status;             // device status word or null (not reported)
  int32_t inject_stall;    // failure-detection test hook
  uint64_t wait_limit_ns;  // 0 = kernel default
};
cudaError_t launch_blockcausal_attn_bwd(const BwdArgs& a, cudaStream_t stream);

// The status word of the current device for the calls without a plan (the
// one-shot forward and the backward), or null if it cannot be looked up.
int* device_status_word();

// Workspace parts (partial results) a launch of p uses on the current device
// (0 when no unit is split), with at most kMaxParts parts.
int chunk_attn_parts(const AttnParams& p);
// Enqueues the attention kernel (and the merge kernel when the key range of
// some units is split); *launches receives the number of kernels enqueued.
cudaError_t launch_chunk_attn(const AttnParams& p, cudaStream_t stream,
                              int* launches);

// ------------------------------------------- operators around the attention
// (include/fastvr_block.h)

constexpr int kRotaryMaxPairs = 256;

struct RotaryArgs {
  const void *q, *k;       // [batch, tokens, heads | kv_heads, head_dim]
  void *q_out, *k_out;
  Strides q_str, k_str, q_out_str, k_out_str;
  const int32_t* positions;
  int64_t pos_batch;
  int32_t batch, tokens, heads, kv_heads, head_dim, pairs, axes, section[3];
  bool f32, half, transpose;
  float magnitude;
  int sms;
  const uint64_t* turn;  // pairs: theta / 2 pi in 2^-64 turns (host memory)
};
cudaError_t launch_rotary(const RotaryArgs& a, cudaStream_t stream);

constexpr int kNormNone = 0, kNormRms = 1, kNormLayer = 2;

struct NormFwdParams {
  const void *x, *y;
  const float *gate, *scale, *shift, *pre_weight, *post_weight;
  void *r, *h;
  int64_t rows, group_tokens;
  FastDiv by_group_tokens;
  int32_t dim, pre, post;
  float eps, residual_scale;
};
cudaError_t launch_norm_fwd(const NormFwdParams& p, bool res_f32,
                            bool block_f32, int sms, cudaStream_t stream);

struct NormBwdSplit {
  int32_t slices;      // CTAs that share a group, or 1
  int64_t cta_groups;  // whole groups of a CTA when slices is 1
  int64_t ctas;
};
NormBwdSplit norm_bwd_split(int64_t all_groups, int64_t group_tokens, int dim,
                            int sms);

struct NormBwdParams {
  const void *dr, *dh, *r, *y;
  const float *gate, *scale, *pre_weight, *post_weight;
  void *dx, *dy;
  float *dgate, *dscale, *dshift, *dpre_weight, *dpost_weight;
  float* partial;         // [ctas, 3, dim] when slices > 1
  float* weight_partial;  // [ctas, 2, dim], or null when neither is wanted
  int64_t all_groups, group_tokens, cta_groups, ctas;
  int32_t slices, dim, pre, post;
  float eps, residual_scale;
};
cudaError_t launch_norm_bwd(const NormBwdParams& p, bool res_f32,
                            bool block_f32, cudaStream_t stream);

// The 4-bit cache: codes [B, Hkv, cache_tokens, d/2] bytes, scales bfloat16
// [B, Hkv, cache_tokens, d/32], for K and for V.
struct Q4AppendParams {
  const uint16_t *k, *v;
  Strides k_str, v_str;
  uint32_t *k_codes, *v_codes;
  uint16_t *k_scales, *v_scales;
  int32_t batch, tokens, heads, head_dim;
  int64_t cache_tokens;
  int64_t first_row;   // cache row of the first token (rows wrap)
  int64_t code_words;  // 32-bit words of a code region (bounds checks)
  int* status;
};
cudaError_t launch_q4_append(const Q4AppendParams& p, int sms,
                             cudaStream_t stream);

struct Q4ReadParams {
  const uint32_t *k_codes, *v_codes;
  const uint16_t *k_scales, *v_scales;
  uint16_t *k_out, *v_out;
  Strides out_str;
  int32_t batch, tokens, heads, head_dim;
  int64_t cache_tokens, first_row, code_words;
  // Null, or the first visible chunk of each batch entry: see q4_cache.cu.
  const int32_t* first_chunk;
  int64_t lo_chunk, chunk_tokens;
  int* status;
};
cudaError_t launch_q4_read(const Q4ReadParams& p, bool head_major, int sms,
                           cudaStream_t stream);

// Whether a call goes straight over the codes (q4_attn.cu) or first writes the
// visible keys and values in bfloat16 to the workspace and runs the tile
// kernel over them.  Per key and key head the former takes about 0.06 ns and
// 0.07 for every 32 query rows (tokens times query heads per key head), the
// latter 0.17 to expand and 0.04 for every query head and 256 tokens: 12 heads
// over 32768 keys take 50.9 us directly with 32 rows, 75.6 with 64 and 84 the
// other way, 8 streams of 32 heads over 8 and 8192 keys 144 us with 96 rows,
// 182 with 128 and 178.  The few keys of a short window leave the direct way's
// shares too small for its second block to pay (4096 keys: 26.8 us with 64 rows
// against 19.4), hence the 8.
inline bool q4_direct(int64_t q_tokens, int64_t group) {
  const int64_t blocks = (q_tokens * group + 31) / 32;
  return 8 + 7 * blocks < 17 + 4 * group * ((q_tokens + 255) / 256);
}
constexpr int kQ4MaxCtas = 512;               // of a launch
constexpr int kQ4MaxParts = 2 * kQ4MaxCtas;   // partial results, two per CTA
constexpr int kQ4PartRows = 32;               // rows of the largest row block
inline size_t q4_partial_bytes(int head_dim) {
  return (size_t)kQ4MaxParts * kQ4PartRows * (head_dim + 2) * sizeof(float);
}
struct Q4AttnParams {
  const uint16_t* q;  // [B, q_tokens, heads, d]
  uint16_t* out;
  float* lse;
  const uint8_t *k_codes, *v_codes, *k_scales, *v_scales;
  const int32_t* first_chunk;
  float* partial;  // kQ4MaxParts parts of kQ4PartRows rows of d + 2
  int* tickets;    // kQ4MaxCtas counters, zero between calls
  int32_t batch, heads, kv_heads, head_dim, q_tokens;
  int32_t group;   // query heads per key head
  int32_t rows;    // q_tokens * group
  int64_t cache_tokens, first_row;  // first_row: oldest visible token's row
  int64_t keys;                     // visible tokens
  int64_t lo_chunk, chunk_tokens;
  float scale_log2;
  int32_t row_blocks;               // filled in by the launch
};
cudaError_t launch_q4_attn(const Q4AttnParams& p, int sms,
                           cudaStream_t stream);

// ------------------------------------------- cross attention, feed-forward

#ifdef __CUDACC__
// Dynamic shared memory of a kernel past 48 KB, set once per device: a decode
// step's host time counts, and the runtime call costs about a microsecond.
template <auto kKernel>
inline cudaError_t allow_smem(int bytes, int device) {
  static std::atomic<uint64_t> done{0};
  const uint64_t bit = device >= 0 && device < 64 ? 1ull << device : 0;
  if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(
      kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}
#endif

struct CrossArgs {
  const uint16_t *q, *k, *v;  // bfloat16, strides in elements
  uint16_t* o;
  float* lse;                 // [batch, heads, q_tokens] or null
  Strides q_str, k_str, v_str, o_str;
  const int32_t* kv_len;      // [batch] or null
  int32_t batch, heads, kv_heads, head_dim, q_tokens, kv_tokens;
  float scale;
  int* status;                // device status word or null (not reported)
  int32_t inject_stall;       // failure-detection test hook
  uint64_t wait_limit_ns;     // 0 = kernel default
  int sms, device;
};
cudaError_t launch_cross_attn(const CrossArgs& a, cudaStream_t stream);

struct CrossBwdArgs {
  CrossArgs f;                // the forward's arguments (o and lse: results)
  const uint16_t* dout;
  uint16_t *dq, *dk, *dv;
  Strides dout_str, dq_str, dk_str, dv_str;
  float* scratch;             // cross_bwd_scratch_floats of them
};
size_t cross_bwd_scratch_floats(int32_t batch, int32_t heads, int32_t kv_heads,
                                int32_t head_dim, int32_t q_tokens,
                                int32_t kv_tokens);
cudaError_t launch_cross_attn_bwd(const CrossBwdArgs& a, cudaStream_t stream);

constexpr int kActSilu = 0, kActGelu = 1, kActGeluTanh = 2;

struct FfnArgs {
  const uint16_t *x, *w_gate, *w_up;  // [tokens, dim], [hidden, dim] twice
  int64_t x_row;                      // elements from row to row of x
  uint16_t *h, *g, *u;                // [tokens, hidden]; g, u nullable
  int32_t tokens, dim, hidden, act;
  int* status;
  int32_t inject_stall;
  uint64_t wait_limit_ns;
  int sms, device;
};
cudaError_t launch_ffn_fwd(const FfnArgs& a, cudaStream_t stream);

struct FfnBwdArgs {
  FfnArgs f;                    // the forward's arguments (h is not used)
  const uint16_t* dh;           // [tokens, hidden]
  uint16_t *dx, *dw_gate, *dw_up;
  uint16_t *dg, *du;            // scratch: [tokens, hidden] each
};
cudaError_t launch_ffn_bwd(const FfnBwdArgs& a, cudaStream_t stream);

#ifdef __CUDACC__
// The first of `keys` tokens (counted from the start of chunk lo_chunk) that
// a batch entry sees when nothing before chunk first_chunk is visible to it.
__device__ __forceinline__ int64_t first_visible_token(int32_t first_chunk,
                                                       int64_t lo_chunk,
                                                       int64_t chunk_tokens,
                                                       int64_t keys) {
  const int64_t hidden = (int64_t)first_chunk - lo_chunk;
  if (hidden <= 0) return 0;
  // hidden * chunk_tokens < 2^31 * 2^31
  const int64_t t = hidden * chunk_tokens;
  return t < keys ? t : keys;
}
#endif

}  // namespace fastvr
