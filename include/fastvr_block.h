/*
 * fastvr_block.h -- C ABI of the operators around the attention of a
 * streaming DiT block on GB300 (sm_103a): rotary positions, the gated
 * residual update fused with the norms before and after a block, and a KV
 * cache held in 4 bits with the attention that reads it.
 *
 * One block of a streaming model runs, per chunk,
 *   fastvr_gated_norm_fwd      residual update of the previous block and this
 *                              block's modulated norm
 *   (the caller's QKV projection)
 *   fastvr_rotary              positions on queries and keys
 *   fastvr_q4_append           keys and values into the 4-bit cache
 *   fastvr_q4_attn_fwd         the chunk's queries over the cache
 *   (the caller's output projection)
 * and training runs fastvr_gated_norm_bwd and fastvr_rotary (transpose = 1)
 * next to fastvr_blockcausal_attn_bwd.
 *
 * The conventions of fastvr_attn.h hold: the caller owns all device memory,
 * pointers are device addresses on the current device, 16-byte aligned unless
 * stated otherwise, work is enqueued on the given stream without
 * synchronising, errors are status codes, and a call that returns an error
 * enqueues no work.  There is no CPU fallback: every call that launches work
 * returns FASTVR_ERR_UNSUPPORTED on a device that is not sm_103.
 */
#ifndef FASTVR_BLOCK_H_
#define FASTVR_BLOCK_H_

#include "fastvr_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of the calls that take more than bfloat16 (the codes of
 * fastvr_one_step_update). */
#define FASTVR_BF16 0
#define FASTVR_F32 1

/* Strides of a [batch, token, head, d] tensor in elements; the d elements of
 * a head are contiguous.  Every stride (of a dimension with more than one
 * entry) is a multiple of 16 bytes; an output's is not 0. */
typedef struct {
  int64_t batch, token, head;
} fastvr_strides_t;

/* ------------------------------------------------------ rotary positions */

#define FASTVR_ROTARY_INTERLEAVED 0 /* pair i: elements 2i and 2i + 1       */
#define FASTVR_ROTARY_HALF 1        /* pair i: elements i and i + rot/2     */

#define FASTVR_SCALING_NONE 0
#define FASTVR_SCALING_LINEAR 1 /* theta / s                               */
#define FASTVR_SCALING_NTK 2    /* base * s^(n / (n - 1)) in place of base */
#define FASTVR_SCALING_YARN 3   /* by parts, see below                     */

#define FASTVR_ROTARY_MAX_AXES 3

/* The first rotary_dim elements of each head are rotated in pairs, the rest
 * pass through.  The rotary_dim / 2 pairs are cut into `axes` consecutive
 * sections (one for text, three for the time, height and width of a video),
 * each with its own coordinate of the token's position and its own ladder of
 * frequencies: pair i of an axis with n pairs turns by p * theta_i with
 *   theta_i = base^(-i / n)                                   (radians).
 * For contexts longer than the model was trained on, with s = factor[axis]:
 *   LINEAR  theta_i / s
 *   NTK     base replaced by base * s^(n / (n - 1)), for n > 1
 *   YARN    (1 - g) theta_i / s + g theta_i,
 *           g = clamp((C theta_i / 2 pi - beta_slow) / (beta_fast -
 *           beta_slow), 0, 1), C = original_context[axis]: pairs that turn
 *           often within the original context keep their frequency, slow
 *           ones are interpolated.  The ramp g is linear in the turns, as in
 *           the method's paper; models trained with a ramp that is linear in
 *           the pair's index have other frequencies in between.
 * Every rotated element is multiplied by `magnitude`; 0 stands for
 * 0.1 ln(max s) + 1 with YARN and for 1 otherwise. */
typedef struct {
  int32_t head_dim;   /* d: a multiple of 8, 8 .. 512                     */
  int32_t rotary_dim; /* even, 2 .. head_dim                              */
  int32_t layout;     /* FASTVR_ROTARY_*                                  */
  int32_t axes;       /* 1 .. 3                                           */
  int32_t section[FASTVR_ROTARY_MAX_AXES]; /* pairs of each axis (>= 1);
                                              their sum is rotary_dim / 2 */
  int32_t scaling;    /* FASTVR_SCALING_*                                 */
  double base;        /* > 1                                              */
  double factor[FASTVR_ROTARY_MAX_AXES];           /* s >= 1              */
  double original_context[FASTVR_ROTARY_MAX_AXES]; /* C > 0 (YARN)        */
  double beta_fast, beta_slow;                     /* fast > slow (YARN)  */
  double magnitude;   /* 0 = default                                      */
} fastvr_rotary_config_t;

/* The rotary_dim / 2 frequencies theta_i (radians per position) of cfg in
 * pair order, and its magnitude.  Host only.
 * Errors: INVALID_ARG. */
FASTVR_API fastvr_status_t fastvr_rotary_frequencies(
    const fastvr_rotary_config_t* cfg, double* theta, double* magnitude);

/* Rotate the queries and keys of a block: for every pair (a, b) of a head at
 * position p, with angle x = p theta,
 *   a' = m (a cos x - b sin x),  b' = m (b cos x + a sin x).
 * transpose != 0 applies the transposed matrix (sin negated): the gradient
 * of the operation, with q and k the gradients of its outputs.
 *   q, k       [batch, tokens, heads, d] and [batch, tokens, kv_heads, d] of
 *              `dtype` (FASTVR_BF16 or FASTVR_F32) with strides q_str, k_str
 *              (null: contiguous); k may be null with kv_heads = 0
 *   positions  int32 [batch, tokens, axes], pos_batch elements from one batch
 *              entry to the next (0: one set for the whole batch), 4-byte
 *              aligned; any int32 value
 *   q_out, k_out  the same shapes and type, strides q_out_str, k_out_str
 *              (null: contiguous).  An output may be its own input with the
 *              same strides (in place); no other overlap.
 * Arithmetic is float32, rounded once.  The angle is reduced exactly: the
 * turn p theta / 2 pi modulo 1 is formed in 64-bit fixed point, so long
 * contexts lose no accuracy.
 * Errors: INVALID_ARG, UNSUPPORTED (device), CUDA. */
FASTVR_API fastvr_status_t fastvr_rotary(
    const fastvr_rotary_config_t* cfg, int32_t batch, int32_t tokens,
    int32_t heads, int32_t kv_heads, int32_t dtype, const void* q,
    const fastvr_strides_t* q_str, const void* k,
    const fastvr_strides_t* k_str, const int32_t* positions,
    int64_t pos_batch, void* q_out, const fastvr_strides_t* q_out_str,
    void* k_out, const fastvr_strides_t* k_out_str, int32_t transpose,
    struct CUstream_st* stream);

/* ------------------------------------- norms, gate and residual of a block */

#define FASTVR_NORM_NONE 0
#define FASTVR_NORM_RMS 1   /* v / sqrt(mean(v^2) + eps)                    */
#define FASTVR_NORM_LAYER 2 /* (v - mean(v)) / sqrt(var(v) + eps)           */

/* Between two blocks of a DiT, y being the first block's output, x the
 * residual stream, every token t of a group g (tokens / groups consecutive
 * tokens, such as the tokens of a latent frame) with its gate, scale and
 * shift vectors:
 *   r = residual_scale x + gate_g o post(y)
 *   h = pre(r) o (1 + scale_g) + shift_g
 * post and pre are the norms above, each followed by an optional weight
 * vector (with post NONE post_weight is not used).  Tensors are contiguous
 * [batch, tokens, dim]. */
typedef struct {
  int32_t batch, tokens, dim; /* dim: a multiple of 8, 8 .. 8192;
                                 batch * tokens below 2^30                  */
  int32_t groups;             /* 1 .. tokens, divides tokens                */
  int32_t pre, post;          /* FASTVR_NORM_*; pre is RMS or LAYER         */
  int32_t residual_dtype;     /* x, r, dr, dx: FASTVR_BF16 or FASTVR_F32    */
  int32_t block_dtype;        /* y, h, dh, dy: FASTVR_BF16 or FASTVR_F32    */
  float eps;                  /* > 0                                        */
  float residual_scale;
} fastvr_norm_config_t;

/* The forward.  gate, scale, shift: float32 [batch, groups, dim], each
 * nullable (gate 1, scale 0, shift 0); pre_weight, post_weight: float32
 * [dim], nullable (1).  y null: no block output (r = residual_scale x; gate
 * and post are not used), as before the first block.  r null: not written.
 * h null: no norm (scale, shift, pre_weight are not used), as after the last
 * block; r and h are not both null.  r may be x (in place).  The norm is
 * taken of r before it is rounded.  Arithmetic is float32; mean and variance
 * are two passes over registers.
 * Errors: INVALID_ARG, UNSUPPORTED (device), CUDA. */
FASTVR_API fastvr_status_t fastvr_gated_norm_fwd(
    const fastvr_norm_config_t* cfg, const void* x, const void* y,
    const float* gate, const float* scale, const float* shift,
    const float* pre_weight, const float* post_weight, void* r, void* h,
    struct CUstream_st* stream);

/* Scratch bytes of fastvr_gated_norm_bwd for cfg: partial sums of the
 * gradients that sum over tokens.  Host only.  Errors: INVALID_ARG. */
FASTVR_API fastvr_status_t fastvr_gated_norm_bwd_scratch_bytes(
    const fastvr_norm_config_t* cfg, size_t* bytes);

/* Gradients.  r is the forward's r (its statistics are recomputed), y the
 * block output or null as in the forward.  dr, dh: gradients of r and h, one
 * of them nullable (zero).  Outputs: dx (residual type), dy (block type; null
 * when y is), and, each nullable, dgate, dscale, dshift float32
 * [batch, groups, dim] and dpre_weight, dpost_weight float32 [dim]:
 *   dn = dh o (1 + scale) o pre_weight,  d = dr + J_pre(r)^T dn
 *   dx = residual_scale d,  du = d o gate,  dy = J_post(y)^T (du o post_weight)
 *   dgate = sum d o post(y),  dscale = sum dh o pre(r),  dshift = sum dh,
 *   dpre_weight = sum dh o (1 + scale) o n(r),
 *   dpost_weight = sum du o n(y)       (n: the norm before its weight)
 * A gradient of the absent: dgate and dpost_weight need y, the latter a post
 * norm; dscale, dshift and dpre_weight need dh; they are zero otherwise.
 * Token sums are float32 in a fixed order (no atomics): repeated calls agree
 * bit for bit.  dx may be dr and dy may be dh (in place, equal types).
 * Errors: INVALID_ARG, CAPACITY (scratch), UNSUPPORTED (device), CUDA. */
FASTVR_API fastvr_status_t fastvr_gated_norm_bwd(
    const fastvr_norm_config_t* cfg, const void* dr, const void* dh,
    const void* r, const void* y, const float* gate, const float* scale,
    const float* pre_weight, const float* post_weight, void* dx, void* dy,
    float* dgate, float* dscale, float* dshift, float* dpre_weight,
    float* dpost_weight, void* scratch, size_t scratch_bytes,
    struct CUstream_st* stream);

/* ----------------------------------------------------- a KV cache in 4 bits
 *
 * The streaming cache of fastvr_attn.h with its keys and values in 4 bits:
 * 4.5 / 16 of the cache's memory, and of the bytes that a call with few queries
 * has to read.  Calls with many queries need a workspace that holds the visible
 * window in bfloat16, as large as the bfloat16 cache: memory is saved where
 * several caches (the layers of a model, streams in turn) share one.  The
 * values of a head are cut into groups of 32 along d; a group stores one scale
 * s and 32 codes c in 1 .. 15 and stands for the values (c - 8) s:
 *   s = max |v| / 7, rounded to 5 significant bits (ties to even),
 *   c = 8 + v / s rounded to the nearest whole number, ties toward zero,
 *       within -7 .. 7.
 * 5 bits of scale and 3 of magnitude make every (c - 8) s an exact bfloat16,
 * so attention over this cache is attention over a bfloat16 cache of those
 * values.  A group with max |v| < 2^-100 stores zeros; a group that holds a
 * NaN, an infinity or a magnitude of 2^120 or more stores s = NaN and reads
 * back as NaN.
 *
 * Layout: codes of K and of V, each [B, kv_heads, T, d/2] bytes with
 * T = S*k*N tokens (S slots as in fastvr_kv_cache_bytes), then their scales
 * bfloat16 [B, kv_heads, T, d/32], each region on a 256-byte boundary, then a
 * control block.  A 32-bit word holds 8 consecutive elements, the first in
 * the lowest bits.  The words of a V row are in order; word w = 4 i + c of a
 * K row (group i, c = 0..3) is stored at position (d/32) c + i. */

/* Bytes of cache and of workspace for cfg with kv_heads key/value heads
 * (cfg->heads query heads, a multiple of kv_heads: consecutive query heads
 * share one).  A head's cache holds fewer than 2^30 tokens, S*k*N, and a
 * chunk has fewer than 2^30 query rows per key head.  A workspace may serve
 * any number of plans whose calls do not overlap on the GPU; nothing is kept
 * in it between calls.
 * Host only.  Errors: INVALID_ARG, UNSUPPORTED (head_dim not 64 or 128). */
FASTVR_API fastvr_status_t fastvr_q4_cache_bytes(
    const fastvr_attn_config_t* cfg, int32_t kv_heads, size_t* bytes);
FASTVR_API fastvr_status_t fastvr_q4_workspace_bytes(
    const fastvr_attn_config_t* cfg, int32_t kv_heads, size_t* bytes);

/* Bind a 4-bit cache and a workspace (device memory, 256-byte aligned).  The
 * plan keeps the stream's state as fastvr_attn_plan's does, and
 * fastvr_plan_reset, _get_state, _set_state, _visible, _launch_count,
 * _destroy and fastvr_get_status take it; fastvr_kv_append and
 * fastvr_chunk_attn_fwd do not (INVALID_ARG), nor do the calls below take a
 * bfloat16 plan.
 * Stream capture: the plan's first call that launches work clears the control
 * block and cannot be a captured one (SEQUENCE, nothing is enqueued).  A
 * captured call keeps the chunk counter of its capture: replays append to, read
 * or attend to the same chunks, and do not move the plan's counter.
 * Errors: INVALID_ARG, UNSUPPORTED, CAPACITY (a buffer is too small). */
FASTVR_API fastvr_status_t fastvr_q4_plan(const fastvr_attn_config_t* cfg,
                                          int32_t kv_heads, void* cache,
                                          size_t cache_bytes, void* workspace,
                                          size_t workspace_bytes,
                                          fastvr_plan_t* out);

/* Quantise the next chunk's keys and values, bfloat16 [B, frames*N, kv_heads,
 * d] with strides k_str, v_str (null: contiguous), into the cache.  frames is
 * 1..k (fewer than k end the stream, as in fastvr_kv_append), or a multiple
 * m*k of k with m <= S: m whole chunks at once (a prefix).
 * Errors: INVALID_ARG, CAPACITY (more frames than k and not such a multiple;
 * past max_chunks), SEQUENCE, UNSUPPORTED, CUDA. */
FASTVR_API fastvr_status_t fastvr_q4_append(fastvr_plan_t plan, const void* k,
                                            const fastvr_strides_t* k_str,
                                            const void* v,
                                            const fastvr_strides_t* v_str,
                                            int32_t frames,
                                            struct CUstream_st* stream);

/* Attention of the newest chunk c over the cache: q bfloat16 [B, f_c*N,
 * heads, d] contiguous, out the same, lse nullable float32 [B, heads, f_c*N],
 * visibility as in fastvr_chunk_attn_fwd.  first_chunk, nullable, is a device
 * array int32 [B] (4-byte aligned): batch entry b sees no chunk before
 * first_chunk[b] (a stream that joined the batch then; any value).  An entry
 * whose first_chunk is later than c sees nothing: its out is 0 and its lse
 * -infinity.  What the cache holds at hidden places does not matter.  out
 * does not overlap q; magnitudes in q are below 2^100.
 * Calls with few query rows (frames * N * heads / kv_heads) read the codes
 * directly; longer ones first write the visible keys and values in bfloat16
 * to the workspace.  A plan whose chunks are all short needs a workspace of
 * a few MB only.  Either way the probabilities are rounded to bfloat16 before
 * their product with the values, and sums and log-sum-exp are float32.  A row
 * with a NaN score is NaN.
 * Errors: INVALID_ARG, SEQUENCE, UNSUPPORTED, CUDA. */
FASTVR_API fastvr_status_t fastvr_q4_attn_fwd(fastvr_plan_t plan,
                                              const void* q,
                                              const int32_t* first_chunk,
                                              void* out, float* lse,
                                              struct CUstream_st* stream);

/* The values that the cache holds for a chunk still in it (one of the last S
 * appended): k, v bfloat16 [B, f*N, kv_heads, d] contiguous.
 * Errors: INVALID_ARG, SEQUENCE (that chunk is not in the cache),
 * UNSUPPORTED, CUDA. */
FASTVR_API fastvr_status_t fastvr_q4_read(fastvr_plan_t plan, int64_t chunk,
                                          void* k, void* v,
                                          struct CUstream_st* stream);

#ifdef __cplusplus
}
#endif

#endif /* FASTVR_BLOCK_H_ */
