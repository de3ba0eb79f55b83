// Host side of the operators around the attention: the C ABI declared in
// include/fastvr_block.h.  Argument checks, the rotary frequencies, the
// 4-bit plan's layout and the choice of kernels; the device work is in
// rotary.cu, block_norm_fwd.cu, block_norm_bwd.cu, q4_cache.cu and q4_attn.cu.
#include "../../include/fastvr_block.h"

#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <new>

#include "fastvr_internal.h"
#include "fastvr_plan.h"

namespace {

using fastvr::aligned16;

bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }

cudaStream_t to_stream(struct CUstream_st* s) {
  return reinterpret_cast<cudaStream_t>(s);
}

// a * b, or -1 when it does not fit (or a factor already did not).
int64_t mul(int64_t a, int64_t b) {
  int64_t r;
  return a < 0 || b < 0 || __builtin_mul_overflow(a, b, &r) ? -1 : r;
}

// ------------------------------------------------------------------ rotary
constexpr double kTwoPi = 6.283185307179586476925286766559;

bool valid_rotary(const fastvr_rotary_config_t* c) {
  if (c == nullptr || c->head_dim < 8 || c->head_dim > 512 ||
      c->head_dim % 8 != 0 || c->rotary_dim < 2 || c->rotary_dim % 2 != 0 ||
      c->rotary_dim > c->head_dim || c->axes < 1 ||
      c->axes > FASTVR_ROTARY_MAX_AXES || !(c->base > 1.0) ||
      !isfinite(c->base) || !(c->magnitude >= 0.0) ||
      !isfinite(c->magnitude) || c->scaling < FASTVR_SCALING_NONE ||
      c->scaling > FASTVR_SCALING_YARN ||
      (c->layout != FASTVR_ROTARY_INTERLEAVED &&
       c->layout != FASTVR_ROTARY_HALF))
    return false;
  int64_t pairs = 0;
  for (int a = 0; a < c->axes; ++a) {
    if (c->section[a] < 1) return false;
    pairs += c->section[a];
    if (c->scaling != FASTVR_SCALING_NONE &&
        (!(c->factor[a] >= 1.0) || !isfinite(c->factor[a])))
      return false;
    if (c->scaling == FASTVR_SCALING_YARN &&
        (!(c->original_context[a] > 0.0) || !isfinite(c->original_context[a])))
      return false;
  }
  if (c->scaling == FASTVR_SCALING_YARN &&
      (!(c->beta_fast > c->beta_slow) || !isfinite(c->beta_fast) ||
       !isfinite(c->beta_slow)))
    return false;
  return pairs == c->rotary_dim / 2;
}

void rotary_frequencies(const fastvr_rotary_config_t& c, double* theta,
                        double* magnitude) {
  double top = 1.0;
  int at = 0;
  for (int a = 0; a < c.axes; ++a) {
    const double n = c.section[a];
    const double s = c.scaling == FASTVR_SCALING_NONE ? 1.0 : c.factor[a];
    top = std::max(top, s);
    double base = c.base;
    if (c.scaling == FASTVR_SCALING_NTK && c.section[a] > 1)
      base *= pow(s, n / (n - 1.0));
    for (int i = 0; i < c.section[a]; ++i) {
      double f = pow(base, -(double)i / n);
      if (c.scaling == FASTVR_SCALING_LINEAR) f /= s;
      if (c.scaling == FASTVR_SCALING_YARN) {
        const double turns = c.original_context[a] * f / kTwoPi;
        const double keep = std::min(
            1.0,
            std::max(0.0, (turns - c.beta_slow) / (c.beta_fast - c.beta_slow)));
        f = (1.0 - keep) * f / s + keep * f;
      }
      theta[at++] = f;
    }
  }
  *magnitude = c.magnitude != 0.0 ? c.magnitude
               : c.scaling == FASTVR_SCALING_YARN ? 0.1 * log(top) + 1.0
                                                  : 1.0;
}

// Turns per position and magnitude of a config.  A program calls with the
// same config step after step and a decode step's host time counts, so each
// host thread keeps what it computed for its last config (compared by value).
struct RotaryTurns {
  fastvr_rotary_config_t cfg;
  bool valid = false;
  float magnitude;
  uint64_t turn[fastvr::kRotaryMaxPairs];
};
const RotaryTurns& rotary_turns(const fastvr_rotary_config_t& c) {
  static thread_local RotaryTurns last;
  if (!last.valid || memcmp(&last.cfg, &c, sizeof(c)) != 0) {
    double theta[fastvr::kRotaryMaxPairs], magnitude;
    rotary_frequencies(c, theta, &magnitude);
    last.cfg = c;
    last.valid = true;
    last.magnitude = (float)magnitude;
    // theta <= 1, so theta / 2 pi < 1 and the product fits 64 bits
    for (int i = 0; i < c.rotary_dim / 2; ++i)
      last.turn[i] = (uint64_t)(theta[i] / kTwoPi * 18446744073709551616.0);
  }
  return last;
}

// Strides in elements that keep every head 16-byte aligned; those of a
// dimension of one entry do not matter.  A tensor that is written may not have
// several entries in one place.
bool get_strides(const fastvr_strides_t* s, int64_t batch, int64_t tokens,
                 int64_t heads, int64_t d, int elem_bytes, bool written,
                 fastvr::Strides* out) {
  if (s == nullptr) {
    out->head = d;
    out->token = heads * d;
    out->batch = tokens * heads * d;
    return true;
  }
  const int64_t size[] = {batch, tokens, heads};
  const int64_t given[] = {s->batch, s->token, s->head};
  int64_t* to[] = {&out->batch, &out->token, &out->head};
  for (int i = 0; i < 3; ++i) {
    *to[i] = size[i] > 1 ? given[i] : 0;
    if (*to[i] % (16 / elem_bytes) != 0) return false;
    if (written && size[i] > 1 && given[i] == 0) return false;
  }
  return true;
}

// ------------------------------------------------------------------- norms
bool valid_norm(const fastvr_norm_config_t* c) {
  return c != nullptr && c->batch > 0 && c->tokens > 0 && c->dim >= 8 &&
         c->dim <= 8192 && c->dim % 8 == 0 && c->groups > 0 &&
         c->tokens % c->groups == 0 &&
         (c->pre == FASTVR_NORM_RMS || c->pre == FASTVR_NORM_LAYER) &&
         c->post >= FASTVR_NORM_NONE && c->post <= FASTVR_NORM_LAYER &&
         (c->residual_dtype == FASTVR_BF16 ||
          c->residual_dtype == FASTVR_F32) &&
         (c->block_dtype == FASTVR_BF16 || c->block_dtype == FASTVR_F32) &&
         c->eps > 0.f && isfinite(c->eps) && isfinite(c->residual_scale) &&
         (int64_t)c->batch * c->tokens <= INT32_MAX / 2;
}

// CTAs of the backward do not depend on the device at hand: the scratch size
// is asked for on the host, possibly without one.
constexpr int kNormSms = 152;

struct BwdLayout {
  fastvr::NormBwdSplit split;
  size_t partial, weights;  // bytes
};
BwdLayout norm_bwd_layout(const fastvr_norm_config_t& c) {
  BwdLayout l;
  const int64_t groups = (int64_t)c.batch * c.groups;
  l.split = fastvr::norm_bwd_split(groups, c.tokens / c.groups, c.dim, kNormSms);
  l.partial = l.split.slices > 1
                  ? (size_t)l.split.ctas * 3 * c.dim * sizeof(float)
                  : 0;
  l.weights = (size_t)l.split.ctas * 2 * c.dim * sizeof(float);
  return l;
}

// -------------------------------------------------------------- 4-bit cache
constexpr size_t kQ4ControlBytes =
    fastvr::kControlBytes + fastvr::kQ4MaxCtas * sizeof(int);

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// Sizes of a 4-bit plan; status other than OK when the config is refused.
struct Q4Layout {
  int64_t slots, slot_tokens, cache_tokens;
  size_t codes, scales;  // one region
  size_t cache, workspace;
};
fastvr_status_t q4_layout(const fastvr_attn_config_t* c, int32_t kv_heads,
                          Q4Layout* l) {
  if (!fastvr::valid_config(c) || kv_heads < 1 || c->heads % kv_heads != 0)
    return FASTVR_ERR_INVALID_ARG;
  if (!fastvr::supported_dim(c->head_dim)) return FASTVR_ERR_UNSUPPORTED;
  l->slots = fastvr::num_slots(*c);
  l->slot_tokens = mul(c->frames_per_chunk, c->tokens_per_frame);
  l->cache_tokens = mul(l->slots, l->slot_tokens);
  const int64_t rows = mul(l->slot_tokens, c->heads / kv_heads);
  const int64_t values =
      mul(mul(mul(c->batch, kv_heads), l->cache_tokens), c->head_dim);
  // Token indices are 32-bit in places, byte offsets are 64-bit.
  if (l->cache_tokens < 1 || l->cache_tokens > INT32_MAX / 2 || rows < 1 ||
      rows > INT32_MAX / 2 || values < 1 || values > (int64_t)1 << 46 ||
      mul(c->batch, c->heads) > INT32_MAX / 2)
    return FASTVR_ERR_INVALID_ARG;
  l->codes = round256((size_t)values / 2);
  l->scales = round256((size_t)values / 32 * 2);
  l->cache = 2 * l->codes + 2 * l->scales + kQ4ControlBytes;
  l->workspace = round256(fastvr::q4_partial_bytes(c->head_dim));
  if (!fastvr::q4_direct(l->slot_tokens, c->heads / kv_heads))
    l->workspace =
        std::max(l->workspace, 2 * round256((size_t)values * 2) +
                                   fastvr::workspace_bytes(c->head_dim));
  return FASTVR_OK;
}

fastvr_status_t ready(fastvr_plan_s* p, struct CUstream_st* stream) {
  return fastvr::ensure_device(p, kQ4ControlBytes, stream);
}

// Regions of a plan's cache.
uint8_t* codes_of(const fastvr_plan_s* p, bool v) {
  return reinterpret_cast<uint8_t*>(p->base) + (v ? p->code_bytes : 0);
}
uint8_t* scales_of(const fastvr_plan_s* p, bool v) {
  return reinterpret_cast<uint8_t*>(p->base) + 2 * p->code_bytes +
         (v ? p->scale_bytes : 0);
}

void fill_read(const fastvr_plan_s* p, fastvr::Q4ReadParams* r) {
  memset(r, 0, sizeof(*r));
  r->k_codes = reinterpret_cast<const uint32_t*>(codes_of(p, false));
  r->v_codes = reinterpret_cast<const uint32_t*>(codes_of(p, true));
  r->k_scales = reinterpret_cast<const uint16_t*>(scales_of(p, false));
  r->v_scales = reinterpret_cast<const uint16_t*>(scales_of(p, true));
  r->batch = p->cfg.batch;
  r->heads = p->kv_heads;
  r->head_dim = p->cfg.head_dim;
  r->cache_tokens = p->cache_tokens;
  r->code_words = (int64_t)p->cfg.batch * p->kv_heads * p->cache_tokens *
                  p->cfg.head_dim / 8;
  r->status = fastvr::control_word(p);
}

// The visible keys and values in bfloat16 into the workspace, oldest first,
// then the tile kernel over them.
cudaError_t attend_expanded(fastvr_plan_s* p, const fastvr::Q4AttnParams& d,
                            cudaStream_t stream) {
  fastvr::Q4ReadParams r;
  fill_read(p, &r);
  const int hd = d.head_dim;
  const size_t region =
      round256((size_t)r.batch * r.heads * p->cache_tokens * hd * 2);
  r.k_out = reinterpret_cast<uint16_t*>(p->workspace);
  r.v_out = reinterpret_cast<uint16_t*>(p->workspace + region);
  r.tokens = (int32_t)d.keys;
  r.out_str.token = hd;
  r.out_str.head = d.keys * hd;
  r.out_str.batch = r.heads * r.out_str.head;
  r.first_row = d.first_row;
  r.first_chunk = d.first_chunk;
  r.lo_chunk = d.lo_chunk;
  r.chunk_tokens = d.chunk_tokens;
  cudaError_t e =
      fastvr::launch_q4_read(r, true, fastvr::device_sms(), stream);
  if (e != cudaSuccess) return e;
  p->launches += 1;

  fastvr::AttnParams a;
  memset(&a, 0, sizeof(a));
  a.q = d.q;
  a.o = d.out;
  a.lse = d.lse;
  a.k = r.k_out;
  a.v = r.v_out;
  a.batch = r.batch;
  a.heads = d.heads;
  a.head_dim = hd;
  a.q_tokens = d.q_tokens;
  a.q_str.head = hd;
  a.q_str.token = (int64_t)d.heads * hd;
  a.q_str.batch = (int64_t)d.q_tokens * d.heads * hd;
  a.kv_str = r.out_str;
  a.kv_tokens = d.keys;
  a.num_segments = 1;
  a.seg_len[0] = (int32_t)d.keys;
  a.scale_log2 = d.scale_log2;
  a.status = fastvr::control_word(p);
  a.workspace = reinterpret_cast<float*>(p->workspace + 2 * region);
  a.workspace_parts = fastvr::kMaxParts;
  a.wait_limit_ns = p->wait_limit_ns;
  a.inject_stall = p->inject_stall;
  a.kv_group = d.group;
  a.first_chunk = d.first_chunk;
  a.lo_chunk = d.lo_chunk;
  a.chunk_tokens = (int32_t)d.chunk_tokens;
  int launched = 0;
  e = fastvr::launch_chunk_attn(a, stream, &launched);
  p->launches += launched;
  return e;
}

}  // namespace

extern "C" {

fastvr_status_t fastvr_rotary_frequencies(const fastvr_rotary_config_t* cfg,
                                          double* theta, double* magnitude) {
  if (!valid_rotary(cfg) || theta == nullptr || magnitude == nullptr)
    return FASTVR_ERR_INVALID_ARG;
  rotary_frequencies(*cfg, theta, magnitude);
  return FASTVR_OK;
}

fastvr_status_t fastvr_rotary(
    const fastvr_rotary_config_t* cfg, int32_t batch, int32_t tokens,
    int32_t heads, int32_t kv_heads, int32_t dtype, const void* q,
    const fastvr_strides_t* q_str, const void* k,
    const fastvr_strides_t* k_str, const int32_t* positions,
    int64_t pos_batch, void* q_out, const fastvr_strides_t* q_out_str,
    void* k_out, const fastvr_strides_t* k_out_str, int32_t transpose,
    struct CUstream_st* stream) {
  if (!valid_rotary(cfg) || batch < 1 || tokens < 1 || heads < 1 ||
      kv_heads < 0 || (dtype != FASTVR_BF16 && dtype != FASTVR_F32) ||
      q == nullptr || q_out == nullptr || !aligned16(q) || !aligned16(q_out) ||
      positions == nullptr || !aligned4(positions))
    return FASTVR_ERR_INVALID_ARG;
  if ((k == nullptr) != (kv_heads == 0) || (k_out == nullptr) != (k == nullptr) ||
      !aligned16(k) || !aligned16(k_out))
    return FASTVR_ERR_INVALID_ARG;
  // the items of a token (heads x vectors) are counted in 32 bits
  if (mul((int64_t)heads + kv_heads, cfg->head_dim) > (1 << 30) ||
      mul(batch, tokens) > (int64_t)INT32_MAX)
    return FASTVR_ERR_INVALID_ARG;
  const int es = dtype == FASTVR_F32 ? 4 : 2;
  fastvr::RotaryArgs a;
  const int d = cfg->head_dim;
  if (!get_strides(q_str, batch, tokens, heads, d, es, false, &a.q_str) ||
      !get_strides(q_out_str, batch, tokens, heads, d, es, true,
                   &a.q_out_str) ||
      !get_strides(k_str, batch, tokens, kv_heads, d, es, false, &a.k_str) ||
      !get_strides(k_out_str, batch, tokens, kv_heads, d, es, true,
                   &a.k_out_str))
    return FASTVR_ERR_INVALID_ARG;
  const fastvr_status_t st = fastvr::check_device();
  if (st != FASTVR_OK) return st;
  a.q = q;
  a.k = k;
  a.q_out = q_out;
  a.k_out = k_out;
  a.positions = positions;
  a.pos_batch = pos_batch;
  a.batch = batch;
  a.tokens = tokens;
  a.heads = heads;
  a.kv_heads = kv_heads;
  a.head_dim = cfg->head_dim;
  a.pairs = cfg->rotary_dim / 2;
  a.axes = cfg->axes;
  for (int i = 0; i < FASTVR_ROTARY_MAX_AXES; ++i)
    a.section[i] = i < cfg->axes ? cfg->section[i] : 0;
  a.f32 = dtype == FASTVR_F32;
  a.half = cfg->layout == FASTVR_ROTARY_HALF;
  a.transpose = transpose != 0;
  a.sms = fastvr::device_sms();
  const RotaryTurns& turns = rotary_turns(*cfg);
  a.magnitude = turns.magnitude;
  a.turn = turns.turn;
  return fastvr::launch_rotary(a, to_stream(stream)) == cudaSuccess
             ? FASTVR_OK
             : FASTVR_ERR_CUDA;
}

fastvr_status_t fastvr_gated_norm_fwd(
    const fastvr_norm_config_t* cfg, const void* x, const void* y,
    const float* gate, const float* scale, const float* shift,
    const float* pre_weight, const float* post_weight, void* r, void* h,
    struct CUstream_st* stream) {
  if (!valid_norm(cfg) || x == nullptr || (r == nullptr && h == nullptr))
    return FASTVR_ERR_INVALID_ARG;
  const void* ptrs[] = {x, y, gate, scale, shift, pre_weight, post_weight,
                        r, h};
  for (const void* ptr : ptrs)
    if (!aligned16(ptr)) return FASTVR_ERR_INVALID_ARG;
  const fastvr_status_t st = fastvr::check_device();
  if (st != FASTVR_OK) return st;
  fastvr::NormFwdParams p;
  p.x = x;
  p.y = y;
  p.gate = gate;
  p.scale = scale;
  p.shift = shift;
  p.pre_weight = pre_weight;
  p.post_weight = post_weight;
  p.r = r;
  p.h = h;
  p.rows = (int64_t)cfg->batch * cfg->tokens;
  p.group_tokens = cfg->tokens / cfg->groups;
  p.by_group_tokens = fastvr::make_div((uint32_t)p.group_tokens);
  p.dim = cfg->dim;
  p.pre = cfg->pre;
  p.post = cfg->post;
  p.eps = cfg->eps;
  p.residual_scale = cfg->residual_scale;
  return fastvr::launch_norm_fwd(p, cfg->residual_dtype == FASTVR_F32,
                                 cfg->block_dtype == FASTVR_F32,
                                 fastvr::device_sms(),
                                 to_stream(stream)) == cudaSuccess
             ? FASTVR_OK
             : FASTVR_ERR_CUDA;
}

fastvr_status_t fastvr_gated_norm_bwd_scratch_bytes(
    const fastvr_norm_config_t* cfg, size_t* bytes) {
  if (!valid_norm(cfg) || bytes == nullptr) return FASTVR_ERR_INVALID_ARG;
  const BwdLayout l = norm_bwd_layout(*cfg);
  *bytes = l.partial + l.weights;
  return FASTVR_OK;
}

fastvr_status_t fastvr_gated_norm_bwd(
    const fastvr_norm_config_t* cfg, const void* dr, const void* dh,
    const void* r, const void* y, const float* gate, const float* scale,
    const float* pre_weight, const float* post_weight, void* dx, void* dy,
    float* dgate, float* dscale, float* dshift, float* dpre_weight,
    float* dpost_weight, void* scratch, size_t scratch_bytes,
    struct CUstream_st* stream) {
  if (!valid_norm(cfg) || (dr == nullptr && dh == nullptr) || r == nullptr ||
      dx == nullptr || (y == nullptr) != (dy == nullptr) || scratch == nullptr)
    return FASTVR_ERR_INVALID_ARG;
  const void* ptrs[] = {dr, dh, r, y, gate, scale, pre_weight, post_weight,
                        dx, dy, dgate, dscale, dshift, dpre_weight,
                        dpost_weight, scratch};
  for (const void* ptr : ptrs)
    if (!aligned16(ptr)) return FASTVR_ERR_INVALID_ARG;
  const BwdLayout l = norm_bwd_layout(*cfg);
  if (scratch_bytes < l.partial + l.weights) return FASTVR_ERR_CAPACITY;
  const fastvr_status_t st = fastvr::check_device();
  if (st != FASTVR_OK) return st;
  fastvr::NormBwdParams p;
  p.dr = dr;
  p.dh = dh;
  p.r = r;
  p.y = y;
  p.gate = gate;
  p.scale = scale;
  p.pre_weight = pre_weight;
  p.post_weight = post_weight;
  p.dx = dx;
  p.dy = dy;
  p.dgate = dgate;
  p.dscale = dscale;
  p.dshift = dshift;
  p.dpre_weight = dpre_weight;
  p.dpost_weight = dpost_weight;
  p.partial = static_cast<float*>(scratch);
  p.weight_partial = dpre_weight != nullptr || dpost_weight != nullptr
                         ? p.partial + l.partial / sizeof(float)
                         : nullptr;
  p.all_groups = (int64_t)cfg->batch * cfg->groups;
  p.group_tokens = cfg->tokens / cfg->groups;
  p.slices = l.split.slices;
  p.cta_groups = l.split.cta_groups;
  p.ctas = l.split.ctas;
  p.dim = cfg->dim;
  p.pre = cfg->pre;
  p.post = cfg->post;
  p.eps = cfg->eps;
  p.residual_scale = cfg->residual_scale;
  return fastvr::launch_norm_bwd(p, cfg->residual_dtype == FASTVR_F32,
                                 cfg->block_dtype == FASTVR_F32,
                                 to_stream(stream)) == cudaSuccess
             ? FASTVR_OK
             : FASTVR_ERR_CUDA;
}

fastvr_status_t fastvr_q4_cache_bytes(const fastvr_attn_config_t* cfg,
                                      int32_t kv_heads, size_t* bytes) {
  if (bytes == nullptr) return FASTVR_ERR_INVALID_ARG;
  Q4Layout l;
  const fastvr_status_t st = q4_layout(cfg, kv_heads, &l);
  if (st == FASTVR_OK) *bytes = l.cache;
  return st;
}

fastvr_status_t fastvr_q4_workspace_bytes(const fastvr_attn_config_t* cfg,
                                          int32_t kv_heads, size_t* bytes) {
  if (bytes == nullptr) return FASTVR_ERR_INVALID_ARG;
  Q4Layout l;
  const fastvr_status_t st = q4_layout(cfg, kv_heads, &l);
  if (st == FASTVR_OK) *bytes = l.workspace;
  return st;
}

fastvr_status_t fastvr_q4_plan(const fastvr_attn_config_t* cfg,
                               int32_t kv_heads, void* cache,
                               size_t cache_bytes, void* workspace,
                               size_t workspace_bytes, fastvr_plan_t* out) {
  if (out == nullptr) return FASTVR_ERR_INVALID_ARG;
  *out = nullptr;
  if (cache == nullptr || workspace == nullptr ||
      (((uintptr_t)cache | (uintptr_t)workspace) & 255u) != 0)
    return FASTVR_ERR_INVALID_ARG;
  Q4Layout l;
  const fastvr_status_t st = q4_layout(cfg, kv_heads, &l);
  if (st != FASTVR_OK) return st;
  if (cache_bytes < l.cache || workspace_bytes < l.workspace)
    return FASTVR_ERR_CAPACITY;
  fastvr_plan_s* p = new (std::nothrow) fastvr_plan_s();
  if (p == nullptr) return FASTVR_ERR_INVALID_ARG;
  p->cfg = *cfg;
  if (p->cfg.softmax_scale == 0.f)
    p->cfg.softmax_scale = 1.f / sqrtf((float)cfg->head_dim);
  if (p->cfg.window_chunks >= 0) p->cfg.max_chunks = 0;
  p->slots = l.slots;
  p->slot_tokens = l.slot_tokens;
  p->cache_tokens = l.cache_tokens;
  p->control_off = l.cache - kQ4ControlBytes;
  p->base = static_cast<char*>(cache);
  p->device = -1;
  p->q4 = true;
  p->kv_heads = kv_heads;
  p->code_bytes = l.codes;
  p->scale_bytes = l.scales;
  p->workspace = static_cast<char*>(workspace);
  *out = p;
  return FASTVR_OK;
}

fastvr_status_t fastvr_q4_append(fastvr_plan_t p, const void* k,
                                 const fastvr_strides_t* k_str, const void* v,
                                 const fastvr_strides_t* v_str, int32_t frames,
                                 struct CUstream_st* stream) {
  if (p == nullptr || !p->q4 || k == nullptr || v == nullptr || frames < 1 ||
      !aligned16(k) || !aligned16(v))
    return FASTVR_ERR_INVALID_ARG;
  const fastvr_attn_config_t& c = p->cfg;
  int64_t chunks = 1;
  if (frames > c.frames_per_chunk) {
    if (frames % c.frames_per_chunk != 0) return FASTVR_ERR_CAPACITY;
    chunks = frames / c.frames_per_chunk;
    if (chunks > p->slots) return FASTVR_ERR_CAPACITY;
  }
  if (p->chunks > 0 && p->last_frames < c.frames_per_chunk)
    return FASTVR_ERR_SEQUENCE;  // the stream already ended with a ragged chunk
  if (c.window_chunks < 0 && p->chunks + chunks > c.max_chunks)
    return FASTVR_ERR_CAPACITY;
  fastvr::Q4AppendParams a;
  memset(&a, 0, sizeof(a));
  const int64_t tokens = (int64_t)frames * c.tokens_per_frame;
  if (!get_strides(k_str, c.batch, tokens, p->kv_heads, c.head_dim, 2, false,
                   &a.k_str) ||
      !get_strides(v_str, c.batch, tokens, p->kv_heads, c.head_dim, 2, false,
                   &a.v_str))
    return FASTVR_ERR_INVALID_ARG;
  const fastvr_status_t st = ready(p, stream);
  if (st != FASTVR_OK) return st;
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.k_codes = reinterpret_cast<uint32_t*>(codes_of(p, false));
  a.v_codes = reinterpret_cast<uint32_t*>(codes_of(p, true));
  a.k_scales = reinterpret_cast<uint16_t*>(scales_of(p, false));
  a.v_scales = reinterpret_cast<uint16_t*>(scales_of(p, true));
  a.batch = c.batch;
  a.tokens = (int32_t)tokens;
  a.heads = p->kv_heads;
  a.head_dim = c.head_dim;
  a.cache_tokens = p->cache_tokens;
  a.first_row = p->chunks % p->slots * p->slot_tokens;
  a.code_words =
      (int64_t)c.batch * p->kv_heads * p->cache_tokens * c.head_dim / 8;
  a.status = fastvr::control_word(p);
  if (fastvr::launch_q4_append(a, fastvr::device_sms(), to_stream(stream)) !=
      cudaSuccess)
    return FASTVR_ERR_CUDA;
  p->launches += 1;
  p->chunks += chunks;
  p->last_frames = chunks > 1 ? c.frames_per_chunk : frames;
  return FASTVR_OK;
}

fastvr_status_t fastvr_q4_attn_fwd(fastvr_plan_t p, const void* q,
                                   const int32_t* first_chunk, void* out,
                                   float* lse, struct CUstream_st* stream) {
  if (p == nullptr || !p->q4 || q == nullptr || out == nullptr || q == out ||
      !aligned16(q) || !aligned16(out) || !aligned4(first_chunk) ||
      !aligned4(lse))
    return FASTVR_ERR_INVALID_ARG;
  if (p->chunks == 0) return FASTVR_ERR_SEQUENCE;
  const fastvr_status_t st = ready(p, stream);
  if (st != FASTVR_OK) return st;
  const fastvr_attn_config_t& c = p->cfg;
  // Visible chunks lo .. newest; their tokens lie in order in the cache from
  // the slot of chunk lo on, wrapping once.
  const int64_t newest = p->chunks - 1;
  const int64_t lo =
      c.window_chunks < 0 ? 0
                          : std::max<int64_t>(0, newest - c.window_chunks);
  fastvr::Q4AttnParams a;
  memset(&a, 0, sizeof(a));
  a.q = static_cast<const uint16_t*>(q);
  a.out = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.k_codes = codes_of(p, false);
  a.v_codes = codes_of(p, true);
  a.k_scales = scales_of(p, false);
  a.v_scales = scales_of(p, true);
  a.first_chunk = first_chunk;
  a.partial = reinterpret_cast<float*>(p->workspace);
  a.tickets = fastvr::control_word(p) + fastvr::kControlBytes / sizeof(int);
  a.batch = c.batch;
  a.heads = c.heads;
  a.kv_heads = p->kv_heads;
  a.head_dim = c.head_dim;
  a.q_tokens = p->last_frames * c.tokens_per_frame;
  a.group = c.heads / p->kv_heads;
  a.rows = a.q_tokens * a.group;
  a.cache_tokens = p->cache_tokens;
  a.first_row = lo % p->slots * p->slot_tokens;
  a.keys = (newest - lo) * p->slot_tokens + a.q_tokens;
  a.lo_chunk = lo;
  a.chunk_tokens = p->slot_tokens;
  a.scale_log2 = c.softmax_scale * 1.4426950408889634f;
  if (!fastvr::q4_direct(a.q_tokens, a.group))
    return attend_expanded(p, a, to_stream(stream)) == cudaSuccess
               ? FASTVR_OK
               : FASTVR_ERR_CUDA;
  if (fastvr::launch_q4_attn(a, fastvr::device_sms(), to_stream(stream)) !=
      cudaSuccess)
    return FASTVR_ERR_CUDA;
  p->launches += 1;
  return FASTVR_OK;
}

fastvr_status_t fastvr_q4_read(fastvr_plan_t p, int64_t chunk, void* k,
                               void* v, struct CUstream_st* stream) {
  if (p == nullptr || !p->q4 || k == nullptr || v == nullptr || chunk < 0 ||
      !aligned16(k) || !aligned16(v))
    return FASTVR_ERR_INVALID_ARG;
  if (chunk >= p->chunks || chunk < p->chunks - p->slots)
    return FASTVR_ERR_SEQUENCE;
  const fastvr_status_t st = ready(p, stream);
  if (st != FASTVR_OK) return st;
  fastvr::Q4ReadParams r;
  fill_read(p, &r);
  r.k_out = static_cast<uint16_t*>(k);
  r.v_out = static_cast<uint16_t*>(v);
  r.tokens = (chunk == p->chunks - 1 ? p->last_frames
                                     : p->cfg.frames_per_chunk) *
             p->cfg.tokens_per_frame;
  get_strides(nullptr, r.batch, r.tokens, r.heads, r.head_dim, 2, true,
              &r.out_str);
  r.first_row = chunk % p->slots * p->slot_tokens;
  if (fastvr::launch_q4_read(r, false, fastvr::device_sms(),
                             to_stream(stream)) != cudaSuccess)
    return FASTVR_ERR_CUDA;
  p->launches += 1;
  return FASTVR_OK;
}

}  // extern "C"
