// Host side of the cross attention and the gated feed-forward: the C ABI
// declared in include/fastvr_block.h.  Argument checks and scratch layouts;
// the device work is in cross_attn.cu, cross_attn_bwd.cu and gated_ffn.cu.
#include <cuda_runtime.h>
#include <math.h>
#include <string.h>

#include <atomic>
#include <mutex>

#include "fastvr_internal.h"
#include "fastvr_plan.h"

bool fastvr::get_strides(const fastvr_strides_t* s, int64_t batch,
                         int64_t tokens, int64_t heads, int64_t d,
                         int elem_bytes, bool written, Strides* out) {
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

namespace {

using fastvr::aligned16;
using fastvr::aligned4;
using fastvr::mul;
using fastvr::to_stream;

// The current device: what the calls ask of it, found once.
constexpr int kMaxDevices = 64;
struct Device {
  std::atomic<bool> ready;
  int sms;
  int* word;
};
Device g_devices[kMaxDevices];
std::mutex g_devices_mutex;

template <class Args>
fastvr_status_t use_device(Args* a) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return FASTVR_ERR_CUDA;
  a->device = dev;
  if (dev < 0 || dev >= kMaxDevices) {
    a->sms = fastvr::device_sms();
    a->status = nullptr;
    return fastvr::check_device();
  }
  Device& d = g_devices[dev];
  if (!d.ready.load(std::memory_order_acquire)) {
    std::lock_guard<std::mutex> lock(g_devices_mutex);
    const fastvr_status_t st = fastvr::check_device();
    if (st != FASTVR_OK) return st;
    d.sms = fastvr::device_sms();
    d.word = fastvr::device_status_word();
    d.ready.store(true, std::memory_order_release);
  }
  a->sms = d.sms;
  a->status = d.word;
  return FASTVR_OK;
}

fastvr_status_t check_cross(const fastvr_cross_config_t* c) {
  if (c == nullptr || c->batch < 1 || c->q_tokens < 1 || c->kv_tokens < 1 ||
      c->heads < 1 || c->kv_heads < 1 || c->heads % c->kv_heads != 0 ||
      c->head_dim < 1 || !(c->softmax_scale >= 0.f) ||
      !isfinite(c->softmax_scale))
    return FASTVR_ERR_INVALID_ARG;
  if (!fastvr::supported_dim(c->head_dim)) return FASTVR_ERR_UNSUPPORTED;
  // Tokens, and units of work (a unit has at least one row), are counted in
  // 32 bits; a tensor's elements and the rows of lse in 64.
  const int64_t heads = mul(c->batch, c->heads);
  const int64_t most = c->q_tokens > c->kv_tokens ? c->q_tokens : c->kv_tokens;
  if (c->q_tokens > INT32_MAX / 2 || c->kv_tokens > INT32_MAX / 2 ||
      heads < 0 || mul(heads, (most + 127) / 128) < 0 ||
      mul(heads, (most + 127) / 128) > INT32_MAX / 4)
    return FASTVR_ERR_INVALID_ARG;
  return FASTVR_OK;
}

// One tensor [batch, tokens, heads, d]: its pointer and strides.  A tile's
// copy takes byte strides below 2^40 and none that are negative; an input's
// batch stride may be 0.
bool check_tensor(const fastvr_cross_config_t& c, const void* p,
                  const fastvr_strides_t* s, bool q, bool written,
                  fastvr::Strides* out) {
  const int64_t tokens = q ? c.q_tokens : c.kv_tokens;
  const int64_t heads = q ? c.heads : c.kv_heads;
  if (p == nullptr || !aligned16(p) ||
      !fastvr::get_strides(s, c.batch, tokens, heads, c.head_dim, 2, written,
                           out))
    return false;
  const int64_t lim = (int64_t)1 << 39;
  if (out->batch < 0 || out->token < 0 || out->head < 0 || out->batch >= lim ||
      out->token >= lim || out->head >= lim)
    return false;
  return (tokens == 1 || out->token > 0) && (heads == 1 || out->head > 0);
}

fastvr::CrossArgs cross_args(const fastvr_cross_config_t& c) {
  fastvr::CrossArgs a;
  memset(&a, 0, sizeof(a));
  a.batch = c.batch;
  a.heads = c.heads;
  a.kv_heads = c.kv_heads;
  a.head_dim = c.head_dim;
  a.q_tokens = c.q_tokens;
  a.kv_tokens = c.kv_tokens;
  a.scale = c.softmax_scale == 0.f ? 1.f / sqrtf((float)c.head_dim)
                                   : c.softmax_scale;
  fastvr::noplan_debug(&a.inject_stall, &a.wait_limit_ns);
  return a;
}

bool valid_ffn(const fastvr_ffn_config_t* c) {
  // A weight's sum runs over all tokens within one bounded wait.
  return c != nullptr && c->tokens >= 1 && c->tokens <= 1 << 28 &&
         c->dim >= 8 && c->dim <= 65536 && c->dim % 8 == 0 && c->hidden >= 8 &&
         c->hidden <= 262144 && c->hidden % 8 == 0 &&
         // tiles are counted in 32 bits
         mul(c->tokens, c->dim > c->hidden ? c->dim : c->hidden) <=
             (int64_t)1 << 44 &&
         c->activation >= FASTVR_ACT_SILU &&
         c->activation <= FASTVR_ACT_GELU_TANH;
}

fastvr_status_t ffn_args(const fastvr_ffn_config_t* c, const void* x,
                         int64_t x_row, const void* w_gate, const void* w_up,
                         fastvr::FfnArgs* a) {
  memset(a, 0, sizeof(*a));
  if (!valid_ffn(c) || x == nullptr || w_gate == nullptr || w_up == nullptr ||
      !aligned16(x) || !aligned16(w_gate) || !aligned16(w_up))
    return FASTVR_ERR_INVALID_ARG;
  if (x_row == 0) x_row = c->dim;
  if (x_row < c->dim || x_row % 8 != 0 || x_row >= ((int64_t)1 << 39))
    return FASTVR_ERR_INVALID_ARG;
  a->x = static_cast<const uint16_t*>(x);
  a->x_row = x_row;
  a->w_gate = static_cast<const uint16_t*>(w_gate);
  a->w_up = static_cast<const uint16_t*>(w_up);
  a->tokens = c->tokens;
  a->dim = c->dim;
  a->hidden = c->hidden;
  a->act = c->activation;
  fastvr::noplan_debug(&a->inject_stall, &a->wait_limit_ns);
  return FASTVR_OK;
}

size_t ffn_region(const fastvr_ffn_config_t& c) {
  return ((size_t)c.tokens * c.hidden * 2 + 255) / 256 * 256;
}

}  // namespace

extern "C" {

fastvr_status_t fastvr_cross_attn_fwd(
    const fastvr_cross_config_t* cfg, const void* q,
    const fastvr_strides_t* q_str, const void* k,
    const fastvr_strides_t* k_str, const void* v,
    const fastvr_strides_t* v_str, const int32_t* kv_len, void* out,
    const fastvr_strides_t* out_str, float* lse, struct CUstream_st* stream) {
  const fastvr_status_t ok = check_cross(cfg);
  if (ok != FASTVR_OK) return ok;
  fastvr::CrossArgs a = cross_args(*cfg);
  if (!check_tensor(*cfg, q, q_str, true, false, &a.q_str) ||
      !check_tensor(*cfg, k, k_str, false, false, &a.k_str) ||
      !check_tensor(*cfg, v, v_str, false, false, &a.v_str) ||
      !check_tensor(*cfg, out, out_str, true, true, &a.o_str) ||
      !aligned4(kv_len) || !aligned4(lse) || out == q || out == k ||
      out == v || out == lse)
    return FASTVR_ERR_INVALID_ARG;
  const fastvr_status_t st = use_device(&a);
  if (st != FASTVR_OK) return st;
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(k);
  a.v = static_cast<const uint16_t*>(v);
  a.o = static_cast<uint16_t*>(out);
  a.lse = lse;
  a.kv_len = kv_len;
  return fastvr::launch_cross_attn(a, to_stream(stream)) == cudaSuccess
             ? FASTVR_OK
             : FASTVR_ERR_CUDA;
}

fastvr_status_t fastvr_cross_attn_bwd_scratch_bytes(
    const fastvr_cross_config_t* cfg, size_t* bytes) {
  if (bytes == nullptr) return FASTVR_ERR_INVALID_ARG;
  const fastvr_status_t st = check_cross(cfg);
  if (st != FASTVR_OK) return st;
  *bytes = fastvr::cross_bwd_scratch_floats(cfg->batch, cfg->heads,
                                            cfg->kv_heads, cfg->head_dim,
                                            cfg->q_tokens, cfg->kv_tokens) *
           sizeof(float);
  return FASTVR_OK;
}

fastvr_status_t fastvr_cross_attn_bwd(
    const fastvr_cross_config_t* cfg, const void* q,
    const fastvr_strides_t* q_str, const void* k,
    const fastvr_strides_t* k_str, const void* v,
    const fastvr_strides_t* v_str, const int32_t* kv_len, const void* out,
    const fastvr_strides_t* out_str, const void* dout,
    const fastvr_strides_t* dout_str, const float* lse, void* dq,
    const fastvr_strides_t* dq_str, void* dk, const fastvr_strides_t* dk_str,
    void* dv, const fastvr_strides_t* dv_str, void* scratch,
    size_t scratch_bytes, struct CUstream_st* stream) {
  const fastvr_status_t ok = check_cross(cfg);
  if (ok != FASTVR_OK) return ok;
  fastvr::CrossBwdArgs a;
  memset(&a, 0, sizeof(a));
  a.f = cross_args(*cfg);
  if (!check_tensor(*cfg, q, q_str, true, false, &a.f.q_str) ||
      !check_tensor(*cfg, k, k_str, false, false, &a.f.k_str) ||
      !check_tensor(*cfg, v, v_str, false, false, &a.f.v_str) ||
      !check_tensor(*cfg, out, out_str, true, false, &a.f.o_str) ||
      !check_tensor(*cfg, dout, dout_str, true, false, &a.dout_str) ||
      !check_tensor(*cfg, dq, dq_str, true, true, &a.dq_str) ||
      !check_tensor(*cfg, dk, dk_str, false, true, &a.dk_str) ||
      !check_tensor(*cfg, dv, dv_str, false, true, &a.dv_str) ||
      !aligned4(kv_len) || lse == nullptr || !aligned4(lse) ||
      scratch == nullptr || !aligned16(scratch))
    return FASTVR_ERR_INVALID_ARG;
  for (const void* p : {q, k, v, out, dout, (const void*)lse})
    if (p == scratch) return FASTVR_ERR_INVALID_ARG;
  for (const void* p : {q, k, v, out, dout, (const void*)lse,
                        (const void*)scratch})
    if (p == dq || p == dk || p == dv) return FASTVR_ERR_INVALID_ARG;
  if (dq == dk || dq == dv || dk == dv) return FASTVR_ERR_INVALID_ARG;
  if (scratch_bytes / sizeof(float) <
      fastvr::cross_bwd_scratch_floats(cfg->batch, cfg->heads, cfg->kv_heads,
                                       cfg->head_dim, cfg->q_tokens,
                                       cfg->kv_tokens))
    return FASTVR_ERR_CAPACITY;
  const fastvr_status_t st = use_device(&a.f);
  if (st != FASTVR_OK) return st;
  a.f.q = static_cast<const uint16_t*>(q);
  a.f.k = static_cast<const uint16_t*>(k);
  a.f.v = static_cast<const uint16_t*>(v);
  a.f.o = static_cast<uint16_t*>(const_cast<void*>(out));
  a.f.lse = const_cast<float*>(lse);
  a.f.kv_len = kv_len;
  a.dout = static_cast<const uint16_t*>(dout);
  a.dq = static_cast<uint16_t*>(dq);
  a.dk = static_cast<uint16_t*>(dk);
  a.dv = static_cast<uint16_t*>(dv);
  a.scratch = static_cast<float*>(scratch);
  return fastvr::launch_cross_attn_bwd(a, to_stream(stream)) == cudaSuccess
             ? FASTVR_OK
             : FASTVR_ERR_CUDA;
}

fastvr_status_t fastvr_gated_ffn_fwd(const fastvr_ffn_config_t* cfg,
                                     const void* x, int64_t x_row,
                                     const void* w_gate, const void* w_up,
                                     void* h, void* g, void* u,
                                     struct CUstream_st* stream) {
  fastvr::FfnArgs a;
  const fastvr_status_t ok = ffn_args(cfg, x, x_row, w_gate, w_up, &a);
  if (ok != FASTVR_OK) return ok;
  if (h == nullptr || (g == nullptr) != (u == nullptr) || !aligned16(h) ||
      !aligned16(g) || !aligned16(u) || h == g || h == u ||
      (g != nullptr && g == u))
    return FASTVR_ERR_INVALID_ARG;
  const void* in[] = {x, w_gate, w_up};
  for (const void* p : in)
    if (p == h || p == g || p == u) return FASTVR_ERR_INVALID_ARG;
  const fastvr_status_t st = use_device(&a);
  if (st != FASTVR_OK) return st;
  a.h = static_cast<uint16_t*>(h);
  a.g = static_cast<uint16_t*>(g);
  a.u = static_cast<uint16_t*>(u);
  return fastvr::launch_ffn_fwd(a, to_stream(stream)) == cudaSuccess
             ? FASTVR_OK
             : FASTVR_ERR_CUDA;
}

fastvr_status_t fastvr_gated_ffn_bwd_scratch_bytes(
    const fastvr_ffn_config_t* cfg, size_t* bytes) {
  if (!valid_ffn(cfg) || bytes == nullptr) return FASTVR_ERR_INVALID_ARG;
  *bytes = 2 * ffn_region(*cfg);
  return FASTVR_OK;
}

fastvr_status_t fastvr_gated_ffn_bwd(
    const fastvr_ffn_config_t* cfg, const void* dh, const void* x,
    int64_t x_row, const void* w_gate, const void* w_up, const void* g,
    const void* u, void* dx, void* dw_gate, void* dw_up, void* scratch,
    size_t scratch_bytes, struct CUstream_st* stream) {
  fastvr::FfnBwdArgs a;
  memset(&a, 0, sizeof(a));
  const fastvr_status_t ok = ffn_args(cfg, x, x_row, w_gate, w_up, &a.f);
  if (ok != FASTVR_OK) return ok;
  if (dh == nullptr || g == nullptr || u == nullptr || dx == nullptr ||
      scratch == nullptr || (dw_gate == nullptr) != (dw_up == nullptr) ||
      !aligned16(dh) || !aligned16(g) || !aligned16(u) || !aligned16(dx) ||
      !aligned16(dw_gate) || !aligned16(dw_up) || !aligned16(scratch) ||
      dx == dw_gate || dx == dw_up || (dw_gate != nullptr && dw_gate == dw_up))
    return FASTVR_ERR_INVALID_ARG;
  const void* in[] = {dh, x, w_gate, w_up, g, u, scratch};
  for (const void* p : in)
    if (p == dx || p == dw_gate || p == dw_up) return FASTVR_ERR_INVALID_ARG;
  for (const void* p : {dh, x, w_gate, w_up, g, u})
    if (p == scratch) return FASTVR_ERR_INVALID_ARG;
  if (scratch_bytes < 2 * ffn_region(*cfg)) return FASTVR_ERR_CAPACITY;
  const fastvr_status_t st = use_device(&a.f);
  if (st != FASTVR_OK) return st;
  a.f.g = static_cast<uint16_t*>(const_cast<void*>(g));
  a.f.u = static_cast<uint16_t*>(const_cast<void*>(u));
  a.dh = static_cast<const uint16_t*>(dh);
  a.dx = static_cast<uint16_t*>(dx);
  a.dw_gate = static_cast<uint16_t*>(dw_gate);
  a.dw_up = static_cast<uint16_t*>(dw_up);
  a.dg = static_cast<uint16_t*>(scratch);
  a.du = reinterpret_cast<uint16_t*>(static_cast<char*>(scratch) +
                                     ffn_region(*cfg));
  return fastvr::launch_ffn_bwd(a, to_stream(stream)) == cudaSuccess
             ? FASTVR_OK
             : FASTVR_ERR_CUDA;
}

}  // extern "C"
