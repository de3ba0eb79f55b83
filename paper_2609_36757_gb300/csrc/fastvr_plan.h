// The plan behind fastvr_plan_t and the host helpers that the entry points of
// both headers share.  Not part of the public ABI.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "../../include/fastvr_block.h"
#include "fastvr_internal.h"

struct fastvr_plan_s {
  fastvr_attn_config_t cfg;
  int64_t slots;         // S
  int64_t slot_tokens;   // k * N
  int64_t cache_tokens;  // S * k * N per head
  size_t kv_bytes;       // bytes of the K region (= the V region); bfloat16
                         // plans only
  size_t control_off;    // byte offset of the control block in the buffer
  char* base;            // caller's cache buffer
  int64_t chunks;        // chunks appended since the last reset
  int32_t last_frames;   // frames of the newest chunk
  bool device_ready;
  int device;
  int64_t launches;        // kernels enqueued since creation
  int32_t inject_stall;    // failure-detection test hook
  uint64_t wait_limit_ns;  // 0 = kernel default
  int64_t append_shift;    // debug builds: next append's destination shift
  // 4-bit plans (fastvr_q4_plan)
  bool q4;
  int32_t kv_heads;
  size_t code_bytes, scale_bytes;  // one region each of K and of V
  char* workspace;
};

namespace fastvr {

constexpr size_t kControlBytes = 256;

bool valid_config(const fastvr_attn_config_t* c);
inline bool supported_dim(int d) { return d == 64 || d == 128; }
int64_t num_slots(const fastvr_attn_config_t& c);
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

inline int* control_word(const fastvr_plan_s* p) {
  return reinterpret_cast<int*>(p->base + p->control_off);
}

// First device call of a plan: checks the device and the buffer, clears the
// control block (control_bytes of it) on the stream.  A 4-bit plan's first call
// cannot be captured (SEQUENCE).
fastvr_status_t ensure_device(fastvr_plan_s* p, size_t control_bytes,
                              struct CUstream_st* stream);

// FASTVR_OK when the current device is sm_103.
fastvr_status_t check_device();

// SM count of the current device, asked from the runtime on every call.
int device_sms();

// The failure-detection hook of the calls without a plan.
void noplan_debug(int32_t* stall, uint64_t* wait_limit_ns);

inline bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
inline cudaStream_t to_stream(struct CUstream_st* s) {
  return reinterpret_cast<cudaStream_t>(s);
}

// a * b, or -1 when it does not fit (or a factor already did not).
inline int64_t mul(int64_t a, int64_t b) {
  int64_t r;
  return a < 0 || b < 0 || __builtin_mul_overflow(a, b, &r) ? -1 : r;
}

// Strides in elements that keep every head 16-byte aligned; those of a
// dimension of one entry do not matter.  A tensor that is written may not have
// several entries in one place.
bool get_strides(const fastvr_strides_t* s, int64_t batch, int64_t tokens,
                 int64_t heads, int64_t d, int elem_bytes, bool written,
                 Strides* out);

}  // namespace fastvr
