// The pool's host side: its state, and what the files of entry points share.  Not part of the
// public ABI.
#pragma once

#include "../../include/fastcache.h"
#include "fc_internal.h"

#include <stddef.h>
#include <stdint.h>

#include <vector>

namespace fc {
// Sets the calling thread's error text (fc_last_error) and returns `code`.
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
constexpr int kProfRing = 32;
// Descriptors of a call to the pool's buffer on the device (*out): through pinned memory, in a
// captured call as kernel arguments (FC_EINVAL there if the buffer would have to grow).
int meta_to_device(fc_pool* pool, const void* image, size_t bytes, const void** out, hipStream_t stream);
}  // namespace fc

#define FC_HIP(call)                                                            \
  do {                                                                          \
    hipError_t e_ = (call);                                                     \
    if (e_ != hipSuccess)                                                       \
      return fail(FC_EDEVICE, "%s failed: %s", #call, hipGetErrorString(e_));   \
  } while (0)

// The calls of a launch sequence change the pool on the device step by step;
// if one of them fails after the first has been queued, the device state and
// the host mirrors no longer agree.  The pool is then marked and every later
// call on it is refused.
#define FC_HIP_STAGE(pool, call)                                                    \
  do {                                                                              \
    hipError_t e_ = (call);                                                         \
    if (e_ != hipSuccess) {                                                         \
      (pool)->poisoned = true;                                                      \
      return fail(FC_EDEVICE, "%s failed: %s; the pool is now unusable", #call,     \
                  hipGetErrorString(e_));                                           \
    }                                                                               \
  } while (0)

#define FC_CHECK_POOL(pool)                                                         \
  do {                                                                              \
    if (!(pool)) return fail(FC_EINVAL, "pool is NULL");                            \
    if ((pool)->poisoned)                                                           \
      return fail(FC_EDEVICE, "a device error in an earlier call left this pool in an " \
                              "undefined state; destroy it");                       \
  } while (0)

// Entry points that read or write fp16 rows only.
#define FC_CHECK_F16(pool, what)                                                    \
  do {                                                                              \
    if ((pool)->dtype != FC_DTYPE_F16)                                              \
      return fail(FC_EINVAL, "%s takes a pool of FC_DTYPE_F16", what);              \
  } while (0)

namespace fc {
// A device buffer that calls share and that grows on demand.  captured: a graph's replays use it;
// what replaces it then leaves it to the pool, to be freed with it.
template <typename T>
struct Scratch {
  T* data = nullptr;
  size_t cap = 0;  // elements
  bool captured = false;
};
}  // namespace fc

struct fc_pool {
  _Float16* kv = nullptr;    // (an 8-bit pool's bytes: see dtype)
  int dtype = FC_DTYPE_F16;
  size_t kv_bytes = 0;
  int n_blocks = 0, n_layers = 0, n_heads = 0, head_dim = 0;
  int32_t* stack = nullptr;  // device
  int top = 0;               // host mirror, exact
  bool poisoned = false;     // a launch failed in the middle of a stage: device and host disagree
  unsigned char* fixed_scratch = nullptr;  // this device's copy of the file-scope scratch array
  // ownership checks (debug mode): one int per block, 0 free, 1 handed out, 2 being released
  bool debug_checks = false;
  int32_t* owner = nullptr;
  int32_t* check_word = nullptr;  // device: what the last release check found

  // scratch, grown on demand
  fc::Scratch<float> raw_scores;
  fc::Scratch<int32_t> kept;
  size_t split_refused = ~(size_t)0;  // least score scratch of split heads that could not be had
  fc::Scratch<int32_t> ids;  // old ids then new ids
  std::vector<void*> retired;  // buffers that graphs use and calls do not any more
  char* dev_meta = nullptr;
  char* host_meta = nullptr;  // pinned
  size_t meta_cap = 0;
  bool meta_captured = false;       // a graph writes and reads dev_meta
  std::vector<char*> meta_retired;  // earlier ones that graphs use, freed with the pool
  hipEvent_t meta_event = nullptr;
  bool meta_pending = false;

  int n_cu = 0;                   // compute units of the pool's device
  float* decode_partial = nullptr;  // states of the segments of a split attention, ...
  int max_states = 0;               // ... and how many it holds
  int32_t* error_flag = nullptr;  // device, one int, zero unless a kernel found something wrong
  int32_t* arrivals = nullptr;    // device, the int after it: zero between calls (BatchParams)
  int score_mode = FC_SCORE_AUTO;
  bool score_pruning = true;       // the fused kernel prunes the second pass of SnapKV units
  int n_sink = 4;
  int compact_mode = FC_COMPACT_FRESH;
  // chunk-MLP compressor weights in operand order (library-owned)
  int mlp_k = 0, mlp_hidden = 0, mlp_activation = 0;
  _Float16* mlp_w1p[2] = {nullptr, nullptr};
  _Float16* mlp_w2p[2] = {nullptr, nullptr};
  float* mlp_b1[2] = {nullptr, nullptr};
  float* mlp_b2[2] = {nullptr, nullptr};
  bool mlp_captured = false;  // a graph reads them

  bool profiling = false;
  // event ring: the last kProfRing profiled calls, [call][kernel][start, stop]
  hipEvent_t ev[fc::kProfRing][fc::K_COUNT][2] = {};
  bool timed[fc::kProfRing][fc::K_COUNT] = {};
  int prof_calls = 0;  // profiled calls since profiling was last switched on
};
